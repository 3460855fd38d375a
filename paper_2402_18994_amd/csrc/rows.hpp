// Rows of a time-major tensor as the kernels of the gated block take them: VEC neighbouring channels a lane, the row's address
// scalar, a lane without a place of its own at an offset where the hardware drops the access.  gfx950 only.
#pragma once
#include "common.hpp"
#include "seq_common.hpp"

namespace snn {

constexpr int ROW_SPAN = 0x7FFF0000, ROW_NOWHERE = 0x7FFFFF00;     // lane offsets that exist stay below the first

template <typename T, int VEC> __device__ __forceinline__ Pack<T, VEC> row_load(const T *row, int at) {
  using Packed = Pack<T, VEC>;
  const rsrc_t r = make_rsrc(row, ROW_SPAN);
  if constexpr (sizeof(T) * VEC == 16) return __builtin_bit_cast(Packed, ld_b128(r, at, 0));
  else if constexpr (sizeof(T) * VEC == 8) return __builtin_bit_cast(Packed, ld_b64(r, at, 0));
  else if constexpr (sizeof(T) * VEC == 4) return __builtin_bit_cast(Packed, ld_b32(r, at, 0));
  else return __builtin_bit_cast(Packed, (unsigned short)__builtin_amdgcn_raw_buffer_load_b16(r, at, 0, 0));
}
template <typename T, int VEC> __device__ __forceinline__ void row_store(T *row, int at, Pack<T, VEC> v) {
  const rsrc_t r = make_rsrc(row, ROW_SPAN);
  if constexpr (sizeof(T) * VEC == 16) st_b128(r, at, 0, __builtin_bit_cast(u32x4, v));
  else if constexpr (sizeof(T) * VEC == 8) st_b64(r, at, 0, __builtin_bit_cast(u32x2, v));
  else if constexpr (sizeof(T) * VEC == 4) st_b32(r, at, 0, __builtin_bit_cast(uint32_t, v));
  else st_b16(r, at, 0, __builtin_bit_cast(unsigned short, v));
}

// v of this lane and of the one 16 (32) lanes away, added: the halves of two copies change places.
__device__ __forceinline__ float add_16_apart(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float add_32_apart(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

}  // namespace snn

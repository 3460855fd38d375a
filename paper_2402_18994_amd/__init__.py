"""MI355X-native surrogate-gradient BPTT for layered LIF spiking networks.

The package is a thin ctypes binding over the C ABI declared in include/snn.h and
include/snn_ops.h (libsnn_hip.so, built from csrc/ by build.py).  Every step of the training path
runs in the library's HIP kernels; Python only marshals arguments.
"""
from .binding import (SNN, SnnError, load_library, library_path, SURROGATES, PRECISIONS,  # noqa: F401
                      TENSORS, STEPS, KERNELS, OPTIONS, weight_grad_static)
from .ops import (AdamW, NetworkAdamW, causal_conv, causal_conv_backward, causal_conv_step, selective_scan,  # noqa: F401
                  selective_scan_backward, selective_scan_step, ConvGrads, ConvOutput, ScanGrads, ScanOutput)

"""NormPre optimizer step (arXiv 2609.36692) for AMD MI355X (gfx950).

The compute path is libnormpre.so (hand-written HIP kernels behind the C ABI of
include/normpre.h); ``normpre`` is its ctypes binding and ``workloads`` draws
seeded synthetic inputs.  ``train_ops`` holds the training-step operators around
the optimizer step (packed attention, 8-bit activation checkpoints).  Importing
the package does not load the library.
"""
__all__ = ["normpre", "train_ops", "workloads"]

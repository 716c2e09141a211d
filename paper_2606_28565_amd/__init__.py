"""MI355X (gfx950) batched kernel-latency evaluator of KernelSight-LM.

The product is libks.so (HIP kernels + C ABI, include/ks.h); ``abi`` is its
thin ctypes binding, ``fit`` a fit of gated heads with its calls."""

__all__ = ["abi", "build", "fit"]

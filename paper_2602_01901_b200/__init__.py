"""B200-native Lazy Attention / Q Cache decode path (arxiv 2602.01901).

The package holds the CUDA kernels and host runtime behind a C ABI (``csrc/``,
``include/qc.h`` at the repository root), a thin ctypes binding (``binding``), the
seeded synthetic workload generators (``workloads``), torch-owned buffers around the cache
(``session``) and the calls on a cache in 4 bits (``quant``).  Importing the package does not
load the native library; ``binding.load()`` does, and raises if it is missing.
"""

__all__ = ["binding", "workloads"]

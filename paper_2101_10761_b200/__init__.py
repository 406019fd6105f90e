"""SIDCo gradient sparsifier for B200 (sm_100a), with 4-bit products and
orthogonalised updates around it: CUDA kernels behind a C ABI, plus a thin
ctypes binding (and :mod:`paper_2101_10761_b200.training` on top of it).  Importing the package does not load the shared
library; the first call into :mod:`paper_2101_10761_b200.binding` does, and it
raises if the library has not been built."""

__all__ = ["binding", "exchange", "training", "workloads"]

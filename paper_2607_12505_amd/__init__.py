"""N:M sparse INT8 GEMM for AMD Instinct MI355X (gfx950).

The compute lives in ``libnmspmm.so`` (hand-written HIP kernels behind a C
ABI, declared in ``include/nmspmm.h``).  ``paper_2607_12505_amd.nmspmm`` is the
thin ctypes binding; ``paper_2607_12505_amd.nmblock`` binds the operators of a
transformer block around the GEMM.  Importing this package does not load the
library.
"""
__all__ = ["nmblock", "nmspmm", "workloads"]

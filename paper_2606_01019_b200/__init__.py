"""B200 (sm_100a) library for the per-step path of Hybrid Verified Decoding.

The package is a thin ctypes binding of ``libhvd_b200.so`` (built in-tree from ``csrc/`` by
``build.py``).  Every step of the path runs in the library's CUDA kernels; there is no CPU or
PyTorch fallback: importing works without a GPU (so the build can be checked), creating a context
does not.
"""
from .binding import (BF16, F16, F32, FREQ_MAX_OCC, NOALLOC_MAX_BATCH, NOALLOC_MAX_ROWS, REQ_BAD_LEN, REQ_BAD_PAGE, REQ_BAD_PATH,
                      REQ_CAPACITY, REQ_OK, ROPE_BANDS, ROPE_BASE, ROPE_HALVES, ROPE_LINEAR, ROPE_PAIRS, ROPE_PARTS, ROPE_PLAIN,
                      STATE_DTYPE, Context, HvdError, KvCache, exported_symbols, hvd_rope_frequencies,
                      hvd_verify_commit_noalloc, library_path, load_library)

__all__ = ["Context", "HvdError", "F32", "BF16", "REQ_OK", "REQ_CAPACITY", "REQ_BAD_LEN",
           "STATE_DTYPE", "exported_symbols", "library_path", "load_library", "hvd_verify_commit_noalloc",
           "NOALLOC_MAX_ROWS", "NOALLOC_MAX_BATCH", "FREQ_MAX_OCC", "F16", "REQ_BAD_PAGE", "REQ_BAD_PATH", "KvCache", "hvd_rope_frequencies",
           "ROPE_HALVES", "ROPE_PAIRS", "ROPE_PLAIN", "ROPE_LINEAR", "ROPE_BASE", "ROPE_PARTS", "ROPE_BANDS"]

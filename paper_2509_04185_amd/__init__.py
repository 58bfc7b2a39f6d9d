"""MI355X (gfx950) Set Block Decoding decode step: HIP kernels behind a C ABI (libsbd.so).

``Sbd`` wraps one library context; ``PageTable``, ``PagedKV``, ``scaled_quantize`` and
``scaled_matmul`` are the operators that need none.  See ``include/sbd.h`` for the semantics of
each call.
"""
from .binding import (LIB_PATH, SIGNATURES, ModelConfig, Sbd, SbdError, load_library,
                      make_config, status_string, workspace_bytes)
from .ops import PagedKV, PagedStep, PageTable, scaled_matmul, scaled_quantize
from .sampler import sample_blocks

__all__ = ["LIB_PATH", "SIGNATURES", "ModelConfig", "PageTable", "PagedKV", "PagedStep", "Sbd", "SbdError",
           "load_library", "make_config", "sample_blocks", "scaled_matmul", "scaled_quantize", "status_string",
           "workspace_bytes"]

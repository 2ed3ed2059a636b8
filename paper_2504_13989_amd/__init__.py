"""MI355X-native online Hadamard rotate-and-quantize (arXiv 2504.13989 hot path).

`binding` wraps the C ABI of librotq.so (HIP kernels for gfx950); `workloads` holds the
seeded synthetic input generators; `build` compiles the library in-tree.
"""
from . import workloads  # noqa: F401
from .binding import (Hadamard, KV4Cache, RotqError, dequantize_rotate, expand_limit, gbs_search, hadamard_build,  # noqa: F401
                      kv4_append, kv4_attention, kv4_cache, kv4_copy_pages, kv4_page_bytes, kv4_read, next_order,
                      quant_error, quant_error_workspace, quantize, quantize_asym, rotate, rotate_quantize,
                      rotate_quantize_asym)
from .pages import PagePool  # noqa: F401

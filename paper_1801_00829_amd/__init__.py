"""Python binding of libfuse: fused-operator templates (Cell, MAgg, Row, Outer) on MI355X.

Beside the templates: the operators of a transformer block (attention over packed sequences, the norms around a block,
the norm of all gradients with clipping, the norms of queries and keys per head with rotary positions, a cache in 8 bits
with attention over it), in bf16, fp16 and fp32 as well.

Only argument marshalling happens here; every step of a call runs in the HIP
kernels of ``libfuse.so`` (see ``include/fuse.h``).  PyTorch is used for device
memory and streams.
"""
from .api import (FuseError, Csr, fuse_cell, fuse_magg, fuse_magg_noalloc, fuse_row, fuse_outer,  # noqa: F401
                  fuse_cell_csr, fuse_magg_csr, check_csr, outer_left_prepare, outer_left_values, fuse_outer_left, prepare_cell_csr, prepare_magg_csr,
                  prepare_cell, prepare_magg, prepare_row, prepare_outer,
                  cache_stats, cache_clear, cache_disk_hits, last_source, last_kernel, probe_copy, probe_read, probe_gather,
                  AGG, SIDE, OPS, lib_path)
from .block_ops import (BlockGrads, fuse_block_norm, fuse_block_norm_backward, fuse_attention, fuse_attention_backward,  # noqa: F401
                        fuse_grad_norm, fuse_grad_clip, NORM, DTYPE)
from .head_ops import (Cache, RotaryGrads, fuse_qk_rotary, fuse_qk_rotary_backward, cache_new, fuse_cache_write,  # noqa: F401
                       fuse_attention_cache, PAIRS)

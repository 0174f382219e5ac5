"""CoSpec verify-and-arbitrate step on MI355X (gfx950).

The computation runs in libcospec.so (HIP kernels behind the C ABI of
include/cospec.h); `binding` marshals torch tensors into it, `workloads` draws
seeded synthetic inputs.
"""
from .binding import (CacheCall, CospecError, PagedCache, SplitBlock, arbitrate, cache_append, cache_keep,
                      hybrid_attention, hybrid_attention_paged, hybrid_mask, lib, prepare_block,
                      prepare_cache_append, prepare_cache_keep, prepare_hybrid_attention_paged, prepare_sps,
                      prepare_tree, prepare_tree_attention, sps_block, tree_attention, verify_block,
                      verify_block_static, verify_tree)

__all__ = ["CacheCall", "CospecError", "PagedCache", "SplitBlock", "arbitrate", "cache_append", "cache_keep",
           "hybrid_attention", "hybrid_attention_paged", "hybrid_mask", "lib", "prepare_block",
           "prepare_cache_append", "prepare_cache_keep", "prepare_hybrid_attention_paged", "prepare_sps",
           "prepare_tree", "prepare_tree_attention", "sps_block", "tree_attention", "verify_block",
           "verify_block_static", "verify_tree"]

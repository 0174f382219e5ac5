"""CoSpec verify-and-arbitrate step on MI355X (gfx950).

The computation runs in libcospec.so (HIP kernels behind the C ABI of
include/cospec.h); `binding` marshals torch tensors into it, `workloads` draws
seeded synthetic inputs.
"""
from .binding import (CacheCall, CospecError, LatentCache, PagePool, PagedCache, PoolCall, SplitBlock,
                      arbitrate, cache_append, cache_keep, expanded_attention, hybrid_attention,
                      hybrid_attention_paged, hybrid_mask, latent_append, latent_attention, latent_keep,
                      latent_tree_attention, lib, pages_compact, pages_copy, pages_fork, pages_release,
                      pages_reserve, prepare_block, prepare_cache_append, prepare_cache_keep,
                      prepare_expanded_attention, prepare_hybrid_attention_paged, prepare_latent_append,
                      prepare_latent_attention, prepare_latent_keep, prepare_latent_tree_attention,
                      prepare_pages_compact, prepare_pages_copy, prepare_pages_fork, prepare_pages_release,
                      prepare_pages_reserve, prepare_sps, prepare_tree, prepare_tree_attention, sps_block,
                      tree_attention, verify_block, verify_block_static, verify_tree)

__all__ = ["CacheCall", "CospecError", "LatentCache", "PagePool", "PagedCache", "PoolCall", "SplitBlock",
           "arbitrate", "cache_append", "cache_keep", "expanded_attention", "hybrid_attention",
           "hybrid_attention_paged", "hybrid_mask", "latent_append", "latent_attention", "latent_keep",
           "latent_tree_attention", "lib", "pages_compact", "pages_copy", "pages_fork", "pages_release",
           "pages_reserve", "prepare_block", "prepare_cache_append", "prepare_cache_keep",
           "prepare_expanded_attention", "prepare_hybrid_attention_paged", "prepare_latent_append",
           "prepare_latent_attention", "prepare_latent_keep", "prepare_latent_tree_attention",
           "prepare_pages_compact", "prepare_pages_copy", "prepare_pages_fork", "prepare_pages_release",
           "prepare_pages_reserve", "prepare_sps", "prepare_tree", "prepare_tree_attention", "sps_block",
           "tree_attention", "verify_block", "verify_block_static", "verify_tree"]

"""Sharded layerwise QK-Norm for AMD MI355X: HIP kernels behind a C ABI.

The computation lives in ``libqkn.so`` (kernels in ``csrc/qkn_kernels.h`` and
``csrc/qkn_proj.hip``, entry points declared in ``include/qkn.h`` and
``include/qkn_proj.h``); ``_lib`` is its ctypes binding. Build with
``python -m paper_2608_09160_amd.build``.

Around the norm, what an attention block needs to serve: rotary positions with
the write into a paged cache (``csrc/qkn_rope.hip``), attention over that cache
(``csrc/qkn_attn*``) and low-rank adapters (``csrc/qkn_adapters.hip``), declared
in ``include/qkn_rope.h``, ``qkn_attn.h``, ``qkn_adapters.h`` and ``qkn_cache.h``;
``_serve`` is their binding, ``block`` runs them together. For long contexts the
cache may be held in 4 bits (``include/qkn_cache4.h``) and its pages be handed out
on the device (``include/qkn_pages.h``, binding ``_pages``).
"""
from ._lib import (QKN_EHIP, QKN_EINVAL, QKN_ENOTSUP, QKN_EOVERLAP, QKN_OK,  # noqa: F401
                   Prepared, PreparedApply, PreparedPartial, QknError, Seg, load, qkn_apply, qkn_full, qkn_fused_shard,
                   qkn_fused_group_wait, qkn_fused_shard_wait, qkn_last_launch, qkn_partial_sumsq,
                   qkn_publish_partials, qkn_set_option, qkn_strerror)
from ._serve import (AdapterSeg, KVCache, KVCache4, PreparedAdapters, PreparedAttn, PreparedCache4Load,  # noqa: F401
                     PreparedRopeCache, RopeSeg, qkn_adapters_add, qkn_attn, qkn_cache4_load, qkn_rope_cache,
                     qkn_rope_table)
from ._pages import (PageBook, PreparedPagesCompact, PreparedPagesCopy, PreparedPagesFork,  # noqa: F401
                     PreparedPagesFree, PreparedPagesGrow, qkn_pages_compact, qkn_pages_copy, qkn_pages_fork,
                     qkn_pages_free, qkn_pages_grow)

"""MI355X (gfx950) KV-block splice path of Nexus (arXiv 2608.20397).

Re-anchoring of rotary keys, splice into a paged KV cache and suffix-redecode causal GQA
attention, as hand-written HIP kernels behind the C ABI of ``include/nexus.h``
(``libnexus.so``); ``paper_2608_20397_amd.nexus`` is the thin Python binding.
"""
from . import nexus  # noqa: F401
from .nexus import (Block, PagedKVCache, NexusError, splice_pages, rephase_k,  # noqa: F401
                    rephase_k_paged, suffix_attn, suffix_attn_varlen, redecode_len,
                    check_page_table, lib, KV8Cache, kv8_append, kv8_append_step,  # noqa: F401
                    kv8_splice, kv8_read, kv8_suffix_attn, kv8_suffix_attn_varlen,  # noqa: F401
                    kv8_decode_attn)  # noqa: F401

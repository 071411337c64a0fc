"""PRESTO draft-to-verify round on MI355X (gfx950).

The four stages of a round run in the HIP kernels of ``libpresto.so``
(C ABI declared in ``include/presto.h``); this package holds those sources
(``csrc/``), their build (``build.py``) and a thin ctypes binding whose
functions carry the C names.
"""
from ._lib import (  # noqa: F401
    EXPORTS, PRESTO_DT_BF16, PRESTO_DT_F32, PRESTO_ERR_HIP, PRESTO_ERR_INVALID_ARG,
    PRESTO_ERR_UNSUPPORTED, PRESTO_ERR_WORKSPACE, PRESTO_FLAG_NAN_DRAFTER, PRESTO_FLAG_NAN_TARGET,
    PRESTO_FLAG_NGRAM_BAD, PRESTO_FLAG_NGRAM_FULL, PRESTO_FLAG_BAD_INDEX, PRESTO_FLAG_KV_COMMIT,
    PRESTO_CTX_PACKED, PRESTO_CTX_SLOTS, CommitDesc, presto_commit_kv, presto_flatten_slots,
    presto_select_slots, presto_topk_rows,
    PRESTO_OK, PRESTO_TREE_BEAM, PRESTO_TREE_BEST_FIRST, PRESTO_TREE_BEST_FIRST_ALG2, AttnDesc,
    PrestoError, TreeDesc, lib, presto_accept, presto_build_tree, presto_entropy_lambda, presto_ngram_clear,
    presto_ngram_gather, presto_ngram_insert, presto_ngram_table_bytes, presto_topk,
    presto_topk_noalloc,
    presto_tree_attention, topk_fallback_chunks, topk_workspace, version,
    PRESTO_FLAG_BAD_PAGE, PRESTO_FLAG_BAD_SEQ, PRESTO_FLAG_NO_PAGES, PagedAttnDesc, PagesDesc,
    PRESTO_DT_FP4, PRESTO_FLAG_NAN_LOGITS, PRESTO_ROPE_RAMP_LOG, PRESTO_ROPE_RAMP_NONE, PRESTO_ROPE_RAMP_TURNS,
    AppendDesc, RopeDesc, RopeFreqDesc,
)
from ._paged import (  # noqa: F401
    paged_attention_workspace, pages_workspace, presto_append_kv, presto_paged_attention,
    presto_pages_compact, presto_pages_fork, presto_pages_free, presto_pages_reserve,
    presto_pages_trim, presto_window_attention,
)
from ._step import (  # noqa: F401
    RopePlan, presto_append_rope, presto_quant_attention, presto_read_kv, presto_rope, presto_rope_steps,
    presto_sample, quant_attention_workspace, quant_pages, rope_plan, sample_workspace,
)

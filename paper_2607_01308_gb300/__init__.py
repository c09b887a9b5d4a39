"""GB300-native CanonicalMerge / LatentFragmentSet (arxiv 2607.01308).

The compute path is libcm.so: hand-written CUDA for sm_103a behind the C ABI of
include/cm.h. This package is its Python binding (ctypes). Importing it fails
loudly if the library has not been built; nothing here computes on the CPU.

    import paper_2607_01308_gb300 as cm
    ctx = cm.Context(device=0, rope_theta=1e6)
    S = cm.FragmentSet(ctx)
    fid, absorbed = S.ingest(K, V)          # Algorithm 2, Ingest
    n, order = S.render(k_out, v_out)       # Algorithm 2, Render (= Algorithm 1)

What decodes from a merged cache reads it in 8 bits (QCache, QBatch):

    cache = cm.QCache(ctx, num_blocks, 16, L, H, d)           # e4m3 codes, a scale per block and head
    batch = cm.QBatch(ctx, requests, table_width, max_rows, 16)
    batch.schedule(context_lens, new_lens, free_blocks)       # block tables and slots
    cache.append(k_out, v_out, batch.slot_map)                # the merged cache into its blocks
    batch.max_new = 1                                         # if no request brings more rows than this
    out, _ = cache.attend(q, batch, layer=0)                  # softmax(q K^T / sqrt(d)) V

and a drafter's trees of tokens are checked against it in one pass (QTree):

    tree = cm.QTree(batch, max_nodes=26)
    tree.plan(parents, context_lens)                          # ancestors and positions
    q, k = cm.rotate_qk(ctx, q, k, tree.positions, q_weight, k_weight)   # norm of each head, rotation
    out, _ = cache.attend(q, batch, layer=0, tree=tree)       # a row sees its context and its ancestors
    tree.verify(parents, tokens, target, accept, sample)      # the accepted path, the next token
    cache.keep(batch, tree, context_lens)                     # its rows to the front, blocks given back
"""
from ._binding import (  # noqa: F401
    CMError, Status, cm_id, cm_fragment, lib, LIB_PATH, EXPORTED,
    cm_abi_version, cm_status_string, cm_last_error_message,
    cm_context_create, cm_context_destroy, cm_context_check, cm_testing_bounds_violations,
    cm_set_create, cm_set_destroy,
    cm_fragment_id, cm_fragment_id_static, cm_ingest, cm_ingest_batch, cm_ingest_many,
    cm_render_many, cm_ingest_render, cm_render_job, cm_set_contains, cm_set_leq, ingest_many, render_many,
    cm_measure_int_alu, cm_context_set_render_warps, cm_context_set_overlap, cm_context_set_dedup_by_bytes,
    cm_context_set_timing, cm_context_kernel_times, cm_kernel_times, cm_union, cm_set_size, cm_set_seq_len, cm_set_ids,
    cm_render, cm_render_incremental, cm_render_paged, cm_paged_cache, cm_bagmerge,
    fragment_from_tensors, Context, FragmentSet,
    cm_qcache, cm_qcache_batch, cm_qcache_query, cm_qk_rows, cm_tree_drafts, CM_PROB_F32, CM_PROB_BF16,
    cm_qcache_tree, cm_qk_rotate, cm_qcache_attend_tree, cm_tree_verify, cm_qcache_keep,
    CM_QCACHE_CONTEXT_LENS, cm_qcache_schedule, cm_qcache_schedule_cut, cm_qcache_append, cm_qcache_attend, cm_qcache_workspace,
)
from .qcache import QBatch, QCache  # noqa: F401
from .tree import QTree, rotate_qk  # noqa: F401

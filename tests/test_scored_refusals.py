"""Arrays at odd addresses, and arrays that a call writes while it reads them: refused before anything is launched, without a GPU.  Nothing here
passes every check of a call."""
import ctypes as C

import pytest
import torch

import scored_ref as R
from paper_2403_20137_amd import kvbfp

D = 128
BAD, WS = kvbfp.ERR_INVALID_ARG, kvbfp.ERR_WORKSPACE
LAYOUT = kvbfp.make_layout(D, 32, 4, 2, 3, 512)
POOL = kvbfp.make_layout(D, 32, 4, 2, 20, 64)
SMALL = kvbfp.make_layout(D, 32, 4, 2, 3, 100)
PLANES = (0x10000000, 0x11000000, 0x12000000, 0x13000000)
OTHERS = (0x20000000, 0x21000000, 0x22000000, 0x23000000)
Q, OUT, LSE, W, W_OUT, LENS, TABLE, KEPT, NEW_LEN, SPACE = (0x30000000 + 0x1000000 * k for k in range(10))
PERM_K, PERM_V, SLOPES, FIRST, PREFIX, TREE, DST_TABLE = (0x40000000 + 0x1000000 * k for k in range(7))
HEADS, TOKENS, LEN = 8, 4, 512
ROWS = 3 * TOKENS * HEADS


def rule(**kw):
    r = kvbfp.make_score_rule(cap=1.0)
    r.slopes, r.first_dev, r.prefix_dev, r.tree_mask, r.tree_stride = SLOPES, FIRST, PREFIX, TREE, TOKENS
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def attend(paged=False, q=Q, out=OUT, lse=LSE, lens=LENS, table=TABLE, space=SPACE, perm_k=PERM_K, perm_v=PERM_V, **kw):
    need = kvbfp.scored_workspace_bytes(LAYOUT, HEADS, TOKENS, LEN)
    tail = (HEADS, TOKENS, q, kvbfp.BF16, lens, LEN, 0.1, perm_k, perm_v, C.byref(rule(**kw)), out, lse, space, need, None)
    cache = C.byref(kvbfp.CachePtrs(*PLANES))
    if paged:
        return kvbfp.lib().kvbfp_decode_attention_scored_paged(C.byref(POOL), cache, table, 8, 3, *tail)
    return kvbfp.lib().kvbfp_decode_attention_scored(C.byref(LAYOUT), cache, *tail)


def collect(paged=False, q=Q, lse=LSE, w=W, w_out=W_OUT, lens=LENS, table=TABLE, perm_k=PERM_K, decay=1.0, **kw):
    tail = (HEADS, TOKENS, q, kvbfp.BF16, lens, LEN, 0.1, perm_k, C.byref(rule(**kw)), lse, decay, w, w_out, 600, None)
    cache = C.byref(kvbfp.CachePtrs(*PLANES))
    if paged:
        return kvbfp.lib().kvbfp_accumulate_weights_paged(C.byref(POOL), cache, table, 8, 3, *tail)
    return kvbfp.lib().kvbfp_accumulate_weights(C.byref(LAYOUT), cache, *tail)


def evict(paged=False, to=OTHERS, w=W, lens=LENS, kept=KEPT, new_len=NEW_LEN, w_out=W_OUT, table=TABLE, dst_table=DST_TABLE):
    tail = (w, 600, lens, LEN, 100, 4, 10, kept, new_len, w_out, None)
    cache, dst = C.byref(kvbfp.CachePtrs(*PLANES)), C.byref(kvbfp.CachePtrs(*to))
    if paged:
        return kvbfp.lib().kvbfp_evict_paged(C.byref(POOL), cache, table, 8, 3, C.byref(POOL), dst, dst_table, 2, *tail)
    return kvbfp.lib().kvbfp_evict(C.byref(LAYOUT), cache, C.byref(SMALL), dst, *tail)


def refused(call, word, **kw):
    assert call(**kw) == BAD, kw
    assert word in kvbfp.last_error(), (kw, kvbfp.last_error())


@pytest.mark.parametrize("call,name,at", [
    (attend, "lse", LSE), (attend, "lens", LENS), (attend, "perm_k", PERM_K), (attend, "perm_v", PERM_V), (attend, "slopes", SLOPES),
    (attend, "first_dev", FIRST), (attend, "prefix_dev", PREFIX), (attend, "tree_mask", TREE), (attend, "tree_mask", TREE + 2),
    (collect, "lse", LSE), (collect, "w", W), (collect, "w_out", W_OUT), (collect, "lens", LENS), (collect, "tree_mask", TREE + 2),
    (evict, "w", W), (evict, "w_out", W_OUT), (evict, "kept", KEPT), (evict, "new_len", NEW_LEN), (evict, "lens", LENS)])
def test_odd_addresses(call, name, at):
    refused(call, "aligned", **{name: at + 2})


def test_odd_tables():
    refused(attend, "aligned", paged=True, table=TABLE + 1)
    refused(collect, "aligned", paged=True, table=TABLE + 1)
    refused(evict, "aligned", paged=True, table=TABLE + 2)
    refused(evict, "aligned", paged=True, dst_table=DST_TABLE + 2)


@pytest.mark.parametrize("paged", [False, True])
def test_attention_writes_nothing_that_it_reads(paged):
    size = 2 * ROWS * D
    for at in (Q + 2, Q - 2, Q + size - 2, Q - size + 2):                  # q itself may be the output, nothing beside it
        refused(attend, "overlap", paged=paged, out=at)
    for out in (LSE, SPACE, LENS, PERM_K, PERM_V, SLOPES, FIRST, PREFIX, TREE, *PLANES):
        refused(attend, "overlap", paged=paged, out=out)
    for lse in (Q, OUT, OUT + size - 4, SPACE, LENS, PERM_K, SLOPES, TREE + 8 * 3 * TOKENS - 4, PLANES[0] + 4, PLANES[1]):
        refused(attend, "overlap", paged=paged, lse=lse)
    for space in (Q, OUT, LSE, LENS, FIRST, TREE, PLANES[3]):
        refused(attend, "overlap", paged=paged, space=space)
    if paged:
        refused(attend, "overlap", paged=True, out=TABLE + 4 * 3 * 8 - 4)
        refused(attend, "overlap", paged=True, lse=TABLE)


@pytest.mark.parametrize("paged", [False, True])
def test_weights_write_nothing_that_they_read(paged):
    size = 4 * 3 * 2 * 600
    for w_out in (W + 4, W - 4, W + size - 4, Q, LSE, LSE + 4 * ROWS - 4, LENS, PERM_K, SLOPES, FIRST, PREFIX, TREE, PLANES[0], PLANES[1], Q - size + 4):
        refused(collect, "overlap", paged=paged, w_out=w_out)
    if paged:
        refused(collect, "overlap", paged=True, w_out=TABLE)


@pytest.mark.parametrize("paged", [False, True])
def test_eviction_writes_nothing_that_it_reads(paged):
    for name in ("kept", "new_len", "w_out"):
        for at in (W, W + 4 * 3 * 2 * 600 - 4, LENS, LENS + 8, *PLANES, *OTHERS):
            refused(evict, "overlap", paged=paged, **{name: at})
    refused(evict, "overlap", paged=paged, kept=NEW_LEN)
    refused(evict, "overlap", paged=paged, kept=W_OUT)
    refused(evict, "overlap", paged=paged, new_len=W_OUT + 4)
    for at in (W, LENS, KEPT, PLANES[0], PLANES[3]):                       # the cache that tokens go to
        refused(evict, "overlap", paged=paged, to=(at, *OTHERS[1:]))
    if paged:
        refused(evict, "overlap", paged=True, kept=TABLE)
        refused(evict, "overlap", paged=True, new_len=DST_TABLE + 4 * 3 * 2 - 4)
        refused(evict, "overlap", paged=True, to=PLANES, kept=PLANES[1])


@pytest.mark.gpu
@pytest.mark.parametrize("n,S", [(1, 90), (1, 3000), (20, 100), (20, 3000), (64, 3000)])
def test_the_queries_may_be_the_output(n, S):
    from test_gpu_scored import BF16, F32, run_case, tree
    for dtype in (F32, BF16):
        case = run_case(80 + n, 3, 2, 4, n, S, 4, 32, dtype, lens=[S, S // 2, 0], tree=tree(n, n), cap=20.0)
        q = case["q"].clone()
        lse = torch.empty_like(case["lse"])
        got = kvbfp.decode_attention_scored(case["cache"], q, S, case["scale"], case["rule"], seq_len_dev=case["lens"], out=q, lse=lse)
        assert got is q and torch.equal(q, case["out"]) and torch.equal(lse, case["lse"])
        w = torch.zeros(3, 2, S, device="cuda")
        kvbfp.accumulate_weights(case["cache"], case["q"], S, case["scale"], lse, w, w, rule=case["rule"], seq_len_dev=case["lens"])
        assert (R.f64(w)[2] == 0).all() and torch.isfinite(w).all()

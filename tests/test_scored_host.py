"""Refusals of the calls with a rule on the scores, of the weights and of the eviction: before anything is launched, without a GPU."""
import ctypes as C

import pytest
import torch

from paper_2403_20137_amd import kvbfp

FAKE = C.c_void_p(0x10000)
LAYOUT = kvbfp.make_layout(128, 32, 4, 2, 3, 512)
POOL = kvbfp.make_layout(128, 32, 4, 2, 20, 64)
PTRS = kvbfp.CachePtrs(0x100000, 0x200000, 0x300000, 0x400000)
OTHER = kvbfp.CachePtrs(0x1100000, 0x1200000, 0x1300000, 0x1400000)
OK_, BAD, UNS, WS = kvbfp.OK, kvbfp.ERR_INVALID_ARG, kvbfp.ERR_UNSUPPORTED, kvbfp.ERR_WORKSPACE


def rule(**kw):
    r = kvbfp.make_score_rule()
    for k, v in kw.items():
        setattr(r, k, v)
    return C.byref(r)


def attend(layout=LAYOUT, cache=PTRS, heads=8, tokens=4, q=FAKE, dtype=kvbfp.BF16, max_len=512, scale=0.1, r=None, out=FAKE, ws=None,
           ws_bytes=0, paged=None):
    tail = (heads, tokens, q, dtype, None, max_len, scale, None, None, r, out, None, ws, ws_bytes, None)
    if paged:
        return kvbfp.lib().kvbfp_decode_attention_scored_paged(C.byref(layout), C.byref(cache), *paged, *tail)
    return kvbfp.lib().kvbfp_decode_attention_scored(C.byref(layout), C.byref(cache), *tail)


def test_scored_attention_refusals():
    assert attend() == WS                                    # complete arguments reach the workspace check
    assert "workspace" in kvbfp.last_error()
    need = kvbfp.scored_workspace_bytes(LAYOUT, 8, 4, 512)
    assert need > 0 and attend(ws=FAKE, ws_bytes=need - 1) == WS
    assert attend(ws=C.c_void_p(0x10010), ws_bytes=need) == WS and "aligned" in kvbfp.last_error()
    assert attend(heads=7) == BAD
    assert attend(heads=0) == BAD
    assert attend(tokens=0) == BAD
    assert attend(tokens=65) == BAD and "n_q_tokens" in kvbfp.last_error()
    assert attend(q=None) == BAD
    assert attend(q=C.c_void_p(0x10001)) == BAD
    assert attend(out=None) == BAD
    assert attend(dtype=7) == BAD
    assert attend(max_len=0) == BAD and attend(max_len=513) == BAD
    assert attend(scale=float("nan")) == BAD and attend(scale=float("inf")) == BAD
    assert attend(scale=3e38) == BAD and attend(scale=-3e38) == BAD
    assert attend(cache=kvbfp.CachePtrs(0x100000, 0x200000, 0, 0)) == BAD
    assert attend(cache=kvbfp.CachePtrs(0x100008, 0x200000, 0x300000, 0x400000)) == BAD
    assert attend(layout=kvbfp.make_layout(64, 32, 4, 2, 3, 512)) == UNS
    assert attend(heads=2 * 600, tokens=64) == UNS


def test_rule_refusals():
    for bad in (dict(struct_bytes=8), dict(cap=-1.0), dict(cap=float("inf")), dict(cap=float("nan")), dict(cap=1e-45), dict(cap=3e38),
                dict(window=-1), dict(tree_mask=0x10000, tree_stride=3), dict(tree_mask=0x10000, tree_stride=-1)):
        assert attend(r=rule(**bad)) == BAD, bad
        assert "rule" in kvbfp.last_error()
    for good in (dict(), dict(cap=50.0), dict(window=2 ** 31 - 1), dict(tree_mask=0x10000, tree_stride=0), dict(tree_mask=0x10000, tree_stride=9)):
        assert attend(r=rule(**good)) == WS, good
    # the scale over the cap: 2e6 * 128 * 2.9 / 1e-30 is no fp32 number; 0.1 over it is one
    assert attend(r=rule(cap=1e-30), scale=2e6) == BAD and "cap" in kvbfp.last_error()
    assert attend(r=rule(cap=1e-30), scale=0.1) == WS and attend(r=rule(cap=1e-38)) == BAD


def test_paged_refusals():
    assert attend(layout=POOL, paged=(FAKE, 8, 3)) == WS
    assert attend(layout=POOL, paged=(None, 8, 3)) == BAD
    assert attend(layout=POOL, paged=(FAKE, 0, 3)) == BAD
    assert attend(layout=POOL, paged=(FAKE, 8, 0)) == BAD
    assert attend(layout=POOL, paged=(FAKE, 7, 3)) == BAD                   # 448 tokens a sequence
    assert attend(layout=kvbfp.make_layout(128, 32, 4, 2, 20, 48), paged=(FAKE, 20, 3)) == UNS
    assert kvbfp.scored_workspace_bytes_paged(POOL, 8, 3, 8, 4, 512) == kvbfp.scored_workspace_bytes(LAYOUT, 8, 4, 512)
    assert kvbfp.scored_workspace_bytes(LAYOUT, 7, 4, 512) == 0 and kvbfp.scored_workspace_bytes(LAYOUT, 8, 0, 512) == 0
    assert kvbfp.scored_workspace_bytes(LAYOUT, 8, 4, 513) == 0 and kvbfp.scored_workspace_bytes_paged(POOL, 0, 3, 8, 4, 512) == 0


def collect(layout=LAYOUT, cache=PTRS, heads=8, tokens=4, q=FAKE, max_len=512, lse=FAKE, decay=1.0, out=FAKE, stride=512, r=None, scale=0.1,
            before=None):
    return kvbfp.lib().kvbfp_accumulate_weights(C.byref(layout), C.byref(cache), heads, tokens, q, kvbfp.BF16, None, max_len, scale, None, r,
                                                lse, decay, before, out, stride, None)


def test_weights_refusals():
    for bad in (dict(lse=None), dict(out=None), dict(stride=511), dict(decay=float("nan")), dict(heads=3), dict(tokens=65), dict(q=None),
                dict(max_len=600), dict(cache=kvbfp.CachePtrs(0, 0x200000, 0, 0)), dict(r=rule(cap=-2.0)), dict(scale=float("nan"))):
        assert collect(**bad) == BAD, bad
    for shift in (4, -4, 3 * 2 * 512 * 4 - 4, 4 - 3 * 2 * 512 * 4):          # neither the same nor apart
        assert collect(out=C.c_void_p(0x1000000), before=C.c_void_p(0x1000000 + shift)) == BAD and "overlap" in kvbfp.last_error()


def test_workspace_grows_with_the_length():
    # a workspace for the longest call holds shorter ones, whatever way they are split
    for heads, batch, rows in ((2, 3, 512), (8, 70, 4096), (8, 8, 40000)):
        layout = kvbfp.make_layout(128, 32, 4, heads, batch, rows)
        for group, tokens in ((4, 1), (4, 5), (12, 5), (4, 32), (4, 64), (17, 8)):
            sizes = [kvbfp.scored_workspace_bytes(layout, heads * group, tokens, n) for n in range(1, rows + 1, 61)]
            assert sizes == sorted(sizes), (heads, batch, group, tokens)


def evict(src=LAYOUT, dst=kvbfp.make_layout(128, 32, 4, 2, 3, 100), cache=PTRS, to=OTHER, w=0x5000000, stride=512, lens=None, max_len=512, keep=100,
          first=4, recent=10, kept=0x6000000, new_len=0x7000000, w_out=None, paged=None):
    tail = (w, stride, lens, max_len, keep, first, recent, kept, new_len, w_out, None)
    if paged:
        table, table_stride, batch, dst_table, dst_stride = paged
        return kvbfp.lib().kvbfp_evict_paged(C.byref(src), C.byref(cache), table, table_stride, batch, C.byref(dst), C.byref(to), dst_table,
                                             dst_stride, *tail)
    return kvbfp.lib().kvbfp_evict(C.byref(src), C.byref(cache), C.byref(dst), C.byref(to), *tail)


def test_evict_refusals():
    small = lambda **kw: kvbfp.make_layout(**{**dict(head_dim=128, block=32, mant_bits=4, n_kv_heads=2, batch=3, max_seq=100), **kw})  # noqa: E731
    for bad in (dict(w=None), dict(kept=None), dict(new_len=None), dict(stride=511), dict(max_len=0), dict(max_len=513), dict(keep=0),
                dict(keep=101), dict(first=-1), dict(recent=-1), dict(first=60, recent=41), dict(first=2 ** 31 - 1, recent=2 ** 31 - 1),
                dict(to=kvbfp.CachePtrs(0x1100000, 0x1200000, 0, 0)), dict(cache=kvbfp.CachePtrs(0x100001, 0x200000, 0x300000, 0x400000)),
                dict(dst=small(block=16)), dict(dst=small(mant_bits=8)), dict(dst=small(n_kv_heads=1)), dict(dst=small(batch=2)),
                dict(to=PTRS), dict(to=kvbfp.CachePtrs(0x1100000, 0x1200000, 0x1300000, 0x100000 + 64)),
                dict(lens=0x7000000 + 8), dict(w_out=0x5000000), dict(w_out=0x5000000 + 3 * 2 * 512 * 4 - 4)):
        assert evict(**bad) == BAD, bad
    pages = (FAKE, 8, 3, FAKE, 2)
    for bad in (dict(paged=(None,) + pages[1:]), dict(paged=pages[:3] + (None, 2)), dict(paged=pages, keep=129), dict(paged=pages, max_len=513),
                dict(paged=pages, to=PTRS, dst=kvbfp.make_layout(128, 32, 4, 2, 21, 64)),
                dict(paged=pages, to=kvbfp.CachePtrs(0x100000, 0x1200000, 0x1300000, 0x1400000))):
        args = {**dict(src=POOL, dst=POOL, to=OTHER), **bad}
        assert evict(**args) == BAD, bad
    assert evict(src=POOL, dst=kvbfp.make_layout(128, 32, 4, 2, 9, 24), paged=pages) == UNS


def test_binding_checks_shapes():
    z = torch.zeros
    with pytest.raises(ValueError):
        kvbfp.make_score_rule(slopes=z(4, dtype=torch.float64))
    with pytest.raises(ValueError):
        kvbfp.make_score_rule(tree_mask=z(2, 4, dtype=torch.int32))
    with pytest.raises(ValueError):
        kvbfp.make_score_rule(first_dev=z(4, dtype=torch.int32))
    with pytest.raises(ValueError):
        kvbfp.make_score_rule(slopes=z(4))                   # host memory
    cache = kvbfp.Cache(LAYOUT, z(1), z(1), z(1), z(1))
    for shape in ((3, 8, 128), (2, 4, 8, 128), (3, 4, 8, 64)):
        with pytest.raises(ValueError):
            kvbfp.decode_attention_scored(cache, z(shape), 512, 0.1)
    with pytest.raises(ValueError):
        kvbfp.decode_attention_scored(cache, z(3, 4, 8, 128).transpose(1, 2), 512, 0.1)
    with pytest.raises(ValueError):
        kvbfp.decode_attention_scored(cache, z(3, 4, 8, 128), 512, 0.1, seq_len_dev=z(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        kvbfp.accumulate_weights(cache, z(3, 4, 8, 128), 512, 0.1, z(3, 4, 4))
    with pytest.raises(ValueError):
        kvbfp.evict(cache, cache, z(3, 2, 512), 512, 100, 4, 10, z(3, 2, 99, dtype=torch.int32), z(3, dtype=torch.int32))

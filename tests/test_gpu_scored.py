"""Attention with a rule on its scores (tree, cap, distance bias, window, documents, prefix) against a plain 64-bit form, over every
type, width, page size and the sizes at which a tile, a split or a mask begins or ends."""
import numpy as np
import pytest
import torch

import scored_ref as R
from paper_2403_20137_amd import kvbfp
from util import assert_attention_close, dev_i32

pytestmark = pytest.mark.gpu
D = 128
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def run_case(seed, B, H, G, n, S, bits, block, dtype, page=0, lens=None, perm=False, cap=0.0, slopes=False, window=0, first=None,
             prefix=None, tree=None, scale=None, with_lse=True, q_offset=0):
    rng = np.random.default_rng(seed)
    cache, table = R.make_cache(rng, B, H, S, bits, block, page, extra=5)
    sizes = list(lens) if lens is not None else [S] * B
    q = torch.from_numpy(rng.standard_normal((B, n, H * G, D)).astype(np.float32)).to(dtype).cuda()
    if q_offset:                                       # elements: the kernels may not count on wide loads
        q = torch.cat([torch.zeros(q_offset, dtype=dtype, device="cuda"), q.flatten()])[q_offset:].view(q.shape)
    pk = np.stack([rng.permutation(D) for _ in range(H)]) if perm else None
    pv = np.stack([rng.permutation(D) for _ in range(H)]) if perm else None
    rule = {"cap": cap, "window": window, "first": first, "prefix": prefix, "tree": tree,
            "slopes": 2.0 ** -rng.uniform(1, 8, H * G).astype(np.float32) if slopes else None}
    dev = kvbfp.make_score_rule(
        cap=cap, window=window, slopes=None if not slopes else torch.tensor(rule["slopes"], dtype=F32).cuda(),
        first_dev=None if first is None else dev_i32(np.array(first)), prefix_dev=None if prefix is None else dev_i32(np.array(prefix)),
        tree_mask=None if tree is None else torch.tensor(tree, dtype=torch.int64).cuda())
    if slopes:
        rule["slopes"] = R.f64(torch.tensor(rule["slopes"], dtype=F32))
    scale = 1 / 11.3 if scale is None else scale
    scale = float(np.float32(scale))
    cap64 = float(np.float32(cap))
    rule["cap"] = cap64
    rule["by_exp"] = dtype != F32
    lse = torch.full((B, n, H * G), 7.0, device="cuda") if with_lse else None
    lens_dev = None if lens is None else dev_i32(np.array(lens))
    args = dict(rule=dev, seq_len_dev=lens_dev, perm_k=dev_i32(pk), perm_v=dev_i32(pv), lse=lse, out=torch.full_like(q, float("nan")))
    if page:
        need = kvbfp.scored_workspace_bytes_paged(cache.layout, table.shape[1], B, H * G, n, S)
    else:
        need = kvbfp.scored_workspace_bytes(cache.layout, H * G, n, S)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    if page:
        out = kvbfp.decode_attention_scored_paged(cache, table, q, S, scale, workspace=ws, **args)
    else:
        out = kvbfp.decode_attention_scored(cache, q, S, scale, workspace=ws, **args)
    torch.cuda.synchronize()
    keys, values = R.decoded(cache, 0, table, S), R.decoded(cache, 1, table, S)
    want, want_lse, tol = R.attention(R.f64(q), keys, values, scale, sizes, pk, pv, rule)
    assert torch.isfinite(out).all()
    assert_attention_close(out.view(B, n * H * G, D), want.reshape(B, n * H * G, D), dtype, "scored %d" % seed)
    if with_lse:
        got = R.f64(lse)
        assert np.array_equal(np.isinf(got), np.isinf(want_lse)) and not np.isnan(got).any()
        some = ~np.isinf(want_lse)
        assert (np.abs(got[some] - want_lse[some]) <= tol[some]).all(), np.max(np.abs(got[some] - want_lse[some]) / tol[some])
    return dict(cache=cache, table=table, q=q, out=out, lse=lse, rule=dev, lens=lens_dev, scale=scale, sizes=sizes, keys=keys, values=values, ref=rule, pk=pk, pv=pv)


def tree(seed, n, batch=None):
    rng = np.random.default_rng(seed)
    return R.random_tree(rng, n) if batch is None else [R.random_tree(rng, n) for _ in range(batch)]


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("bits,block", [(4, 16), (4, 32), (4, 64), (4, 128), (8, 16), (8, 32), (8, 128)])
def test_formats(dtype, bits, block):
    run_case(1, 2, 2, 3, 5, 300, bits, block, dtype, lens=[300, 211], perm=True, cap=20.0, slopes=True, tree=tree(1, 5, 2))


@pytest.mark.parametrize("S", [1, 2, 15, 16, 17, 31, 32, 33, 127, 128, 129, 255, 257, 700])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_lengths(S, dtype):
    run_case(S, 1, 1, 4, 1, S, 4, 32, dtype, cap=5.0)
    run_case(S + 1, 3, 2, 2, 7, S, 4, 32, dtype, lens=[S, S // 2, 0], tree=tree(S, 7, 3), window=S // 3)


@pytest.mark.parametrize("G,n", [(1, 1), (15, 1), (16, 1), (17, 1), (1, 32), (3, 11), (4, 16), (5, 13), (4, 17), (2, 64), (8, 33), (40, 1), (7, 64)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_rows_of_a_head(G, n, dtype):
    run_case(G * 100 + n, 1, 2, G, n, 197, 4, 32, dtype, lens=[190], tree=tree(n, n), cap=30.0)
    run_case(G * 100 + n + 1, 1, 1, G, n, 140, 8, 32, dtype, prefix=[100], slopes=True)


@pytest.mark.parametrize("page", [16, 32, 128, 512])
@pytest.mark.parametrize("n", [1, 9, 40])
def test_pages(page, n):
    run_case(page + n, 3, 2, 4, n, 333, 4, 32, BF16, page=page, lens=[333, 16, 47], perm=True, tree=tree(n, n))
    run_case(page + n, 2, 1, 2, n, 90, 8, 16, F16, page=page, lens=[90, 65], window=33, slopes=True)


@pytest.mark.parametrize("window", [1, 2, 16, 31, 129, 300, 2 ** 31 - 1])
@pytest.mark.parametrize("n", [1, 6])
def test_windows(window, n):
    run_case(window % 1000, 2, 2, 2, n, 500, 4, 32, BF16, lens=[500, 123], window=window)
    run_case(window % 1000, 2, 1, 2, n, 500, 4, 32, F32, lens=[500, 123], window=window, prefix=[40, 2], tree=tree(3, n))


def test_documents_and_prefixes():
    first = [[0, 0, 100, 390, 395], [60, 60, 60, 299, 2 ** 31 - 1], [-5, 0, 1, 2, 3]]
    for dtype in (F32, BF16):
        run_case(5, 3, 2, 2, 5, 400, 4, 32, dtype, lens=[400, 300, 7], first=first)
        run_case(6, 3, 2, 2, 5, 400, 4, 32, dtype, lens=[400, 300, 7], first=first, prefix=[130, -3, 2 ** 31 - 1], window=50, slopes=True)


def test_long_prefix_and_far_documents_skip_what_nobody_sees():
    # the tiles between the prefix and the document hold exponent 255 everywhere: they are not read, or count for nothing
    case = run_case(9, 1, 1, 4, 3, 3000, 4, 32, BF16, first=[[2500, 2500, 2600]], prefix=[70])
    cache = case["cache"]
    cache.k_exp[:, :, 70:2500] = 255
    cache.v_exp[:, :, 70:2500] = 255
    cache.k_mant[:, :, 70:2500] = 0x7F
    cache.v_mant[:, :, 70:2500] = 0x7F
    again = kvbfp.decode_attention_scored(cache, case["q"], 3000, case["scale"], case["rule"])
    assert torch.equal(again, case["out"])


def test_masked_rows_at_the_end_of_the_range_do_not_count():
    # unseen nodes (the last tokens) with the largest exponents and codes: no infinity times 0
    n, masks = 6, [1, 3, 1 | 4, 1 | 8, 0, 1 << 5]
    for bits, block in ((4, 32), (8, 32), (4, 16), (8, 16)):
        for dtype in (F32, BF16):
            case = run_case(11, 1, 1, 2, n, 60, bits, block, dtype, tree=masks, first=[[10, 10, 10, 10, 10, 60]])
            cache = case["cache"]
            for t in (0, 9, 58):                           # behind the documents' begin; node 4, which nobody sees
                for e, m in ((cache.k_exp, cache.k_mant), (cache.v_exp, cache.v_mant)):
                    e[:, :, t] = 255
                    m[:, :, t] = 0x7F
            again = kvbfp.decode_attention_scored(cache, case["q"], 60, case["scale"], case["rule"])
            assert torch.equal(again, case["out"]), (bits, block, dtype)
            assert again[0, 4].any()                        # tokens from 10 on
            assert not again[0, 5].any()                    # its document begins behind the last token


def test_rows_that_see_nothing():
    n = 4
    case = run_case(12, 2, 2, 3, n, 4, 4, 32, BF16, lens=[4, 2], tree=[0, 0, 1 << 3, 1 << 2 | 1 << 3])
    assert torch.isinf(case["lse"][0, :2]).all() and not case["out"][0, :2].any()
    for dtype in (F32, F16, BF16):
        case = run_case(13, 2, 1, 2, 1, 64, 4, 32, dtype, lens=[0, 0])
        assert torch.isinf(case["lse"]).all() and not case["out"].any()


def test_caps():
    for cap in (1e-3, 0.5, 5.0, 50.0, 1e4, 1e20):
        for dtype in (F32, BF16):
            run_case(14, 1, 1, 4, 1, 200, 4, 32, dtype, cap=cap)
    run_case(15, 1, 1, 4, 1, 200, 8, 32, F32, cap=3.0, scale=4.0)          # every score far beyond the cap
    run_case(16, 1, 1, 4, 2, 200, 8, 32, F32, scale=0.0)


def test_all_bits_of_a_mask():
    n = 64
    masks = tree(4, n)
    assert min(masks) < 0                                   # bit 63 is in use
    run_case(17, 1, 1, 2, n, 1000, 4, 32, BF16, tree=masks, slopes=True)
    run_case(18, 1, 1, 1, n, 30, 4, 32, F32, tree=[-1] * n, lens=[30])     # fewer tokens than nodes, everyone sees everyone


def test_alignment_of_queries_and_exponents():
    case = run_case(19, 1, 2, 4, 2, 300, 4, 16, BF16, q_offset=1)
    run_case(19, 1, 2, 4, 2, 300, 4, 16, F32, q_offset=3)
    cache = case["cache"]
    moved = []
    for e in (cache.k_exp, cache.v_exp):
        raw = torch.zeros(e.numel() + 1, dtype=torch.uint8, device="cuda")
        raw[1:] = e.flatten()
        moved.append(raw[1:].view(e.shape))
    odd = kvbfp.Cache(cache.layout, cache.k_mant, moved[0], cache.v_mant, moved[1])
    assert torch.equal(kvbfp.decode_attention_scored(odd, case["q"], 300, case["scale"], case["rule"]), case["out"])


def test_without_a_rule_it_is_the_causal_call():
    for dtype in (F32, F16, BF16):
        case = run_case(20, 2, 2, 4, 5, 400, 4, 32, dtype, lens=[400, 3])
        plain = kvbfp.decode_attention_scored(case["cache"], case["q"], 400, case["scale"], None, seq_len_dev=case["lens"])
        assert torch.equal(plain, case["out"])
        other = kvbfp.decode_attention_multi(case["cache"], case["q"], 400, case["scale"], seq_len_dev=case["lens"])
        step = {F32: 2e-5, F16: 2.0 ** -10, BF16: 2.0 ** -7}[dtype]          # either side may be off by half a step of its type
        assert ((plain.float() - other.float()).norm(dim=-1) <= step * other.float().norm(dim=-1) + 1e-6).all()


def test_pages_and_regions_give_the_same_bits():
    case = run_case(21, 2, 2, 4, 9, 500, 4, 32, BF16, page=64, lens=[500, 77], tree=tree(5, 9, 2), cap=10.0)
    pool, table = case["cache"], case["table"]
    flat = kvbfp.alloc_cache(kvbfp.make_layout(D, 32, 4, 2, 2, table.shape[1] * 64))
    for src, dst in zip(pool.planes(), flat.planes()):
        dst.copy_(src[table.long()].transpose(1, 2).flatten(2, 3))
    got = kvbfp.decode_attention_scored(flat, case["q"], 500, case["scale"], case["rule"], seq_len_dev=case["lens"])
    assert torch.equal(got, case["out"])


def test_same_bits_every_time_and_on_another_stream():
    case = run_case(22, 4, 2, 4, 16, 900, 4, 32, BF16, lens=[900, 800, 1, 450], tree=tree(6, 16))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    outs = []
    with torch.cuda.stream(side):
        for _ in range(3):
            outs.append(kvbfp.decode_attention_scored(case["cache"], case["q"], 900, case["scale"], case["rule"], seq_len_dev=case["lens"]))
    by_handle = kvbfp.decode_attention_scored(case["cache"], case["q"], 900, case["scale"], case["rule"], seq_len_dev=case["lens"],
                                              stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    for o in outs + [by_handle]:
        assert torch.equal(o, case["out"])


def test_graph_replays_follow_the_inputs():
    case = run_case(23, 2, 2, 4, 8, 600, 4, 32, BF16, lens=[600, 590], tree=tree(7, 8, 2), cap=20.0)
    q, lens, rule, cache = case["q"], case["lens"], case["rule"], case["cache"]
    out, lse = torch.empty_like(q), torch.empty_like(case["lse"])
    ws = torch.empty(kvbfp.scored_workspace_bytes(cache.layout, q.shape[2], q.shape[1], 600), dtype=torch.uint8, device="cuda")
    weights = torch.zeros(2, 2, 600, device="cuda")
    call = lambda: (kvbfp.decode_attention_scored(cache, q, 600, case["scale"], rule, seq_len_dev=lens, out=out, lse=lse, workspace=ws),  # noqa: E731
                    kvbfp.accumulate_weights(cache, q, 600, case["scale"], lse, None, weights, rule=rule, seq_len_dev=lens))
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for k in range(4):
        lens.copy_(torch.tensor([600 - 37 * k, 590 - 100 * k], dtype=torch.int32))
        q.mul_(1.0 + 0.25 * k)
        rule.tensors[3].copy_(torch.tensor(tree(50 + k, 8, 2), dtype=torch.int64))
        weights.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone(), weights.clone()
        weights.zero_()
        call()
        torch.cuda.synchronize()
        for g, w in zip(got, (out, lse, weights)):
            assert torch.equal(g, w)


@pytest.mark.parametrize("seed", range(24))
def test_random_calls(seed):
    rng = np.random.default_rng(1000 + seed)
    B, H, G, n = int(rng.integers(1, 5)), int(rng.choice([1, 2, 5])), int(rng.choice([1, 2, 3, 4, 8, 9])), int(rng.choice([1, 1, 2, 5, 16, 31]))
    S = int(np.exp(rng.uniform(0, np.log(1500))))
    S = min(S, max(1, 60000 // (B * H * G * n)) + 40)
    pick = lambda p: rng.random() < p  # noqa: E731
    run_case(seed, B, H, G, n, S, int(rng.choice([4, 8])), int(rng.choice([16, 32, 64, 128])), [F32, F16, BF16][seed % 3],
             page=int(rng.choice([0, 0, 16, 64])), lens=[S] + [int(rng.integers(0, S + 1)) for _ in range(B - 1)] if pick(0.7) else None,
             perm=pick(0.5), cap=float(rng.choice([0.0, 2.0, 30.0])), slopes=pick(0.4), window=int(rng.integers(1, S + 1)) if pick(0.4) else 0,
             first=[[int(rng.integers(0, S)) for _ in range(n)] for _ in range(B)] if pick(0.3) else None,
             prefix=[int(rng.integers(0, S)) for _ in range(B)] if pick(0.3) else None,
             tree=(tree(seed, n, B) if pick(0.5) else tree(seed, n)) if pick(0.6) else None, with_lse=pick(0.7))


def test_offsets_beyond_32_bits():
    # the planes of one sequence pass 4 GiB: 8 heads of 2^23 + 300 tokens, 64 bytes a row; only its last tokens are seen
    S = (1 << 23) + 300
    cache = kvbfp.alloc_cache(kvbfp.make_layout(D, 128, 4, 9, 1, S), fill=0)
    rng = np.random.default_rng(3)
    rows = lambda: torch.from_numpy(rng.standard_normal((1, 200, 9, D)).astype(np.float32)).cuda()  # noqa: E731
    k, v = rows(), rows()
    kvbfp.quantize_append(cache, k, v, pos0=S - 200)
    small = kvbfp.alloc_cache(kvbfp.make_layout(D, 128, 4, 9, 1, 200))
    kvbfp.quantize_append(small, k, v)
    q = torch.from_numpy(rng.standard_normal((1, 3, 18, D)).astype(np.float32)).cuda()
    for window in (150,):
        rule = kvbfp.make_score_rule(window=window)
        lse, lse_small = torch.empty(1, 3, 18, device="cuda"), torch.empty(1, 3, 18, device="cuda")
        got = kvbfp.decode_attention_scored(cache, q, S, 0.1, rule, lse=lse)
        want = kvbfp.decode_attention_scored(small, q, 200, 0.1, rule, lse=lse_small)
        assert torch.allclose(lse, lse_small, rtol=1e-5, atol=1e-5)
        assert ((got - want).norm(dim=-1) <= 2e-5 * want.norm(dim=-1)).all()
        w, w_small = torch.zeros(1, 9, S, device="cuda"), torch.zeros(1, 9, 200, device="cuda")
        kvbfp.accumulate_weights(cache, q, S, 0.1, lse, None, w, rule=rule)
        kvbfp.accumulate_weights(small, q, 200, 0.1, lse_small, None, w_small, rule=rule)
        assert torch.allclose(w[..., -200:], w_small, rtol=1e-4, atol=1e-6) and not w[..., :-200].any()

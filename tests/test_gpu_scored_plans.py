"""Attention with a rule on its scores and the collected weights where the way of the work changes: rows of a workgroup, splits, more sequences
than lanes, few and many tokens for the rows; blocks at the end of the exponents' range."""
import numpy as np
import pytest
import torch

import scored_ref as R
from paper_2403_20137_amd import kvbfp
from test_gpu_evict import collect
from test_gpu_scored import BF16, F16, F32, run_case, tree
from util import dev_i32

pytestmark = pytest.mark.gpu
D = 128


def short(seed, batch, most, length):
    """Lengths up to `most`, one empty and one of `length` tokens among them."""
    lens = np.random.default_rng(seed).integers(0, most + 1, batch)
    lens[batch // 2], lens[-1] = 0, length
    return lens.tolist()


# cache length, batch and rows decide: 128, 64 or 32 rows a workgroup, partial results or none, places shared out or not
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("B,H,G,n,S", [
    (16, 2, 5, 60, 5600),        # 300 rows in tiles of 128 (bf16) or 64, shared out
    (66, 2, 3, 50, 2000),        # the same, more sequences than lanes, one split
    (16, 2, 4, 12, 2100),        # 48 rows, tiles of 64, shared out
    (70, 4, 11, 4, 300),         # 44 rows, one split
    (3, 1, 3, 64, 200),          # 192 rows in tiles of 32
    (2, 2, 16, 2, 4000),         # 32 rows of two long sequences
    (70, 4, 1, 9, 900),          # 9 rows, one split
    (70, 4, 4, 2, 300),          # 8 rows
    (5, 80, 2, 3, 700),          # two splits only because lengths differ
])
def test_ways_of_the_work(B, H, G, n, S, dtype):
    case = run_case(B + n, B, H, G, n, S, 4, 32, dtype, lens=short(S, B, 40, min(S, 333)), tree=tree(n, n), cap=30.0)
    collect(case, True, 0.9, S)
    case = run_case(B + n + 1, B, H, G, n, S, 8, 64, dtype, lens=short(n, B, 70, min(S, 170)), perm=True, window=60)
    collect(case, False, 1.0, S)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("bits,block,page", [(4, 16, 0), (4, 128, 16), (8, 16, 32), (8, 32, 0)])
def test_weights_of_few_rows_and_many_tokens(bits, block, page, dtype):
    # 300 tiles of 256 tokens at least: lengths that end in every part of a tile
    lens = [1, 15, 63, 64, 65, 128, 255, 256, 257, 300, 511, 513, 700, 767, 769, 800, 0, 801, 900, 1000]
    for k, (G, n) in enumerate(((4, 1), (16, 1), (3, 5))):
        extra = (dict(cap=20.0), dict(slopes=True, window=200), dict(tree=tree(k, n), prefix=[90] * 20))[k]
        case = run_case(60 + k, 20, 4, G, n, 1000, bits, block, dtype, page=page, lens=lens, perm=True, **extra)
        collect(case, k > 0, 0.9, 1000, in_place=k == 2)


def test_all_empty_and_one_token():
    for B in (2, 64, 65):
        for n in (1, 20):
            run_case(B, B, 2, 2, n, 700, 4, 32, BF16, lens=[0] * B)
            run_case(B, B, 2, 2, n, 700, 4, 32, BF16, lens=[0] * (B - 1) + [1])


def test_bits_behind_the_last_node_mean_nothing():
    n = 5
    plain = tree(9, n)
    case = run_case(31, 1, 1, 2, n, 90, 4, 32, BF16, tree=plain, slopes=True)
    more = kvbfp.make_score_rule(slopes=case["rule"].tensors[0], tree_mask=torch.tensor([m - (1 << 63) + (1 << 40) + (1 << n) for m in plain],
                                                                                        dtype=torch.int64).cuda())
    lse = torch.empty_like(case["lse"])
    got = kvbfp.decode_attention_scored(case["cache"], case["q"], 90, case["scale"], more, lse=lse)
    assert torch.equal(got, case["out"]) and torch.equal(lse, case["lse"])


@pytest.mark.parametrize("n", [1, 2, 6, 24])
@pytest.mark.parametrize("bits,block,most", [(4, 32, 254), (4, 16, 254), (8, 32, 251)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_large_exponents(n, bits, block, most, dtype):
    # values of 2^74 to the end of the range in some tokens, keys at the end of theirs with a scale to match
    rng = np.random.default_rng(n + bits)
    S, H, G = 400, 2, 4
    for high_keys in (False, True):
        cache, _ = R.make_cache(rng, 1, H, S, bits, block)
        spots = torch.from_numpy(rng.choice(S, 40, replace=False)).cuda()
        for t in spots[:20].tolist():
            cache.v_exp[:, :, t] = int(rng.integers(201, most + 1))
        cache.v_exp[:, :, spots[0]] = most
        scale = 0.09
        if high_keys:
            cache.k_exp[:] = torch.from_numpy(rng.integers(most - 4, most + 1, tuple(cache.k_exp.shape)).astype(np.uint8)).cuda()
            scale = 2.0 ** (127 - most) / 20
        q = torch.from_numpy(rng.standard_normal((1, n, H * G, D)).astype(np.float32)).to(dtype).cuda()
        lse = torch.empty(1, n, H * G, device="cuda")
        got = R.f64(kvbfp.decode_attention_scored(cache, q, S, scale, lse=lse))
        keys, values = R.decoded(cache, 0), R.decoded(cache, 1)
        want, want_lse, tol = R.attention(R.f64(q), keys, values, float(np.float32(scale)), [S], rule={"by_exp": dtype != F32})
        size, _, _ = R.attention(R.f64(q), keys, np.abs(values), float(np.float32(scale)), [S], rule={})
        assert (np.abs(R.f64(lse) - want_lse) <= tol).all()
        # weights are off by the scores' error either way (twice what lse's bound has) and by their 16 bits, the sums by S + 8 roundings,
        # the result by half a step
        off = size * (2 * tol[..., None] + 2.0 ** -16 * (dtype != F32) + (S + 8) * R.U) + np.abs(want) * torch.finfo(dtype).eps / 2
        assert np.isfinite(got).all() and (np.abs(got - want) <= off).all(), np.max(np.abs(got - want) / off)


def test_two_streams_with_a_workspace_each():
    cases = [run_case(40 + k, 3, 2, 4, 10, 1500, 4, 32, BF16, lens=[1500, 700, 90], tree=tree(k, 10)) for k in range(2)]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(6):
        for k, (case, stream) in enumerate(zip(cases, streams)):
            with torch.cuda.stream(stream):
                outs[k].append(kvbfp.decode_attention_scored(case["cache"], case["q"], 1500, case["scale"], case["rule"], seq_len_dev=case["lens"]))
    torch.cuda.synchronize()
    for case, got in zip(cases, outs):
        assert all(torch.equal(o, case["out"]) for o in got)


def test_odd_addresses_of_the_output():
    for n, S in ((1, 90), (1, 1500), (20, 100), (20, 1500)):
        case = run_case(50 + n, 2, 2, 4, n, S, 4, 32, BF16, perm=True, lens=[S, S // 3])
        args = dict(rule=case["rule"], seq_len_dev=case["lens"], perm_k=dev_i32(case["pk"]), perm_v=dev_i32(case["pv"]))
        raw = torch.full((case["q"].numel() + 9,), -3.0, dtype=BF16, device="cuda")
        odd = raw[1:1 + case["q"].numel()].view(case["q"].shape)
        kvbfp.decode_attention_scored(case["cache"], case["q"], S, case["scale"], out=odd, **args)
        assert torch.equal(odd, case["out"]) and raw[0] == -3 and (raw[1 + odd.numel():] == -3).all()


def test_captured_weights_and_eviction_follow_the_inputs():
    rng = np.random.default_rng(70)
    B, H, S, keep = 16, 4, 1000, 300
    cache, _ = R.make_cache(rng, B, H, S, 4, 32)
    dst = kvbfp.alloc_cache(kvbfp.make_layout(D, 32, 4, H, B, keep), fill=0)
    q = torch.from_numpy(rng.standard_normal((B, 1, H * 4, D)).astype(np.float32)).to(BF16).cuda()
    lens, new_len = dev_i32(np.full(B, S)), torch.zeros(B, dtype=torch.int32, device="cuda")
    lse, weights = torch.empty(B, 1, H * 4, device="cuda"), torch.zeros(B, H, S, device="cuda")
    kept, left = torch.zeros(B, H, keep, dtype=torch.int32, device="cuda"), torch.zeros(B, H, keep, device="cuda")
    ws = torch.empty(kvbfp.scored_workspace_bytes(cache.layout, H * 4, 1, S), dtype=torch.uint8, device="cuda")

    def step():
        kvbfp.decode_attention_scored(cache, q, S, 0.09, seq_len_dev=lens, lse=lse, workspace=ws)
        kvbfp.accumulate_weights(cache, q, S, 0.09, lse, None, weights, seq_len_dev=lens)
        kvbfp.evict(cache, dst, weights, S, keep, 4, 32, kept, new_len, weights_out=left, seq_len_dev=lens)

    outputs = [weights, kept, left, new_len, *dst.planes()]
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        lens.copy_(torch.from_numpy(rng.integers(0, S + 1, B).astype(np.int32)))
        q.mul_(1.0 + 0.25 * k)
        got = []
        for run in (graph.replay, step):
            for o in outputs:
                o.zero_()
            run()
            torch.cuda.synchronize()
            got.append([o.clone() for o in outputs])
        assert all(torch.equal(a, b) for a, b in zip(*got)), k
        assert torch.equal(new_len, lens.clamp(max=keep))

"""Capped scores as exact as fp32 holds them, with every type of input: each query token sees itself alone, so lse is its score and its weight
is 1, and queries of one channel leave nothing to the products but exact numbers."""
import math

import numpy as np
import pytest
import torch

import scored_ref as R
from paper_2403_20137_amd import kvbfp

pytestmark = pytest.mark.gpu
D = 128
U = R.U


@pytest.mark.parametrize("cap", [0.75, 5.0, 30.0, 50.0, 64.0, 65.0, 66.5, 67.0, 1000.0])
@pytest.mark.parametrize("dtype,G", [(torch.float32, 2), (torch.float16, 2), (torch.bfloat16, 2), (torch.bfloat16, 1), (torch.bfloat16, 3)])
@pytest.mark.parametrize("n", [1, 7, 64])                   # 16 rows at most, up to 64, more
def test_capped_scores_keep_the_bits_of_fp32(n, dtype, G, cap):
    rng = np.random.default_rng(n + G)
    B, H, S = 3, 2, 90
    cache, _ = R.make_cache(rng, B, H, S, 8, 32)
    keys = R.decoded(cache, 0)
    # one channel a row; scores from a thousandth of the cap to three times it, either sign
    q = torch.zeros(B, n, H * G, D)
    at = torch.from_numpy(rng.integers(0, D, (B, n, H * G, 1)))
    aim = cap * 3.0 * 10.0 ** rng.uniform(-3.5, 0, (B, n, H * G)) * rng.choice([-1, 1], (B, n, H * G))
    own = np.empty_like(aim)
    for b, i, h in np.ndindex(*aim.shape):
        own[b, i, h] = keys[b, h // G, S - n + i, int(at[b, i, h])]
    scale = 0.25
    q.scatter_(-1, at, torch.from_numpy(np.where(own != 0, aim / np.where(own != 0, own, 1) / scale, 0.0)).float().unsqueeze(-1))
    q = q.to(dtype).cuda()
    rule = kvbfp.make_score_rule(cap=cap, window=1)
    lse = torch.empty(B, n, H * G, device="cuda")
    out = kvbfp.decode_attention_scored(cache, q, S, scale, rule, lse=lse)
    weights = kvbfp.accumulate_weights(cache, q, S, scale, lse, rule=rule)
    cap = float(np.float32(cap))
    with np.errstate(invalid="ignore"):
        y = cap * np.tanh(R.f64(q).max(-1) * own * scale / cap) + cap * np.tanh(R.f64(q).min(-1) * own * scale / cap)
    # roundings: log2(e) times the scale and times the cap, its inverse, the product with the scale, 6 of the cap's form, ln 2 and the
    # product with it: 12 of half a step, and one of the result's own
    # (a query of fp16 that would have to pass 65504 for its score is none that the calls take: its kv-head is left out)
    there = np.isfinite(R.f64(q)).all(-1).all(1).reshape(B, H, G).all(-1)
    assert there.any()
    rows = np.broadcast_to(there.repeat(G, 1)[:, None], y.shape)
    y = np.where(rows, y, 0.0)
    off = np.where(rows, np.abs(R.f64(lse) - y), 0.0)
    assert (off <= 13 * U * np.abs(y) + 1e-37).all(), np.max(off / (U * np.abs(y) + 1e-37))
    values = R.decoded(cache, 1)
    want = np.stack([values[:, h // G, S - n:] for h in range(H * G)], 2)
    step = 2.0 ** -16 + {torch.float32: U, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}[dtype]
    off = np.where(rows[..., None], np.abs(R.f64(out) - want), 0.0)
    assert (off <= step * np.abs(want) + 2.0 ** -25).all()                  # (fp16 has steps of 2^-24 at its lower end)
    # a weight is e to the difference of the score and lse, each with log2(e) and its roundings: relative to their size and to 1
    got = np.where(there[..., None], R.f64(weights), np.where(np.arange(S) >= S - n, G, 0))
    most = np.abs(y).reshape(B, n, H, G).max(-1).transpose(0, 2, 1)
    assert (np.abs(got[:, :, S - n:] - G) <= G * (13 + 4) * U * (1 + most)).all() and not got[:, :, :S - n].any()


def test_log_sums_and_weights_of_capped_scores_agree():
    # 16-bit inputs, ordinary scores: lse of fp32 products of 128 channels, so that a row's weights add up to 1 as fp32 does them
    rng = np.random.default_rng(5)
    B, H, G, S = 2, 2, 4, 700
    cache, _ = R.make_cache(rng, B, H, S, 4, 32)
    q = torch.from_numpy(rng.standard_normal((B, 1, H * G, D)).astype(np.float32)).to(torch.bfloat16).cuda()
    rule = kvbfp.make_score_rule(cap=50.0)
    lse = torch.empty(B, 1, H * G, device="cuda")
    kvbfp.decode_attention_scored(cache, q, S, 1 / math.sqrt(D), rule, lse=lse)
    got = R.f64(kvbfp.accumulate_weights(cache, q, S, 1 / math.sqrt(D), lse, rule=rule)).sum(-1)
    # both calls form the same sums of products (their orders differ by the splits alone, not within a score): what is left is the cap's
    # roundings either way, lse's, and S roundings of the sums
    tol = (2 * 6 * U * 30 + 8 * U * (np.abs(R.f64(lse)).max() + 1) + 2 * S * U) * G
    assert (np.abs(got - G) <= tol).all(), (np.abs(got - G).max(), tol)


def test_negative_scales():
    from test_gpu_scored import BF16, F32, run_case, tree
    from test_gpu_evict import collect
    for dtype in (F32, BF16):
        for n in (1, 30):
            case = run_case(61, 2, 2, 4, n, 300, 4, 32, dtype, lens=[300, 77], scale=-0.07, tree=tree(1, n), cap=25.0)
            collect(case, True, 0.9, 300)
            case = run_case(62, 2, 2, 4, n, 300, 4, 32, dtype, lens=[300, 77], scale=-0.07, slopes=True, window=100)
            collect(case, False, 1.0, 300)

"""Attention with a rule on its scores over values at the end of the exponents' range: the sums of many of them pass fp32's range long before the
result does."""
import numpy as np
import pytest
import torch

import scored_ref as R
from paper_2403_20137_amd import kvbfp
from test_gpu_scored import BF16, F32

pytestmark = pytest.mark.gpu
D = 128


@pytest.mark.parametrize("B,S", [(1, 70), (1, 400), (2, 9000), (60, 130)])      # one part, a few, many; one split for many sequences
@pytest.mark.parametrize("n", [1, 3, 12, 40])
@pytest.mark.parametrize("bits,block,most", [(4, 32, 254), (4, 16, 254), (8, 64, 251), (8, 16, 251)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_every_value_at_the_end_of_the_range(dtype, bits, block, most, n, B, S):
    rng = np.random.default_rng(S + n + bits)
    H, G = 1, 4
    cache, _ = R.make_cache(rng, B, H, S, bits, block)
    top = (1 << (bits - 1)) - 1
    cache.v_mant.fill_(top if bits == 8 else top * 17)
    cache.v_exp.fill_(most)
    # other signs in some channels, no value in others; small ones among the large in the second half of the tokens
    cache.v_mant[..., 3] |= 0x88 if bits == 4 else 0x80
    cache.v_mant[..., 7] = 0
    cache.v_exp[:, :, S // 2:: 3] = 100
    for flat in (True, False):                              # all scores alike; ordinary ones
        q = torch.from_numpy(rng.standard_normal((B, n, H * G, D)).astype(np.float32) * (not flat)).to(dtype).cuda()
        lse = torch.empty(B, n, H * G, device="cuda")
        got = R.f64(kvbfp.decode_attention_scored(cache, q, S, 0.09, lse=lse))
        assert np.isfinite(got).all()
        check = [0, B - 1] if B > 1 else [0]
        keys, values = (R.decoded(cache, k)[check] for k in (0, 1))
        args = (float(np.float32(0.09)), [S] * len(check))
        want, want_lse, tol = R.attention(R.f64(q)[check], keys, values, *args)
        size, _, _ = R.attention(R.f64(q)[check], keys, np.abs(values), *args)
        assert (np.abs(R.f64(lse)[check] - want_lse) <= tol).all()
        # as for single large values: the scores' error either way, 16 bits of the weights, S + 8 roundings of the sums, half a step
        off = size * (2 * tol[..., None] + 2.0 ** -16 * (dtype != F32) + (S + 8) * R.U) + np.abs(want) * torch.finfo(dtype).eps / 2
        assert (np.abs(got[check] - want) <= off).all(), np.max(np.abs(got[check] - want) / np.maximum(off, 1e-300))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_large_values_in_one_part_only(dtype):
    # the last tokens of a long sequence: other parts are joined with theirs, and light ones among them keep their bits
    rng = np.random.default_rng(9)
    S, H, G = 5000, 2, 4
    cache, _ = R.make_cache(rng, 1, H, S, 4, 32)
    cache.v_exp[:, :, S - 200:] = 254
    for n in (1, 20):
        q = torch.from_numpy(rng.standard_normal((1, n, H * G, D)).astype(np.float32)).to(dtype).cuda()
        rule = kvbfp.make_score_rule(slopes=torch.full((H * G,), 0.01, device="cuda"))
        got = R.f64(kvbfp.decode_attention_scored(cache, q, S, 0.09, rule))
        keys, values = R.decoded(cache, 0), R.decoded(cache, 1)
        extra = {"slopes": np.full(H * G, float(np.float32(0.01)))}
        want, _, tol = R.attention(R.f64(q), keys, values, float(np.float32(0.09)), [S], rule=extra)
        size, _, _ = R.attention(R.f64(q), keys, np.abs(values), float(np.float32(0.09)), [S], rule=extra)
        off = size * (2 * tol[..., None] + 2.0 ** -16 * (dtype != F32) + (S + 8) * R.U) + np.abs(want) * torch.finfo(dtype).eps / 2
        assert np.isfinite(got).all() and (np.abs(got - want) <= off).all()

"""What the calls with a rule on the scores count on the device, built with plain g++ and checked on the CPU; and the longest sequences through the
calls themselves."""
import shutil

import numpy as np
import pytest
import torch

import scored_ref as R
from paper_2403_20137_amd import kvbfp
from test_host_native_checks import _build_and_run
from util import dev_i32

D = 128


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_what_is_read_stays_in_32_bits(tmp_path):
    out = _build_and_run(tmp_path, "tokens_read_check", ["tests/cpp/tokens_read_check.cpp"],
                         ["-O1", "-fsanitize=undefined", "-fno-sanitize-recover=undefined"], timeout=60)
    assert "tokens_read ok" in out


@pytest.mark.gpu
def test_the_longest_window_beside_the_longest_prefix():
    # sequences of up to 2^30 tokens over two pages of 16384, used again and again: a window and a prefix of 2^30 add up to more than 32 bits,
    # and the splits are shared out by what a sequence reads
    page, S = 16384, 1 << 30
    rng = np.random.default_rng(30)
    pool = kvbfp.alloc_cache(kvbfp.make_layout(D, 128, 4, 1, 2, page))
    rows = lambda: torch.from_numpy(rng.standard_normal((2, page, 1, D)).astype(np.float32)).cuda()  # noqa: E731
    kvbfp.quantize_append(pool, rows(), rows())
    table = (torch.arange(S // page, dtype=torch.int32, device="cuda") & 1).expand(3, -1).contiguous()
    sizes = [S, S - 5, 1000]
    lens = dev_i32(np.array(sizes))
    rule = kvbfp.make_score_rule(window=S, prefix_dev=dev_i32(np.array([S, 0, 0])))
    q = torch.from_numpy(rng.standard_normal((3, 1, 2, D)).astype(np.float32)).to(torch.bfloat16).cuda()
    lse = torch.empty(3, 1, 2, device="cuda")
    out = R.f64(kvbfp.decode_attention_scored_paged(pool, table, q, S, 0.05, rule, seq_len_dev=lens, lse=lse))
    keys, values = (R.decoded(pool, k).reshape(2 * page, D) for k in (0, 1))
    y = R.f64(q)[:, 0] @ keys.T * float(np.float32(0.05))
    for b, size in enumerate(sizes):
        times = np.full(2 * page, size // (2 * page), np.float64)                # how often each row is there
        times[: size % (2 * page)] += 1
        p = times * np.exp(y[b])
        want, total = p @ values / p.sum(-1, keepdims=True), p.sum(-1)
        # a lane adds four numbers a tile of 128 tokens, and has no more than a two hundredth of the tiles: half a step each, in the sum of
        # the weights and in those of the values
        off = R.U * (4 * (size / 128 / 200 + 1) + 1000)
        assert (np.abs(R.f64(lse)[b, 0] - np.log(total)) <= off + 8 * R.U * 30).all()
        mean = p @ np.abs(values) / total[:, None]
        assert (np.abs(out[b, 0] - want) <= mean * (2 * off + 2.0 ** -16) + 2.0 ** -8 * np.abs(want)).all()
    weights = kvbfp.accumulate_weights_paged(pool, table, q, S, 0.05, lse, rule=rule, seq_len_dev=lens)
    for b, size in enumerate(sizes):                          # (136 roundings of a score's products, 6 in all, and some of lse: below 1e-4)
        each = np.exp(y[b] - R.f64(lse)[b, 0][:, None]).sum(0)
        whole = weights[b, 0, : size // (2 * page) * 2 * page].view(-1, 2 * page)
        rest = R.f64(weights[b, 0, whole.numel(): size])
        for got in (R.f64(whole[:1]), R.f64(whole[-1:])) if len(whole) else ():
            assert (np.abs(got - each) <= 1e-4 * each).all()
        # (tiles that every row sees are multiplied and added at once, the others round between: each is within 1e-4 all the same)
        assert ((whole - whole[:1]).abs() <= 2e-4 * whole[:1]).all() and (np.abs(rest - each[: rest.size]) <= 1e-4 * each[: rest.size]).all()
        assert not weights[b, 0, size:].any()

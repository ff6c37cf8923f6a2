"""Buffers that a call of the binding makes itself belong to the stream that its kernels run on: filled there, and given back to nothing that comes before
them."""
import contextlib

import numpy as np
import pytest
import torch

import scored_ref as R
from paper_2403_20137_amd import kvbfp
from test_gpu_scored import BF16, run_case, tree

D = 128


class _Quiet:
    """Stands for the library: every size is 4096, every call succeeds."""
    def __getattr__(self, name):
        return lambda *args: 4096 if name.endswith(("_bytes", "_bytes_paged")) else kvbfp.OK


def calls(cache, pool, table, stream):
    rows, tokens = torch.zeros(3, 8, D), torch.zeros(3, 4, 8, D)
    new, theta = torch.zeros(3, 2, D), torch.zeros(2, D)
    lse = torch.zeros(3, 4, 8)
    s = dict(stream=stream)
    return {
        "dequantize": lambda: kvbfp.dequantize(cache, 0, 0, 5, **s),
        "dequantize_paged": lambda: kvbfp.dequantize_paged(pool, table, 0, 0, 5, **s),
        "decode_attention": lambda: kvbfp.decode_attention(cache, rows, 512, 0.1, **s),
        "decode_attention_qbfp": lambda: kvbfp.decode_attention_qbfp(cache, rows, 512, 0.1, 8, **s),
        "decode_attention_rope": lambda: kvbfp.decode_attention_rope(cache, rows, 512, 0.1, theta, theta.int(), theta, **s),
        "decode_attention_paged": lambda: kvbfp.decode_attention_paged(pool, table, rows, 512, 0.1, **s),
        "append_decode_attention": lambda: kvbfp.append_decode_attention(cache, new, new, rows, 512, 0.1, **s),
        "append_decode_attention_paged": lambda: kvbfp.append_decode_attention_paged(pool, table, new, new, rows, 512, 0.1, **s),
        "decode_attention_multi": lambda: kvbfp.decode_attention_multi(cache, tokens, 512, 0.1, **s),
        "decode_attention_multi_paged": lambda: kvbfp.decode_attention_multi_paged(pool, table, tokens, 512, 0.1, **s),
        "decode_attention_scored": lambda: kvbfp.decode_attention_scored(cache, tokens, 512, 0.1, **s),
        "decode_attention_scored_paged": lambda: kvbfp.decode_attention_scored_paged(pool, table, tokens, 512, 0.1, **s),
        "accumulate_weights": lambda: kvbfp.accumulate_weights(cache, tokens, 512, 0.1, lse, **s),
        "accumulate_weights_paged": lambda: kvbfp.accumulate_weights_paged(pool, table, tokens, 512, 0.1, lse, **s),
    }


@pytest.mark.parametrize("name", list(calls(None, None, None, None)))
def test_made_on_the_stream_of_the_call(name, monkeypatch):
    z = lambda: torch.zeros(1, dtype=torch.uint8)  # noqa: E731
    cache = kvbfp.Cache(kvbfp.make_layout(D, 32, 4, 2, 3, 512), z(), z(), z(), z())
    pool = kvbfp.Cache(kvbfp.make_layout(D, 32, 4, 2, 20, 64), z(), z(), z(), z())
    table = torch.zeros(3, 8, dtype=torch.int32)
    todo = calls(cache, pool, table, 0x5000)[name]
    current, made = [None], []

    @contextlib.contextmanager
    def on(stream):
        current.append(stream)
        yield
        current.pop()

    def watched(make):
        def f(*args, **kw):
            made.append(current[-1])
            return make(*args, **kw)
        return f

    monkeypatch.setattr(kvbfp, "_lib", _Quiet())
    monkeypatch.setattr(kvbfp, "_dev_ptr", lambda t, dtype=None: None if t is None else t.data_ptr())
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle: handle)
    for make in ("empty", "empty_like", "zeros"):
        monkeypatch.setattr(torch, make, watched(getattr(torch, make)))
    todo()
    assert made and all(stream == 0x5000 for stream in made), made


@pytest.mark.gpu
@pytest.mark.parametrize("by_handle", [False, True])
def test_calls_on_another_stream_make_their_own_buffers(by_handle):
    # both streams busy: the current one would fill the weights too late, and take the workspace for its own tensors too early
    n, S = 12, 2000
    case = run_case(70, 3, 2, 4, n, S, 4, 32, BF16, lens=[S, S - 1, 900], tree=tree(1, n))
    plain = kvbfp.accumulate_weights(case["cache"], case["q"], S, case["scale"], case["lse"], rule=case["rule"], seq_len_dev=case["lens"])
    multi = kvbfp.decode_attention_multi(case["cache"], case["q"], S, case["scale"], seq_len_dev=case["lens"])
    big = torch.randn(8192, 8192, device="cuda", dtype=BF16)
    busy = {k: torch.empty_like(big) for k in "ab"}
    need = kvbfp.scored_workspace_bytes(case["cache"].layout, 8, n, S)
    side = torch.cuda.Stream()
    stream = side.cuda_stream if by_handle else side
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(side):
            torch.mm(big, big, out=busy["a"])
        torch.mm(big, big, out=busy["b"])
        args = dict(seq_len_dev=case["lens"], stream=stream)
        out = kvbfp.decode_attention_scored(case["cache"], case["q"], S, case["scale"], case["rule"], **args)
        other = kvbfp.decode_attention_multi(case["cache"], case["q"], S, case["scale"], **args)
        weights = kvbfp.accumulate_weights(case["cache"], case["q"], S, case["scale"], case["lse"], rule=case["rule"], **args)
        taken = [torch.full((need,), 0x7F, dtype=torch.uint8, device="cuda") for _ in range(4)]
        torch.cuda.synchronize()
        assert torch.equal(out, case["out"]) and torch.equal(other, multi) and torch.equal(weights, plain)
        assert all((t == 0x7F).all() for t in taken)


@pytest.mark.gpu
def test_the_default_stream_by_its_handle():
    case = run_case(71, 2, 2, 4, 5, 300, 4, 32, BF16, lens=[300, 20])
    got = kvbfp.decode_attention_scored(case["cache"], case["q"], 300, case["scale"], case["rule"], seq_len_dev=case["lens"], stream=0)
    weights = kvbfp.accumulate_weights(case["cache"], case["q"], 300, case["scale"], case["lse"], seq_len_dev=case["lens"],
                                       stream=torch.cuda.default_stream())
    again = kvbfp.accumulate_weights(case["cache"], case["q"], 300, case["scale"], case["lse"], seq_len_dev=case["lens"], stream=0)
    assert torch.equal(got, case["out"]) and torch.equal(weights, again)
    assert np.allclose(R.f64(weights).sum(-1), 20.0, atol=1e-2)

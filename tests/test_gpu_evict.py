"""The weights that cached tokens collect and the eviction by them, against plain forms; and attention, weights, eviction and attention
again as a serving loop runs them."""
import numpy as np
import pytest
import torch

import scored_ref as R
from paper_2403_20137_amd import kvbfp
from test_gpu_scored import BF16, F16, F32, run_case, tree
from util import assert_attention_close, dev_i32

pytestmark = pytest.mark.gpu
D = 128


def collect(case, before, decay, S, in_place=False):
    keys = case["keys"]
    B, n, Hq, _ = case["q"].shape
    rng = np.random.default_rng(1)
    w_in = torch.from_numpy(rng.random((B, keys.shape[1], S + 3)).astype(np.float32)).cuda() if before else None
    out = w_in if in_place else torch.full((B, keys.shape[1], S + 3), -5.0, device="cuda")
    old = w_in.clone() if before else None
    args = dict(decay=decay, rule=case["rule"], seq_len_dev=case["lens"], perm_k=dev_i32(case["pk"]))
    if case["table"] is not None:
        got = kvbfp.accumulate_weights_paged(case["cache"], case["table"], case["q"], S, case["scale"], case["lse"], w_in, out, **args)
    else:
        got = kvbfp.accumulate_weights(case["cache"], case["q"], S, case["scale"], case["lse"], w_in, out, **args)
    torch.cuda.synchronize()
    assert got is out
    want, tol = R.weights(R.f64(case["q"]), keys, case["scale"], case["sizes"], R.f64(case["lse"]), None if old is None else R.f64(old)[..., :S],
                          float(np.float32(decay)), case["pk"], case["ref"])
    have = R.f64(got)
    rest = R.f64(old) if in_place else np.full(have.shape, -5.0)
    for b, size in enumerate(case["sizes"]):
        off = np.abs(have[b, :, :size] - want[b, :, :size])
        assert (off <= tol[b, :, :size]).all(), (b, np.max(off / tol[b, :, :size]))
        assert np.array_equal(have[b, :, size:], rest[b, :, size:])          # behind the last token nothing is written
    return got


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("bits,block", [(4, 16), (4, 32), (4, 64), (4, 128), (8, 16), (8, 64)])
def test_weights_formats(dtype, bits, block):
    case = run_case(2, 2, 2, 3, 5, 300, bits, block, dtype, lens=[300, 211], perm=True, cap=20.0, slopes=True, tree=tree(1, 5, 2))
    collect(case, True, 0.75, 300)
    collect(case, True, 1.0, 300, in_place=True)
    collect(case, False, 0.5, 300)


@pytest.mark.parametrize("S", [1, 16, 31, 33, 127, 129, 700])
@pytest.mark.parametrize("G,n", [(1, 1), (4, 1), (16, 1), (17, 1), (4, 9), (3, 40)])
def test_weights_sizes(S, G, n):
    case = run_case(S + n, 3, 2, G, n, S, 4, 32, BF16, lens=[S, S // 2, 0], tree=tree(n, n), window=max(1, S // 3))
    collect(case, True, 0.9, S)


@pytest.mark.parametrize("page", [16, 64])
def test_weights_pages(page):
    case = run_case(page, 3, 2, 4, 6, 333, 8, 32, F16, page=page, lens=[333, 16, 47], prefix=[20, 20, 20], first=[[100] * 6] * 3)
    collect(case, True, 0.9, 333)


def test_weights_of_all_rows_add_up():
    # every row that sees something gives 1 in all: 8 query tokens of 4 heads per kv-head; sums of some 500 rounded numbers
    case = run_case(5, 1, 2, 4, 8, 500, 4, 32, F32)
    got = collect(case, False, 1.0, 500)
    assert np.allclose(R.f64(got)[0, :, :500].sum(-1), 32.0, rtol=0, atol=32 * 2e-5)


def test_weights_are_the_same_every_time():
    case = run_case(6, 2, 2, 4, 17, 700, 4, 32, BF16)
    a, b = collect(case, True, 0.9, 700), collect(case, True, 0.9, 700)
    assert torch.equal(a[..., :700], b[..., :700])


# ---- eviction ----

def evict_case(seed, B, H, S, bits, block, n_keep, n_first, n_recent, lens=None, page=0, dst_page=0, values=None, same_pool=False, slack=2):
    rng = np.random.default_rng(seed)
    cache, table = R.make_cache(rng, B, H, S, bits, block, page)
    w = rng.random((B, H, S + 1)).astype(np.float32) if values is None else np.broadcast_to(values, (B, H, S + 1)).astype(np.float32)
    w = torch.from_numpy(np.ascontiguousarray(w)).cuda()
    sizes = list(lens) if lens is not None else [S] * B
    cut = n_keep + slack
    if page:
        dst_page = page if same_pool else dst_page or page
        per = -(-cut // dst_page)
        if same_pool:                                        # the free pages of a larger pool
            old, pages = cache, cache.layout.batch
            pool = kvbfp.alloc_cache(kvbfp.make_layout(D, block, bits, H, pages + B * per, page), fill=0xFF)
            for a, b in zip(old.planes(), pool.planes()):
                b[:pages] = a
            cache = dst = pool
            dst_table = torch.arange(pages, pages + B * per, dtype=torch.int32, device="cuda").view(B, per)
        else:
            dst = kvbfp.alloc_cache(kvbfp.make_layout(D, block, bits, H, B * per + 1, dst_page), fill=0xFF)
            dst_table = torch.from_numpy(rng.permutation(B * per + 1)[: B * per].reshape(B, per).astype(np.int32)).cuda()
    else:
        dst, dst_table = kvbfp.alloc_cache(kvbfp.make_layout(D, block, bits, H, B, cut), fill=0xFF), None
    before = [p.clone() for p in cache.planes()]
    kept = torch.full((B, H, n_keep), -77, dtype=torch.int32, device="cuda")
    new_len = torch.full((B,), -77, dtype=torch.int32, device="cuda")
    w_out = torch.full((B, H, n_keep), -77.0, device="cuda")
    lens_dev = None if lens is None else dev_i32(np.array(lens))
    args = (w, S, n_keep, n_first, n_recent, kept, new_len)
    if page:
        kvbfp.evict_paged(cache, table, dst, dst_table, *args, weights_out=w_out, seq_len_dev=lens_dev)
    else:
        kvbfp.evict(cache, dst, *args, weights_out=w_out, seq_len_dev=lens_dev)
    torch.cuda.synchronize()

    def flat(planes, t):
        out = []
        for p in planes:
            p = p.cpu().numpy()
            out.append(p if t is None else p[t.cpu().numpy()].transpose(0, 2, 1, 3, 4).reshape(t.shape[0], H, -1, p.shape[-1]))
        return out

    src, got = flat(before, table), flat(dst.planes(), dst_table)
    wn, kn, wo = w.cpu().numpy(), kept.cpu().numpy(), w_out.cpu().numpy()
    for b, size in enumerate(sizes):
        count = min(size, n_keep)
        assert int(new_len[b]) == count
        for h in range(H):
            stay = R.keep(wn[b, h], size, n_keep, n_first, n_recent)
            assert kn[b, h].tolist() == stay + [-1] * (n_keep - count), (b, h)
            assert np.array_equal(wo[b, h, :count], wn[b, h, stay], equal_nan=True) and (wo[b, h, count:] == -77.0).all()
            for s, g in zip(src, got):
                assert np.array_equal(g[b, h, :count], s[b, h, stay])
                assert (g[b, h, count:] == 0xFF).all()       # rows behind the last one that stays are left as they were
    if not same_pool:
        for a, p in zip(before, cache.planes()):
            assert torch.equal(a, p)


@pytest.mark.parametrize("bits,block", [(4, 16), (4, 32), (4, 64), (4, 128), (8, 16), (8, 32), (8, 128)])
def test_evict_formats(bits, block):
    evict_case(1, 2, 3, 500, bits, block, 200, 4, 32, lens=[500, 321])


@pytest.mark.parametrize("S,keep,first,recent", [(1, 1, 0, 0), (2, 1, 0, 0), (2, 1, 1, 0), (2, 1, 0, 1), (64, 63, 0, 0), (65, 64, 32, 32),
                                                 (1000, 1, 0, 0), (1000, 999, 3, 5), (1025, 1024, 0, 1024), (1025, 500, 500, 0),
                                                 (2047, 700, 0, 0), (3001, 1500, 16, 700), (70000, 5000, 4, 100)])
def test_evict_sizes(S, keep, first, recent):
    evict_case(S + keep, 1 if S > 9999 else 2, 2, S, 4, 32, keep, first, recent, lens=None if S > 9999 else [S, S // 2])


def test_evict_keeps_short_and_empty_sequences_whole():
    evict_case(3, 4, 2, 300, 4, 32, 150, 2, 10, lens=[300, 150, 149, 0])
    evict_case(4, 2, 2, 40, 4, 32, 60, 2, 10)


def test_evict_ties_and_unusual_weights():
    S = 400
    rng = np.random.default_rng(8)
    evict_case(5, 1, 2, S, 4, 32, 100, 3, 7, values=np.zeros(S + 1))                       # all alike: the lowest indices
    evict_case(6, 1, 2, S, 4, 32, 100, 0, 0, values=rng.integers(0, 3, S + 1))
    evict_case(7, 1, 2, S, 4, 32, 100, 0, 0, values=np.where(np.arange(S + 1) % 2, 0.0, -0.0))
    special = rng.standard_normal(S + 1)
    special[::7], special[1::7], special[2::7] = np.nan, np.inf, -np.inf
    evict_case(8, 1, 2, S, 4, 32, 100, 0, 0, values=special)
    evict_case(8, 1, 2, S, 4, 32, 380, 0, 0, values=special)
    evict_case(9, 1, 1, S, 4, 32, 100, 0, 0, values=rng.standard_normal(S + 1) * 1e-40)    # subnormal numbers


@pytest.mark.parametrize("page,dst_page", [(16, 16), (64, 16), (32, 256)])
def test_evict_pages(page, dst_page):
    evict_case(page, 3, 2, 333, 4, 32, 120, 4, 20, lens=[333, 120, 50], page=page, dst_page=dst_page)
    evict_case(page, 2, 2, 200, 8, 16, 90, 0, 90, page=page, dst_page=dst_page)


def test_evict_to_other_pages_of_the_same_pool():
    evict_case(10, 2, 2, 300, 4, 32, 100, 4, 20, lens=[300, 64], page=32, same_pool=True)


def test_serving_loop():
    """Draft trees verified, weights collected, the cache evicted and attended again, with appended tokens in between."""
    rng = np.random.default_rng(77)
    B, H, G, S, n, keep = 2, 2, 4, 260, 7, 100
    cache, _ = R.make_cache(rng, B, H, S, 4, 32, extra=40)
    lens = dev_i32(np.array([260, 200]))
    sizes = [260, 200]
    scale = float(np.float32(0.09))
    weights = torch.zeros(B, H, 300, device="cuda")
    want_w = np.zeros((B, H, 300))
    tol_w = np.zeros((B, H, 300))
    for step in range(3):
        masks = [R.random_tree(rng, n) for _ in range(B)]
        rule = kvbfp.make_score_rule(cap=30.0, tree_mask=torch.tensor(masks, dtype=torch.int64).cuda())
        q = torch.from_numpy(rng.standard_normal((B, n, H * G, D)).astype(np.float32)).to(BF16).cuda()
        lse = torch.empty(B, n, H * G, device="cuda")
        out = kvbfp.decode_attention_scored(cache, q, 300, scale, rule, seq_len_dev=lens, lse=lse)
        kvbfp.accumulate_weights(cache, q, 300, scale, lse, weights, decay=0.5, rule=rule, seq_len_dev=lens)
        keys, values = R.decoded(cache, 0), R.decoded(cache, 1)
        want, _, _ = R.attention(R.f64(q), keys, values, scale, sizes, rule={"cap": 30.0, "tree": masks})
        assert_attention_close(out.view(B, -1, D), want.reshape(B, -1, D), BF16, "loop %d" % step)
        new, tol = R.weights(R.f64(q), keys, scale, sizes, R.f64(lse), want_w[..., :keys.shape[2]], 0.5, rule={"cap": 30.0, "tree": masks})
        for b in range(B):
            want_w[b, :, :sizes[b]], tol_w[b, :, :sizes[b]] = new[b, :, :sizes[b]], 0.5 * tol_w[b, :, :sizes[b]] + tol[b, :, :sizes[b]]
            assert (np.abs(R.f64(weights)[b, :, :sizes[b]] - want_w[b, :, :sizes[b]]) <= tol_w[b, :, :sizes[b]]).all()
        x = torch.from_numpy(rng.standard_normal((B, 5, H, D)).astype(np.float32)).cuda()
        kvbfp.quantize_append(cache, x, x, pos_dev=lens)
        lens = lens + 5
        sizes = [s + 5 for s in sizes]
    dst = kvbfp.alloc_cache(kvbfp.make_layout(D, 32, 4, H, B, keep + 20), fill=0xFF)
    kept, new_len = torch.empty(B, H, keep, dtype=torch.int32, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
    left = torch.zeros(B, H, keep, device="cuda")
    kvbfp.evict(cache, dst, weights, 300, keep, 4, 16, kept, new_len, weights_out=left, seq_len_dev=lens)
    w = weights.cpu().numpy()
    for b in range(B):
        for h in range(H):
            assert kept[b, h].tolist() == R.keep(w[b, h], sizes[b], keep, 4, 16)
    assert torch.equal(left, weights.gather(2, kept.long()))
    q = torch.from_numpy(rng.standard_normal((B, 1, H * G, D)).astype(np.float32)).to(BF16).cuda()
    out = kvbfp.decode_attention_scored(dst, q, keep, scale, seq_len_dev=new_len)
    old_k, old_v = R.decoded(cache, 0), R.decoded(cache, 1)
    at = kept.cpu().numpy()[..., None].astype(np.int64)
    want, _, _ = R.attention(R.f64(q), np.take_along_axis(old_k, at, 2), np.take_along_axis(old_v, at, 2), scale, [keep] * B)
    assert_attention_close(out.view(B, -1, D), want.reshape(B, -1, D), BF16, "after eviction")

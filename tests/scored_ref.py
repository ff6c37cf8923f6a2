"""Plain 64-bit forms of attention with a rule on its scores, of the weights that cached tokens collect and of their eviction, one
sequence, query token and head at a time, with bounds on what fp32 arithmetic may add."""
import numpy as np
import torch

from paper_2403_20137_amd import kvbfp

D = 128
U = 2.0 ** -24                                    # half a step of fp32, relative


def f64(t):
    return t.detach().cpu().double().numpy()


def decoded(cache, which, table=None, length=None):
    """[batch][head][token][128] in 64 bits, from the bytes."""
    L = cache.layout
    mant, exps = (x.cpu().numpy() for x in (cache.planes()[2 * which], cache.planes()[2 * which + 1]))
    if table is not None:
        t = table.cpu().numpy()
        mant, exps = (x[t].transpose(0, 2, 1, 3, 4).reshape(t.shape[0], L.n_kv_heads, -1, x.shape[-1]) for x in (mant, exps))
    if length is not None:
        mant, exps = mant[:, :, :length], exps[:, :, :length]
    if L.mant_bits == 4:
        codes = np.empty(mant.shape[:-1] + (D,), np.int64)
        codes[..., 0::2], codes[..., 1::2] = mant & 15, mant >> 4
    else:
        codes = mant.astype(np.int64)
    half = 1 << (L.mant_bits - 1)
    signed = np.where(codes >= half, half - codes, codes).astype(np.float64)
    return np.ldexp(signed, np.repeat(exps.astype(np.int64) - 127 - (L.mant_bits - 2), L.block, axis=-1))


def seen_and_far(n, size, mask=None, window=0, first=None, prefix=0):
    """bool [n][size], int [n][size] for one sequence of `size` tokens whose last n are the query tokens."""
    base = size - n
    masks = [(2 << i) - 1 for i in range(n)] if mask is None else [int(x) & (2 ** n - 1) for x in mask]
    depth = [bin(m & ~(1 << i)).count("1") for i, m in enumerate(masks)]
    seen, far = np.zeros((n, size), bool), np.zeros((n, size), np.int64)
    for i in range(n):
        for t in range(size):
            node = t - base
            far[i, t] = depth[i] - depth[node] if node >= 0 else base + depth[i] - t
            ok = bool(masks[i] >> node & 1) if node >= 0 else True
            ok = ok and (first is None or t >= first[i]) and (window == 0 or far[i, t] < window)
            seen[i, t] = ok or t < prefix
    return seen, far


def scores(q, keys, scale, sizes, perm_k, rule):
    """q: [B][n][Hq][128], keys: decoded.  Yields (b, i, head, y with -inf where unseen, bound on its error in fp32)."""
    B, n, Hq, _ = q.shape
    G = Hq // keys.shape[1]
    cap, slopes = rule.get("cap", 0.0), rule.get("slopes")
    for b in range(B):
        size = sizes[b]
        if size == 0:
            continue
        mask = rule.get("tree")
        mask = mask if mask is None or np.ndim(mask) == 1 else mask[b]
        seen, far = seen_and_far(n, size, mask, rule.get("window", 0), None if rule.get("first") is None else rule["first"][b],
                                 0 if rule.get("prefix") is None else rule["prefix"][b])
        for head in range(Hq):
            h = head // G
            k = keys[b, h, :size]
            qq = q[b, :, head][:, perm_k[h]] if perm_k is not None else q[b, :, head]
            y = qq @ k.T * scale
            # products summed in fp32 in any order, the scale, and the change of base on the way
            off = (D + 8) * U * (np.abs(qq) @ np.abs(k).T * abs(scale))
            if cap:
                y = cap * np.tanh(y / cap)
                # up to eight roundings of the result, or of the cap where the exponential form stands alone (16-bit I/O)
            off = off + 8 * U * np.maximum(np.abs(y), cap if rule.get("by_exp") and cap <= 64 else 0)
            if slopes is not None:
                bias = slopes[head] * np.abs(far)
                y = y - bias
                off = off + 4 * U * (np.abs(bias) + np.abs(y))
            yield b, head, np.where(seen, y, -np.inf), np.where(seen, off, 0.0)


def attention(q, keys, values, scale, sizes, perm_k=None, perm_v=None, rule=None):
    """out, lse, bound on lse's error."""
    B, n, Hq, _ = q.shape
    G = Hq // keys.shape[1]
    out, lse, tol = np.zeros(q.shape), np.full(q.shape[:3], -np.inf), np.zeros(q.shape[:3])
    for b, head, y, off in scores(q, keys, scale, sizes, perm_k, rule or {}):
        h = head // G
        for i in range(n):
            if np.isinf(y[i]).all():
                continue
            top = y[i].max()
            p = np.exp(y[i] - top)
            o = p @ values[b, h, :sizes[b]] / p.sum()
            if perm_v is not None:
                out[b, i, head, perm_v[h]] = o
            else:
                out[b, i, head] = o
            lse[b, i, head] = top + np.log(p.sum())
            # lse moves by at most the largest error of a score; a few roundings of itself and of the sum
            tol[b, i, head] = off[i].max() + 8 * U * (abs(lse[b, i, head]) + 1) + sizes[b] * U
    return out, lse, tol


def weights(q, keys, scale, sizes, lse, before, decay, perm_k=None, rule=None):
    """The sums and a bound on their error; rows whose lse is -inf add nothing."""
    B, n, Hq, _ = q.shape
    H = keys.shape[1]
    new = np.zeros((B, H, keys.shape[2])) if before is None else decay * before
    tol = 2 * U * np.abs(new)
    for b, head, y, off in scores(q, keys, scale, sizes, perm_k, rule or {}):
        h = head // (Hq // H)
        for i in range(n):
            if np.isinf(lse[b, i, head]):
                continue
            p = np.exp(y[i] - lse[b, i, head])
            new[b, h, :sizes[b]] += p
            tol[b, h, :sizes[b]] += p * (2 * off[i] + 8 * U * (np.abs(lse[b, i, head]) + np.where(np.isinf(y[i]), 0, np.abs(y[i])) + 1) + n * Hq * U)
    return new, tol + 1e-37


def keep(w, size, n_keep, n_first, n_recent):
    """Indices that stay, in order; w: numpy float32 [size]."""
    if size <= n_keep:
        return list(range(size))
    middle = list(range(n_first, size - n_recent))
    rank = lambda t: (np.isnan(w[t]), -w[t] if not np.isnan(w[t]) else 0.0, t)  # noqa: E731
    best = sorted(middle, key=rank)[: n_keep - n_first - n_recent]
    return list(range(n_first)) + sorted(best) + list(range(size - n_recent, size))


def random_tree(rng, n):
    """64-bit ancestor masks (as signed numbers) of a random forest of n nodes."""
    seen = []
    for i in range(n):
        up = int(rng.integers(max(0, i - 6), i + 1)) if i else 0
        seen.append((seen[up] if up < i else 0) | 1 << i)
    return [s - (1 << 64) if s >> 63 else s for s in seen]


def make_cache(rng, B, H, S, bits, block, page=0, extra=0):
    """A cache of S tokens whose rows have outlier channels, written by quantize_append; over pages where page > 0, in any order.
    Everything that no token of the cache occupies holds 0xFF.  Returns (cache, table or None)."""
    def rows():
        x = rng.standard_normal((B, S, H, D)).astype(np.float32)
        x[..., rng.choice(D, 4, replace=False)] *= 10
        return torch.from_numpy(x).cuda()

    if not page:
        cache = kvbfp.alloc_cache(kvbfp.make_layout(D, block, bits, H, B, S + extra), fill=0xFF)
        kvbfp.quantize_append(cache, rows(), rows())
        return cache, None
    per = -(-S // page)
    pool = kvbfp.alloc_cache(kvbfp.make_layout(D, block, bits, H, B * per + 2, page), fill=0xFF)
    table = torch.from_numpy(rng.permutation(B * per + 2)[: B * per].reshape(B, per).astype(np.int32)).cuda()
    kvbfp.quantize_append_paged(pool, table, rows(), rows())
    return pool, table

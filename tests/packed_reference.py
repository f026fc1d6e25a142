"""The 4-bit cache in plain float64 and bytes, value by value of the definition in include/flasheval_packed.h, for the tests of
its calls: what a block is held as, where a row lies in its page, the weights that rows receive, and eviction."""
import math

import numpy as np

SIZES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def hold(x):
    """(codes [..][n / 2], scales [..][n / 32]) uint8 of float64 rows x [..][n]: every block's smallest power of two, every
    value's nearest size, found among all of them."""
    x = np.asarray(x, np.float64)
    b = x.reshape(*x.shape[:-1], -1, 32)
    top = np.abs(b).max(-1)
    number = np.isfinite(b).all(-1)
    units = 2.0 ** (np.arange(2, 253) - 127.0)
    e = np.full(top.shape, 255, np.int64)
    e[number] = np.minimum(np.searchsorted(6 * units, top[number]), 250) + 2   # the first unit with top <= 6 units
    unit = np.where(number, 2.0 ** (np.minimum(e, 252) - 127.0), 1.0)
    a = np.where(number[..., None], np.abs(b), 0.0) / unit[..., None]
    far = np.abs(a[..., None] - np.array(SIZES))
    near = far.min(-1, keepdims=True)
    hit = far == near                                                          # one, or two that are as near
    low = hit.argmax(-1)
    code = np.where((low % 2 == 1) & (hit.sum(-1) == 2), low + 1, low)
    code = np.where(number[..., None], code | (np.signbit(b) << 3), 0).reshape(x.shape)
    return (code[..., ::2] | code[..., 1::2] << 4).astype(np.uint8), e.astype(np.uint8)


def values(codes, scales):
    """The float64 values [..][2 n] that codes [..][n] and scales [..][n / 16] stand for."""
    nib = np.stack((codes & 15, codes >> 4), -1).reshape(*codes.shape[:-1], -1)
    v = np.array(SIZES)[nib & 7] * np.where(nib & 8, -1.0, 1.0)
    unit = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return v * np.repeat(unit, 32, -1)


def held_values(x):
    return values(*hold(x))


def head_bytes(P, dh):
    return -(-P * (dh + dh // 16) // 16) * 16


def place(P, dh, part, r):
    """Byte ranges in a head's part of a page of row r's codes and scales, of the keys (part 0) or the values (1)."""
    c, s = (part * P + r) * (dh // 2), P * dh + (part * P + r) * (dh // 32)
    return slice(c, c + dh // 2), slice(s, s + dh // 32)


def write(pages, page, r, P, dh, k, v):
    """Rows k, v [Hkv][dh] float64 into row r of a page of pages [n][Hkv][head_bytes]."""
    for part, x in ((0, k), (1, v)):
        codes, scales = hold(x)
        c, s = place(P, dh, part, r)
        pages[page, :, c], pages[page, :, s] = codes, scales


def write_rows(pages, page, r, P, dh, k, v):
    """Rows k, v [n][Hkv][dh] into rows r [n] of pages page [n]."""
    for part, x in ((0, k), (1, v)):
        for bytes_, width, start in zip(hold(x), (dh // 2, dh // 32), (0, P * dh)):
            at = start + (part * P + r) * width
            h, c = np.arange(pages.shape[1])[None, :, None], np.arange(width)[None, None]
            pages[page[:, None, None], h, at[:, None, None] + c] = bytes_


def read(pages, page, r, P, dh):
    """(k, v) [Hkv][dh] of a row."""
    return tuple(values(pages[page, :, place(P, dh, part, r)[0]], pages[page, :, place(P, dh, part, r)[1]]) for part in (0, 1))


def weigh(q, ck, ok, lse, *, causal, scale, ctx_len, q_len, own_len, ctx_w, own_w, ctx_seen=None, own_seen=None):
    """{name: (value, bound)} of the weights [B][Hkv][T] and [B][K][Hkv][L] after the rows q [B][K][S][H][dh] with lse
    [B][K][S][H] have met the keys ck [B][T][Hkv][dh], ok [B][K][L][Hkv][dh]; entries past the lengths are left out (NaN bound).

    Bound: a score is off by (dh + 2) e smax, its difference to lse and the exponent by 2 e (smax + |lse|), exp2 by 4 e, so a
    weight is off by r = e ((dh + 6) smax + 4 |lse| + 8) relative; a sum of N weights and w adds (N + 2) e of their sum."""
    B, K, S, H, dh = q.shape
    Hkv = ctx_w.shape[1]
    G, e = H // Hkv, 2.0 ** -24
    ctx, one = ctx_w.astype(np.float64).copy(), own_w.astype(np.float64).copy()
    cb, ob = np.zeros_like(ctx), np.zeros_like(one)
    rows_c = np.zeros(B)
    rows_o = np.zeros((B, K))
    for b in range(B):
        for k in range(K):
            n, m, t = q_len[b, k], own_len[b, k], ctx_len[b]
            for i in range(n):
                for h in range(H):
                    l = float(lse[b, k, i, h])
                    if l == -math.inf:
                        continue
                    g = h // G
                    rows_c[b] += 1
                    rows_o[b, k] += 1
                    to = min(max(m - n + i + 1, 0), m) if causal else m
                    for keys, seen, w, bound, cut in ((ck[b, :t, g], ctx_seen and ctx_seen[b], ctx[b, g], cb[b, g], t),
                                                      (ok[b, k, :to, g], own_seen and own_seen[b][k], one[b, k, g], ob[b, k, g], to)):
                        x = q[b, k, i, h]
                        p = np.exp(keys @ x * scale - l)
                        r = e * ((dh + 6) * (np.abs(keys) @ np.abs(x)) * abs(scale) + 4 * abs(l) + 8)
                        live = np.ones(cut, bool) if seen is None else np.array(seen[:cut], bool)
                        w[:cut] += np.where(live, p, 0)
                        bound[:cut] += np.where(live, p * r, 0)
    cb += e * (rows_c[:, None, None] + 2) * np.abs(ctx)
    ob += e * (rows_o[:, :, None, None] + 2) * np.abs(one)
    for b in range(B):
        cb[b, :, ctx_len[b]:] = np.nan
        for k in range(K):
            ob[b, k, :, own_len[b, k]:] = np.nan
    return dict(ctx_w=(ctx, cb), own_w=(one, ob))


def evict_rows(w, n, keep, first, recent):
    """The rows of one sequence and head that stay, ascending, by sorting (weight, index) pairs."""
    m = min(keep, n)
    first = min(first, m)
    recent = min(recent, m - first)
    rank = lambda i: (1, 0.0, i) if math.isnan(w[i]) else (0, -float(w[i]), i)         # noqa: E731
    rest = sorted(range(first, n - recent), key=rank)[:m - first - recent]
    return sorted(list(range(first)) + rest + list(range(n - recent, n)))

"""Plain float64 shared-prefix attention, its gradient and the paged-cache append, list by list and row
by row of the definition in include/flasheval_prefix.h, for the tests of those calls.  `attend` also
derives how far a kernel that rounds as the header says may be off."""
import numpy as np

HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}     # a rounding is off by at most this, relative
TWO_PARTS = 2.0 ** -16     # a number as two bf16: the second is off by a half step of what the first left, 2^-8 of it
REST = 2.0 ** -15          # out with its rest: 16 bits of the significand, the others cut


def clamp_lengths(B, K, S, T, L, ctx_len, q_len, own_len):
    full = lambda v, n, shape: np.full(shape, n) if v is None else np.clip(np.asarray(v, np.int64).reshape(shape), 0, n)  # noqa: E731
    return full(ctx_len, T, (B,)), full(q_len, S, (B, K)), full(own_len, L, (B, K))


def attend(q, ck, cv, ok, ov, *, dtype, causal, scale=None, ctx_len=None, q_len=None, own_len=None, dout=None, seen=None,
           up_out=None, up_own=None, u_rest=None):
    """q [B][K][S][H][dh], ck/cv [B][T][Hkv][dh], ok/ov [B][K][L][Hkv][dh] (float64; anything outside the lengths).
    `seen` [B][K][L]: own keys that count at all (pages inside the pool).  Returns {name: (value, bound)} of out and
    lse, and with dout of dq, dck, dcv, dok, dov.

    Bounds, u the half step of the type, e = 2^-24, per row with n keys and smax = max_j scale sum |q||k_j|:
      a score's dot product of dh terms is off by (dh + 2) e smax; the probability's exponent is the difference
      of two scores, scaled and rounded a few more times, and the sum has n terms, so p is off by
        rp = 2 e ((dh + 8) smax + |lse| + n + 16)              relative
      (exp itself is good to a few e), plus u where p is rounded for a product (bf16);
      out   is off by (rp + u_p + n e) sum p|v|, and u |out| for its rounding;
      delta = dout.out takes that error times |dout|, plus dh e sum |dout||out|;
      dp    is off by dh e sum |dout||v|;
      ds = p (dp - delta) is off by p (err dp + err delta) + (rp + u_p + 2 e) |ds|, and dq, dk sum it times |k|, |q|;
      dv sums (rp + u_p) p |dout|; the sums of N terms add N e times the sum of the terms' sizes.
    up_out, up_own: another u for the p of out, and for the p and ds of own keys' gradients; u_rest: D = dout.out is taken
    from an out that is off by this, relative, in place of its rounding (dq, dk and dv of shared keys keep u for p and ds).
    FE_F32's products in three parts are good to 2^-21 = 8 e each and add a part's six sums every 32 terms: both lie inside
    (dh + 2) e for a score and dh e for dp (dh >= 32), and inside rp >= 32 e in the sums over keys and rows."""
    B, K, S, H, dh = q.shape
    T, Hkv, L = ck.shape[1], ck.shape[2] if ck.shape[1] else ok.shape[3], ok.shape[2]
    G, scale = H // Hkv, dh ** -0.5 if scale is None else scale
    u, e = HALF_STEP[dtype], 2.0 ** -24
    up = u if dtype == "bf16" else 0.0
    up_out, up_own = up if up_out is None else up_out, up if up_own is None else up_own
    nc, nq, no = clamp_lengths(B, K, S, T, L, ctx_len, q_len, own_len)
    zero = lambda *shape: (np.zeros(shape), np.zeros(shape))     # noqa: E731
    out, dq = zero(B, K, S, H, dh), zero(B, K, S, H, dh)
    lse = (np.full((B, K, S, H), -np.inf), np.zeros((B, K, S, H)))
    dck, dcv, dok, dov = zero(B, T, Hkv, dh), zero(B, T, Hkv, dh), zero(B, K, L, Hkv, dh), zero(B, K, L, Hkv, dh)
    terms_c = np.zeros(B)
    for b in range(B):
        for k in range(K):
            n, m, t = nq[b, k], no[b, k], nc[b]
            if n == 0:
                continue
            see = np.ones((n, t + m), bool)
            if causal:
                see[:, t:] = np.arange(m)[None] <= (m - n + np.arange(n))[:, None]
            if seen is not None:
                see[:, t:] &= seen[b, k, :m]
            for h in range(H):
                g = h // G
                kk = np.concatenate((ck[b, :t, g], ok[b, k, :m, g])).reshape(-1, dh)
                vv = np.concatenate((cv[b, :t, g], ov[b, k, :m, g])).reshape(-1, dh)
                if seen is not None:
                    gone = np.concatenate((np.zeros(t, bool), ~seen[b, k, :m]))
                    kk[gone] = vv[gone] = 0
                qq = q[b, k, :n, h]
                some = see.any(1)
                if not some.any():
                    continue
                s = np.where(see, qq @ kk.T * scale, -np.inf)
                mx = np.where(some, s.max(1), 0.0)
                ex = np.exp(s - mx[:, None])
                l = np.where(some, ex.sum(1), 1.0)
                p = ex / l[:, None]
                ls = np.where(some, mx + np.log(l), 0.0)
                lse[0][b, k, :n, h] = np.where(some, ls, -np.inf)
                o = p @ vv
                out[0][b, k, :n, h] = o
                smax = np.where(see, np.abs(qq) @ np.abs(kk).T * abs(scale), 0.0).max(1)
                rp = 2 * e * ((dh + 8) * smax + np.abs(ls) + t + m + 16)
                oa = p @ np.abs(vv)
                eo = (rp + up_out + (t + m) * e)[:, None] * oa
                out[1][b, k, :n, h] = eo + u * (np.abs(o) + eo)
                lse[1][b, k, :n, h] = rp + 4 * e * (np.abs(ls) + 1)
                if dout is None:
                    continue
                do = dout[b, k, :n, h]
                delta = (do * o).sum(1)
                ed = out[1][b, k, :n, h] if u_rest is None else eo + u_rest * (np.abs(o) + eo)
                ed = (np.abs(do) * ed).sum(1) + dh * e * (np.abs(do) * np.abs(o)).sum(1)
                dp = do @ vv.T
                dpa = np.abs(do) @ np.abs(vv).T
                ds = p * (dp - delta[:, None])
                ups = np.where(np.arange(t + m) < t, up, up_own)
                es = p * (dh * e * dpa + ed[:, None] + 2 * e * (dpa + np.abs(delta)[:, None]))
                eq = es + (rp + up + 4 * e)[:, None] * np.abs(ds)
                es = es + (rp[:, None] + ups + 4 * e) * np.abs(ds)
                ep = (rp[:, None] + ups) * p
                nk, nr = t + m, K * S * G
                d = ds @ kk * scale
                err = scale * (eq @ np.abs(kk) + nk * e * (np.abs(ds) + eq) @ np.abs(kk))
                dq[0][b, k, :n, h] = d
                dq[1][b, k, :n, h] = abs(err) + u * (np.abs(d) + abs(err))
                dk, dv = ds.T @ qq * scale, p.T @ do
                ek = abs(scale) * ((es + nr * e * (np.abs(ds) + es)).T @ np.abs(qq))
                ev = (ep + nr * e * (p + ep)).T @ np.abs(do)
                for (val, bound), x, ex_ in ((dck, dk, ek), (dcv, dv, ev)):
                    val[b, :t, g] += x[:t]
                    bound[b, :t, g] += ex_[:t]
                for (val, bound), x, ex_ in ((dok, dk, ek), (dov, dv, ev)):
                    val[b, k, :m, g] += x[t:]
                    bound[b, k, :m, g] += ex_[t:]
    res = dict(out=out, lse=lse)
    if dout is not None:
        res["dq"] = dq
        for name, (val, bound) in dict(dck=dck, dcv=dcv, dok=dok, dov=dov).items():
            res[name] = (val, bound + u * (np.abs(val) + bound))
    return res


def turned(x, pos, freq, neighbours):
    """x [..][heads][dh] float64 with its first 2 len(freq) columns turned by pos * freq (pos [..])."""
    n = len(freq)
    y = x.copy()
    ang = pos[..., None, None] * freq
    ia, ib = (np.arange(0, 2 * n, 2), np.arange(1, 2 * n, 2)) if neighbours else (np.arange(n), np.arange(n, 2 * n))
    a, b = x[..., ia], x[..., ib]
    y[..., ia] = a * np.cos(ang) - b * np.sin(ang)
    y[..., ib] = b * np.cos(ang) + a * np.sin(ang)
    return y


def turned_bound(x, freq, neighbours, dtype):
    """Bound of |kernel - turned|: each product and the sum round to fp32 and sine and cosine are good to 2^-22, then one
    rounding to the type: (u + 2^-21) (|a| + |b|); copied columns are exact."""
    n = len(freq)
    ia, ib = (np.arange(0, 2 * n, 2), np.arange(1, 2 * n, 2)) if neighbours else (np.arange(n), np.arange(n, 2 * n))
    y = np.zeros_like(x)
    y[..., ia] = y[..., ib] = (HALF_STEP[dtype] + 2.0 ** -21) * (np.abs(x[..., ia]) + np.abs(x[..., ib]))
    return y


def append(k, v, q, k_pages, v_pages, table, length, new_len, pos0, freq, neighbours):
    """The cache and q_out after the call, and the status, by loops; arrays are copied.  Rows of q_out that the call
    leaves alone are NaN."""
    N, S = k.shape[:2]
    pages, P = k_pages.shape[:2]
    kp, vp, st = k_pages.copy(), v_pages.copy(), np.zeros(N, np.int64)
    qo = None if q is None else np.full(q.shape, np.nan)
    for s in range(N):
        n = S if new_len is None else min(max(int(new_len[s]), 0), S)
        for i in range(n):
            j = max(int(length[s]), 0) + i
            pos = np.array((0 if pos0 is None else int(pos0[s])) + j, np.float64)
            if q is not None:
                qo[s, i] = turned(q[s, i], pos, freq, neighbours)
            page = int(table[s, j // P]) if j < table.shape[1] * P else -1
            if not 0 <= page < pages:
                st[s] = 4
                continue
            kp[page, j % P] = turned(k[s, i], pos, freq, neighbours)
            vp[page, j % P] = v[s, i]
    return kp, vp, qo, st

"""The library's 4-bit cache: its append, the attention over it, the weights its rows received, and eviction by them, as cases
that can be timed and checked.

The cache holds keys and values in blocks of 32 columns of a head: 4-bit floats (sign, two exponent bits, one mantissa bit:
0, 0.5, 1, 1.5, 2, 3, 4, 6) times one power of two, a byte e that stands for 2^(e - 127).  `append` puts new rows into
their pages, keys turned by their positions, and reads them back as the values they stand for; `attend` is the attention of a
request's K lists over shared rows and their own, both held so; `weigh` adds up the attention weight that every
cached row received; `evict` keeps the rows that received most, and reads what it kept.

  listed()              the cases that are always measured
  draw(rng)             one more case of the same ranges
  prepare(case, seed)   the inputs a program has in hand before the call, on the GPU
  run(state)            one pass: through the public binding where `own` is true, in plain torch otherwise
  work(case)            bytes and operations the pass cannot do without
  exact(case, seed)     the outputs in float64
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def listed():
    return [
        # one new token of each of 128 hypotheses (8 documents x 16), the text workload's heads: launches and latency
        dict(name="append_step", kind="append", N=128, S=1, H=8, Hkv=8, dh=64, rot=64, P=16, cap=80, pair="half",
             ragged=False, dtype="bf16"),
        # prompts of every length entering the cache at once: shared key heads, a partial rotation of neighbouring pairs
        dict(name="append_prompt", kind="append", N=24, S=1999, H=16, Hkv=4, dh=128, rot=96, P=24, cap=2200,
             pair="neighbour", ragged=True, dtype="bf16"),
        # one user's request answered online: the last element of five growing slates
        dict(name="attend_one_request", kind="attend", B=1, K=5, S=1, H=4, Hkv=4, dh=32, T=181, L=12, P=16, causal=True,
             ragged=True, dtype="bf16"),
        # the next token of 16 hypotheses for each of 8 documents
        dict(name="attend_text_step", kind="attend", B=8, K=16, S=1, H=8, Hkv=8, dh=64, T=1024, L=64, P=16, causal=True,
             ragged=True, dtype="bf16"),
        # the next token of 32 continuations of a very long document, grouped heads
        dict(name="attend_long_step", kind="attend", B=4, K=32, S=1, H=32, Hkv=8, dh=128, T=32768, L=512, P=64, causal=True,
             ragged=True, dtype="bf16"),
        # scoring the 50 slates of 64 recommendation requests at once, [CLS] and ten elements each
        dict(name="attend_lists", kind="attend", B=64, K=50, S=11, H=4, Hkv=4, dh=32, T=256, L=11, P=11, causal=False,
             ragged=False, dtype="bf16"),
        # the next part of a long text entering a cache that holds what came before it
        dict(name="attend_prompt", kind="attend", B=2, K=1, S=2048, H=16, Hkv=4, dh=128, T=4096, L=2048, P=64, causal=True,
             ragged=False, dtype="bf16"),
        # a few rows more of lists of every length, fp32 queries, odd sizes
        dict(name="attend_ragged_f32", kind="attend", B=3, K=19, S=7, H=6, Hkv=2, dh=64, T=777, L=23, P=5, causal=True,
             ragged=True, dtype="f32"),
        # what the rows of 8 documents and of their 16 hypotheses each received in one step
        dict(name="weigh_text_step", kind="weigh", B=8, K=16, S=1, H=8, Hkv=8, dh=64, T=1024, L=64, P=16, causal=True,
             ragged=True, dtype="bf16"),
        # ... and those of very long documents with 32 continuations
        dict(name="weigh_long_step", kind="weigh", B=4, K=32, S=1, H=32, Hkv=8, dh=128, T=32768, L=512, P=64, causal=True,
             ragged=True, dtype="bf16"),
        # the own rows of 128 hypotheses brought back to three quarters of their pages
        dict(name="evict_lists", kind="evict", N=128, Hkv=8, dh=64, T=64, P=16, to_P=16, keep=48, first=2, recent=16,
             ragged=True, dtype="bf16"),
        # long documents brought back to a quarter of their rows
        dict(name="evict_long", kind="evict", N=4, Hkv=8, dh=128, T=32768, P=64, to_P=64, keep=8192, first=4, recent=1024,
             ragged=False, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One case of the listed kinds; no drawn case costs more than the largest listed one of its kind."""
    kind = rng.choice(["append", "attend", "attend", "weigh", "evict"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    dh = rng.choice([32, 64, 64, 128])
    hkv = rng.choice([1, 2, 4, 8])
    h = hkv * rng.choice([1, 1, 2, 3, 4])
    most = max((c for c in listed() if c["kind"] == kind), key=_cost)
    for _ in range(1000):
        if kind == "append":
            n, s, p = _log(rng, 1, 256), _log(rng, 1, 2048), rng.choice([1, 5, 16, 16, 48, 64])
            case = dict(kind=kind, N=n, S=s, H=h, Hkv=hkv, dh=dh, rot=rng.choice([0, 16, dh, dh, dh]), P=p,
                        cap=s + _log(rng, 1, 400), pair=rng.choice(["half", "neighbour"]), ragged=rng.random() < 0.5,
                        dtype=dtype)
        elif kind == "evict":
            t = _log(rng, 2, 32768)
            keep = _log(rng, 1, t + 5)
            case = dict(kind=kind, N=_log(rng, 1, 256), Hkv=hkv, dh=dh, T=t, P=rng.choice([1, 5, 16, 16, 48, 64]),
                        to_P=rng.choice([1, 7, 16, 16, 64]), keep=keep, first=rng.choice([0, 1, 4]),
                        recent=rng.choice([0, 1, keep // 4, keep]), ragged=rng.random() < 0.5, dtype=dtype)
        else:
            step = rng.random() < 0.6
            s = rng.choice([1, 1, 2, 5]) if step else _log(rng, 2, 500)
            l = s + _log(rng, 1, 512) if step else s
            case = dict(kind=kind, B=_log(rng, 1, 64), K=_log(rng, 1, 64), S=s, H=h, Hkv=hkv, dh=dh,
                        T=_log(rng, 1, 32768 if step else 4096), L=l, P=rng.choice([1, 5, 16, 16, 48, 64]),
                        causal=step or rng.random() < 0.5, ragged=rng.random() < 0.6, dtype=dtype)
        if _cost(case) <= _cost(most) and (kind in ("append", "evict") or _heavy(case) <= _heavy(most)):
            return case
    return dict({k: v for k, v in most.items() if k != "name"}, dtype=dtype)


def _cost(case):
    w = work(case)
    return w["bytes"] / 5e12 + w["flops"] / 5e14


def _heavy(case):
    """Scores of the plain form (every capacity row counted): what its memory goes by."""
    return case["B"] * case["H"] * case["K"] * case["S"] * (case["T"] + case["L"])


def _spread(lo, hi, n):
    """n whole numbers spread evenly over lo .. hi: the lengths of a ragged batch, before they are shuffled."""
    return [lo + (hi - lo) * i // max(1, n - 1) for i in range(n)] if n > 1 else [hi]


def _lengths(case):
    """(ctx, q, own): shared rows of each request; query rows and own rows of the lists of a request."""
    B, K, S, T, L = (case[n] for n in ("B", "K", "S", "T", "L"))
    if not case["ragged"]:
        return [T] * B, [S] * K, [L] * K
    ctx = _spread((T + 1) // 2, T, B)
    if L > S:
        return ctx, [S] * K, _spread(S, L, K)
    q = _spread(1, S, K)
    return ctx, q, list(q)


# ---------------------------------------------------------------------------------------------
# The cache's layout
# ---------------------------------------------------------------------------------------------

def _head_bytes(P, dh):
    """Bytes of one head of a page: key codes, value codes, key scales, value scales, up to a multiple of 16."""
    return -(-P * (dh + dh // 16) // 16) * 16


def _views(pages, P, Hkv, dh):
    """(key codes, value codes, key scales, value scales) of pages [n][bytes]: [n][Hkv][P][dh / 2] or [..][dh / 32]."""
    x = pages.view(pages.shape[0], Hkv, -1)
    c, s = P * dh // 2, P * dh // 32
    return (x[..., :c].unflatten(-1, (P, dh // 2)), x[..., c:2 * c].unflatten(-1, (P, dh // 2)),
            x[..., 2 * c:2 * c + s].unflatten(-1, (P, dh // 32)), x[..., 2 * c + s:2 * c + 2 * s].unflatten(-1, (P, dh // 32)))


def _quantise(x):
    """Codes [..][dh / 2] and scales [..][dh / 32] of float64 rows x [..][dh]: the smallest power of two by which a block's
    largest magnitude is at most 6, the nearest 4-bit float, ties to the even code."""
    b = x.unflatten(-1, (-1, 32))
    top = b.abs().amax(-1)
    m, e = torch.frexp(top)                                  # top = m 2^e, 0.5 <= m < 1
    e = torch.where(top == 0, -125, e.long() - 2 - (m <= 0.75).long()).clamp(-125, 125)
    a = b.abs() * ((1023 - e) << 52).view(torch.float64).unsqueeze(-1)
    code = ((a > 0.25).byte() + (a >= 0.75).byte() + (a > 1.25).byte() + (a >= 1.75).byte() + (a > 2.5).byte() +
            (a >= 3.5).byte() + (a > 5).byte()) | (torch.signbit(b).byte() << 3)
    code = code.flatten(-2)
    return code[..., ::2] | (code[..., 1::2] << 4), (e + 127).byte()


def _values(codes, scales):
    """The fp32 values [..][dh] that codes [..][dh / 2] and scales [..][dh / 32] stand for."""
    lut = torch.tensor(E2M1 + [-v for v in E2M1], dtype=torch.float32, device=codes.device)
    x = lut[torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()]
    unit = (scales.int() << 23).view(torch.float32).unsqueeze(-1)
    return (x.unflatten(-1, (-1, 32)) * unit).flatten(-2)


def _fill(pages, table, rows, P, Hkv, dh, g, dtype):
    """Random keys and values, rounded to `dtype`, for the first `rows` rows of every sequence of table [N][cols]."""
    parts = _views(pages, P, Hkv, dh)
    gain = torch.exp(0.5 * torch.randn(dh, generator=g, device=DEV))     # some columns of the keys are larger than others
    gain = gain / gain.square().mean().sqrt()
    N = table.shape[0]
    per = max(1, (1 << 25) // (rows * Hkv * dh))
    j = torch.arange(rows, device=DEV)
    for s in range(0, N, per):
        t = table[s:s + per].long()
        page, row = t[:, j // P].flatten(), (j % P).repeat(t.shape[0])
        for codes, scales, by in ((parts[0], parts[2], gain), (parts[1], parts[3], None)):
            x = torch.randn(page.numel(), Hkv, dh, generator=g, device=DEV)
            x = (x if by is None else x * by).to(dtype).double()
            codes[page, :, row], scales[page, :, row] = _quantise(x)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    dt, dh, Hkv, P, kind = TYPES[case["dtype"]], case["dh"], case["Hkv"], case["P"], case["kind"]

    def rows(*shape):
        return torch.randn(*shape, generator=g, device=DEV).to(dt)

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device=DEV)

    def shuffled(values, times=None):
        v = ints(values)
        if times is None:
            return v[torch.randperm(len(values), generator=g, device=DEV)]
        order = torch.rand(times, len(values), generator=g, device=DEV).argsort(1)
        return v[order].contiguous()

    def pool(*counts, page_rows=P):
        """Pages for sequences x columns of each count, tables over them, and three pages that no table names."""
        n = sum(N * cols for N, cols in counts) + 3
        pages = torch.zeros(n, Hkv * _head_bytes(page_rows, dh), dtype=torch.uint8, device=DEV)
        order = torch.randperm(n, generator=g, device=DEV).int()
        tables, at = [], 0
        for N, cols in counts:
            tables.append(order[at:at + N * cols].view(N, cols).contiguous())
            at += N * cols
        return pages, tables

    st = dict(case=case)
    if kind == "append":
        N, S, H, rot = case["N"], case["S"], case["H"], case["rot"]
        st["pages"], (st["table"],) = pool((N, -(-case["cap"] // P)))
        # queries, keys and values as the column blocks of one fused projection
        qkv = rows(N, S, H + 2 * Hkv, dh)
        st.update(q=qkv[:, :, :H], k=qkv[:, :, H:H + Hkv], v=qkv[:, :, H + Hkv:],
                  new=shuffled(_spread(1, S, N)) if case["ragged"] else ints([S] * N),
                  len=torch.randint(0, case["cap"] - S + 1, (N,), generator=g, device=DEV).int(),
                  # the cached rows follow a context of some length: positions count on from there
                  pos0=torch.randint(0, 100000, (N,), generator=g, device=DEV).int(),
                  freq=10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / max(1, rot)),
                  q_out=torch.zeros(N, S, H, dh, dtype=dt, device=DEV),
                  k_out=torch.zeros(N, S, Hkv, dh, dtype=dt, device=DEV),
                  v_out=torch.zeros(N, S, Hkv, dh, dtype=dt, device=DEV),
                  len_out=torch.empty(N, dtype=torch.int32, device=DEV))
        if own:
            from paper_2603_02565_amd import PagedCache4
            st["cache"] = PagedCache4(st["pages"], st["table"], P, Hkv, dh, st["len"])
        return st
    if kind == "evict":
        N, T, keep, to_P = case["N"], case["T"], case["keep"], case["to_P"]
        cols = -(-keep // to_P)
        st["pages"], (st["table"],) = pool((N, -(-T // P)))
        st["to_pages"], (st["to_table"],) = pool((N, cols), page_rows=to_P)
        _fill(st["pages"], st["table"], T, P, Hkv, dh, g, dt)
        cap = st["table"].shape[1] * P
        w = torch.rand(N, Hkv, cap, generator=g, device=DEV)
        # a few rows receive most of the weight, many the same little, and some nothing
        w = torch.where(w < 0.1, torch.zeros((), device=DEV), torch.where(w < 0.4, (w * 20).floor() / 1024, w.pow(12)))
        st.update(weights=w, len=shuffled(_spread((T + 1) // 2, T, N)) if case["ragged"] else ints([T] * N),
                  to_len=torch.zeros(N, dtype=torch.int32, device=DEV),
                  weights_out=torch.zeros(N, Hkv, cols * to_P, device=DEV),
                  kept=torch.empty(N, Hkv, keep, dtype=torch.int32, device=DEV),
                  k_out=torch.zeros(N, keep, Hkv, dh, dtype=dt, device=DEV),
                  v_out=torch.zeros(N, keep, Hkv, dh, dtype=dt, device=DEV))
        if own:
            from paper_2603_02565_amd import PagedCache4
            st["cache"] = PagedCache4(st["pages"], st["table"], P, Hkv, dh, st["len"])
            st["to"] = PagedCache4(st["to_pages"], st["to_table"], to_P, Hkv, dh, st["to_len"])
        return st
    B, K, S, H, T, L = (case[n] for n in ("B", "K", "S", "H", "T", "L"))
    ctx, q, o = _lengths(case)
    st["pages"], (st["ctx_table"], st["own_table"]) = pool((B, -(-T // P)), (B * K, -(-L // P)))
    _fill(st["pages"], st["ctx_table"], T, P, Hkv, dh, g, dt)
    _fill(st["pages"], st["own_table"], L, P, Hkv, dh, g, dt)
    pair = torch.rand(B, K, generator=g, device=DEV).argsort(1)
    st.update(q=rows(B, K, S, H, dh), ctx_len=shuffled(ctx), own_len=ints(o)[pair].flatten().contiguous(),
              q_len=ints(q)[pair].contiguous() if case["ragged"] else None)
    if kind == "weigh":
        had = 8 * S * (H // Hkv) / (T + L)                  # about what a few such calls before gave a row of one list
        st.update(lse=_plain_attend(st)["lse"],
                  ctx_w=torch.rand(B, Hkv, st["ctx_table"].shape[1] * P, generator=g, device=DEV) * had * K,
                  own_w=torch.rand(B * K, Hkv, st["own_table"].shape[1] * P, generator=g, device=DEV) * had)
        st.update(ctx_w_out=torch.zeros_like(st["ctx_w"]), own_w_out=torch.zeros_like(st["own_w"]))
    if own:
        from paper_2603_02565_amd import PagedCache4, PrefixAttention4
        st["ctx"] = PagedCache4(st["pages"], st["ctx_table"], P, Hkv, dh, st["ctx_len"])
        st["own"] = PagedCache4(st["pages"], st["own_table"], P, Hkv, dh, st["own_len"])
        st["plan"] = PrefixAttention4(B=B, K=K, S=S, T=st["ctx_table"].shape[1] * P, L=st["own_table"].shape[1] * P,
                                      n_heads=H, n_kv_heads=Hkv, dh=dh, dtype=case["dtype"], causal=case["causal"])
    return st


# ---------------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------------

def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"append": _own_append, "attend": _own_attend, "weigh": _own_weigh, "evict": _own_evict}[kind](state)
    return {"append": _plain_append, "attend": _plain_attend, "weigh": _plain_weigh, "evict": _plain_evict}[kind](state)


def _own_append(st):
    cache, case = st["cache"], st["case"]
    cache.append(st["k"], st["v"], q=st["q"], q_out=st["q_out"], new_len=st["new"], pos0=st["pos0"],
                 freq=st["freq"] if case["rot"] else None, neighbours=case["pair"] == "neighbour", len_out=st["len_out"])
    cache.read(st["k_out"], st["v_out"], start=st["len"], count=st["new"])
    return dict(q=st["q_out"], k=st["k_out"], v=st["v_out"], len=st["len_out"])


def _own_attend(st):
    out = st["plan"].run(st["q"], st["ctx"], st["own"], q_len=st["q_len"])
    return dict(out=out, lse=st["plan"].lse)


def _own_weigh(st):
    st["plan"].weigh(st["q"], st["lse"], st["ctx"], st["own"], st["ctx_w"], st["own_w"], q_len=st["q_len"],
                     ctx_w_out=st["ctx_w_out"], own_w_out=st["own_w_out"])
    return dict(ctx_w=st["ctx_w_out"], own_w=st["own_w_out"])


def _own_evict(st):
    case = st["case"]
    st["cache"].evict(st["weights"], st["to"], keep=case["keep"], first=case["first"], recent=case["recent"],
                      weights_out=st["weights_out"], kept=st["kept"])
    st["to"].read(st["k_out"], st["v_out"])
    return dict(kept=st["kept"], weights=st["weights_out"], len=st["to_len"], k=st["k_out"], v=st["v_out"])


def _turn(x, angle, neighbours):
    """x [rows][heads][dh] in fp64 with the pairs of its first 2 * angle.shape[1] columns turned by angle [rows][pairs]."""
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    n = angle.shape[1]
    a, b = (x[..., 0:2 * n:2], x[..., 1:2 * n:2]) if neighbours else (x[..., :n], x[..., n:2 * n])
    u, w = a * c - b * s, b * c + a * s
    turned = torch.stack((u, w), -1).flatten(-2) if neighbours else torch.cat((u, w), -1)
    return torch.cat((turned, x[..., 2 * n:]), -1)


def _plain_append(st):
    case, P = st["case"], st["case"]["P"]
    kc, vc, ks, vs = _views(st["pages"], P, case["Hkv"], case["dh"])
    i = torch.arange(case["S"], device=DEV)
    n, i = (i[None] < st["new"][:, None]).nonzero(as_tuple=True)      # the new rows: sequence, row
    j = st["len"].long()[n] + i
    angle = (st["pos0"].long()[n] + j).double()[:, None] * st["freq"]
    page, row = st["table"].long()[n, j // P], j % P
    near, dt = case["pair"] == "neighbour", st["q_out"].dtype
    # turned and quantised in fp64: a key next to the border between two codes
    kc[page, :, row], ks[page, :, row] = _quantise(_turn(st["k"][n, i].double(), angle, near))
    vc[page, :, row], vs[page, :, row] = _quantise(st["v"][n, i].double())
    st["q_out"][n, i] = _turn(st["q"][n, i].double(), angle, near).to(dt)
    st["k_out"][n, i] = _values(kc[page, :, row], ks[page, :, row]).to(dt)
    st["v_out"][n, i] = _values(vc[page, :, row], vs[page, :, row]).to(dt)
    torch.add(st["len"], st["new"], out=st["len_out"])
    return dict(q=st["q_out"], k=st["k_out"], v=st["v_out"], len=st["len_out"])


def _score(st):
    """(q, w_ctx, w_own, row): queries [B][Hkv][K][S * G][dh], the scaled scores against shared and own rows, -infinity where a
    row does not see a key, and which rows are in use."""
    case = st["case"]
    B, K, S, H = st["q"].shape[:4]
    dh, Hkv, P = case["dh"], case["Hkv"], case["P"]
    G, scale = H // Hkv, 1 / math.sqrt(dh)
    q = st["q"].float().view(B, K, S, Hkv, G, dh).permute(0, 3, 1, 2, 4, 5).reshape(B, Hkv, K, S * G, dh)
    ck, ok = _gather(st, "ctx", 0), _gather(st, "own", 0)
    T, L = ck.shape[2], ok.shape[3]
    s, j = torch.arange(S, device=DEV), torch.arange(L, device=DEV)
    own_len = st["own_len"].long().view(B, K)
    q_len = torch.full((B, K), S, device=DEV) if st["q_len"] is None else st["q_len"].long()
    see_ctx = torch.arange(T, device=DEV) < st["ctx_len"][:, None, None, None, None]
    last = (own_len - q_len)[:, None, :, None] + s if case["causal"] else (own_len - 1)[:, None, :, None].expand(B, 1, K, S)
    see_own = (j < own_len[:, None, :, None, None]) & (j <= last[..., None])
    row = (s < q_len[:, None, :, None]).repeat_interleave(G, 3)[..., None]          # [B][1][K][S * G][1]
    see_own = see_own.repeat_interleave(G, 3)
    w_ctx = (q.reshape(B, Hkv, K * S * G, dh) @ ck.transpose(-1, -2)).view(B, Hkv, K, S * G, T) * scale
    w_own = q @ ok.transpose(-1, -2) * scale
    return q, w_ctx.masked_fill(~see_ctx, -math.inf), w_own.masked_fill(~see_own, -math.inf), row


def _gather(st, which, part):
    """The cache's keys (part 0) or values (1) in fp32, shared [B][Hkv][T][dh] or own [B][Hkv][K][L][dh]."""
    case = st["case"]
    parts = _views(st["pages"], case["P"], case["Hkv"], case["dh"])
    t = st[which + "_table"].long()
    x = _values(parts[part][t], parts[2 + part][t]).transpose(1, 2).flatten(2, 3)     # [sequences][Hkv][rows][dh]
    return x if which == "ctx" else x.unflatten(0, (case["B"], case["K"])).transpose(1, 2)


def _back(st, x):
    """[B][Hkv][K][S * G][n] -> [B][K][S][H][n]"""
    B, K, S, H = st["q"].shape[:4]
    Hkv = st["case"]["Hkv"]
    return x.view(B, Hkv, K, S, H // Hkv, -1).permute(0, 2, 3, 1, 4, 5).reshape(B, K, S, H, -1)


def _plain_attend(st):
    q, w_ctx, w_own, row = _score(st)
    top = torch.maximum(w_ctx.amax(-1, keepdim=True), w_own.amax(-1, keepdim=True))
    p_ctx, p_own = torch.exp(w_ctx - top), torch.exp(w_own - top)
    total = p_ctx.sum(-1, keepdim=True) + p_own.sum(-1, keepdim=True)
    cv, ov = _gather(st, "ctx", 1), _gather(st, "own", 1)
    out = (p_ctx.flatten(2, 3) @ cv).view_as(q) + p_own @ ov
    out = torch.where(row, out / total, torch.zeros((), device=DEV))
    lse = torch.where(row, top + torch.log(total), torch.full((), -math.inf, device=DEV))
    return dict(out=_back(st, out).to(st["q"].dtype), lse=_back(st, lse)[..., 0])


def _plain_weigh(st):
    B, K, S, H = st["q"].shape[:4]
    Hkv = st["case"]["Hkv"]
    _, w_ctx, w_own, row = _score(st)
    lse = st["lse"].view(B, K, S, Hkv, H // Hkv).permute(0, 3, 1, 2, 4).reshape(B, Hkv, K, -1, 1)
    p_ctx, p_own = (torch.where(row, torch.exp(w - lse), torch.zeros((), device=DEV)) for w in (w_ctx, w_own))
    ctx = p_ctx.flatten(2, 3).sum(2)                                                # [B][Hkv][T]
    one = p_own.sum(3).transpose(1, 2).flatten(0, 1)                                # [B * K][Hkv][L]
    for_ctx = torch.arange(ctx.shape[2], device=DEV) < st["ctx_len"][:, None, None]
    for_own = torch.arange(one.shape[2], device=DEV) < st["own_len"][:, None, None]
    return dict(ctx_w=torch.where(for_ctx, st["ctx_w"] + ctx, st["ctx_w_out"]),
                own_w=torch.where(for_own, st["own_w"] + one, st["own_w_out"]))


def _plain_evict(st):
    case = st["case"]
    P, Hkv, dh, keep, to_P = (case[n] for n in ("P", "Hkv", "dh", "keep", "to_P"))
    w, length = st["weights"], st["len"].long()[:, None, None]
    N, cap = w.shape[0], w.shape[2]
    i = torch.arange(cap, device=DEV)
    most = length.clamp(max=keep)                                                   # rows kept of each sequence
    first = most.clamp(max=case["first"])
    recent = (most - first).clamp(max=case["recent"])
    # protected rows, then the others from the greatest weight down (equal ones in their order), then what is no row
    rank = (~((i < first) | (i >= length - recent))).byte() + (i >= length).byte() * 2
    order = w.sort(dim=-1, descending=True, stable=True).indices
    order = order.gather(-1, rank.expand(N, Hkv, cap).gather(-1, order).sort(dim=-1, stable=True).indices)
    n = min(keep, cap)
    chosen = torch.where(torch.arange(n, device=DEV) < most, order[..., :n], cap).sort(-1).values      # [N][Hkv][n]
    live = chosen < cap
    st["kept"].fill_(-1)
    st["kept"][..., :n] = torch.where(live, chosen, -1).int()
    s, h, d = live.nonzero(as_tuple=True)
    j = chosen[s, h, d]
    page, to_page = st["table"].long()[s, j // P], st["to_table"].long()[s, d // to_P]
    st["weights_out"][s, h, d] = w[s, h, j]
    st["to_len"].copy_(most[:, 0, 0])
    parts, to = _views(st["pages"], P, Hkv, dh), _views(st["to_pages"], to_P, Hkv, dh)
    for x, y in zip(parts, to):
        y[to_page, h, d % to_P] = x[page, h, j % P]
    for name, c, e in (("k_out", to[0], to[2]), ("v_out", to[1], to[3])):
        st[name][s, d, h] = _values(c[to_page, h, d % to_P], e[to_page, h, d % to_P]).to(st[name].dtype)
    return dict(kept=st["kept"], weights=st["weights_out"], len=st["to_len"], k=st["k_out"], v=st["v_out"])


# ---------------------------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------------------------

def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    Hkv, dh, kind = case["Hkv"], case["dh"], case["kind"]
    row = Hkv * (dh // 2 + dh // 32)                        # bytes of a row's keys (or values) in the cache
    if kind == "append":
        H = case["H"]
        n = sum(_spread(1, case["S"], case["N"])) if case["ragged"] else case["N"] * case["S"]
        return {"bytes": 2 * n * (H + 2 * Hkv) * dh * e + 2 * n * row, "flops": 3 * n * (H + Hkv) * case["rot"]}
    if kind == "evict":
        lens = _spread((case["T"] + 1) // 2, case["T"], case["N"]) if case["ragged"] else [case["T"]] * case["N"]
        m = sum(min(n, case["keep"]) for n in lens)
        return {"bytes": sum(lens) * Hkv * 4 + m * (4 * row + Hkv * (8 + 2 * dh * e)), "flops": 0}
    H = case["H"]
    ctx, q, o = _lengths(case)
    B = case["B"]
    rows = B * sum(q)
    pairs = sum(ctx) * sum(q)
    for n, m in zip(q, o):
        pairs += B * (n * (m - n) + n * (n + 1) // 2 if case["causal"] else n * m)
    cached = sum(ctx) + B * sum(o)
    if kind == "weigh":
        return {"bytes": rows * H * (dh * e + 4) + cached * (row + 8 * Hkv), "flops": 2 * pairs * H * dh}
    return {"bytes": rows * H * (2 * dh * e + 4) + 2 * cached * row, "flops": 4 * pairs * H * dh}


# ---------------------------------------------------------------------------------------------
# The outputs in float64
# ---------------------------------------------------------------------------------------------

def exact(case, seed):
    if case["kind"] == "evict" and case["N"] * case["Hkv"] * case["T"] > 6e6:
        return None                                         # sorted on the host
    st = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "weigh": _exact_weigh, "evict": _exact_evict}[case["kind"]](st)


def _nearest(x):
    """The values that blocks of 32 of float64 rows x [..][dh] are held as, from the distances to all 4-bit floats."""
    b = x.unflatten(-1, (-1, 32))
    top = b.abs().amax(-1, keepdim=True).clamp(min=2.0 ** -140)
    e = torch.ceil(torch.log2(top / 6))
    e = e + (6 * torch.pow(2.0, e) < top).double()
    e = (e - (6 * torch.pow(2.0, e - 1) >= top).double()).clamp(-125, 125)
    unit = torch.pow(2.0, e)
    a = b.abs() / unit
    even = torch.tensor(E2M1[::2], dtype=torch.float64, device=x.device)     # codes 0, 2, 4, 6; the others lie between
    odd = torch.tensor(E2M1[1::2], dtype=torch.float64, device=x.device)
    de, ie = (a.unsqueeze(-1) - even).abs().min(-1)
    do, io = (a.unsqueeze(-1) - odd).abs().min(-1)
    v = torch.where(de <= do, even[ie], odd[io])
    return (torch.copysign(v, b) * unit).flatten(-2)


def _exact_append(st):
    """Each sequence's new rows as complex numbers times exp(i angle)."""
    case = st["case"]
    rot = case["rot"]
    q_out, k_out, v_out = (st[n].double() for n in ("q_out", "k_out", "v_out"))

    def turned(x, pos):
        x = x.double()
        r = x[..., :rot]
        if rot:
            z = r.unflatten(-1, (rot // 2, 2)) if case["pair"] == "neighbour" else r.unflatten(-1, (2, rot // 2)).transpose(-1, -2)
            z = torch.view_as_complex(z.contiguous()) * torch.exp(1j * pos[:, None, None] * st["freq"])
            z = torch.view_as_real(z)
            r = z.flatten(-2) if case["pair"] == "neighbour" else z.transpose(-1, -2).flatten(-2)
        return torch.cat((r, x[..., rot:]), -1)

    new, length, pos0 = st["new"].tolist(), st["len"].tolist(), st["pos0"].tolist()
    for s in range(case["N"]):
        pos = torch.arange(length[s], length[s] + new[s], device=DEV).double() + pos0[s]
        q_out[s, :new[s]] = turned(st["q"][s, :new[s]], pos)
        k_out[s, :new[s]] = _nearest(turned(st["k"][s, :new[s]], pos))
        v_out[s, :new[s]] = _nearest(st["v"][s, :new[s]].double())
    return dict(q=q_out, k=k_out, v=v_out, len=None)


def _decoded(st, which, s, n, part):
    """Keys (part 0) or values (1) [Hkv][n][dh] of the first n rows of a sequence in float64, by the formula of its bits."""
    case = st["case"]
    P, Hkv, dh = case["P"], case["Hkv"], case["dh"]
    head = st["pages"].view(st["pages"].shape[0], Hkv, -1)
    j = torch.arange(n, device=DEV)
    page, r = st[which][s].long()[j // P], (j % P)[:, None, None]
    h, c = torch.arange(Hkv, device=DEV)[None, :, None], torch.arange(dh, device=DEV)[None, None]
    page = page[:, None, None]
    byte = head[page, h, (part * P + r) * (dh // 2) + c // 2].long()
    scale = head[page, h, P * dh + (part * P + r) * (dh // 32) + c // 32].double()
    nib = torch.where(c % 2 == 0, byte & 15, byte >> 4)
    exponent, mantissa = (nib >> 1) & 3, nib & 1
    size = torch.where(exponent == 0, mantissa * 0.5, (1 + mantissa * 0.5) * torch.pow(2.0, exponent.double() - 1))
    return (torch.where(nib >= 8, -size, size) * torch.pow(2.0, scale - 127)).transpose(0, 1)


def _exact_lists(st, each):
    """each(b, k, n, t, m, s, value): scaled scores s [Hkv][G * n][t + m] of list k of request b, -infinity where hidden."""
    case = st["case"]
    B, K, S, H = st["q"].shape[:4]
    Hkv, dh = case["Hkv"], case["dh"]
    G = H // Hkv
    ctx_len, own_len = st["ctx_len"].tolist(), st["own_len"].tolist()
    q_len = [[S] * K] * B if st["q_len"] is None else st["q_len"].tolist()
    for b in range(B):
        t = ctx_len[b]
        shared = [_decoded(st, "ctx_table", b, t, part) for part in (0, 1)]
        for k in range(K):
            n, m = q_len[b][k], own_len[b * K + k]
            key, val = (torch.cat((shared[part], _decoded(st, "own_table", b * K + k, m, part)), 1) for part in (0, 1))
            q = st["q"][b, k, :n].double().unflatten(1, (Hkv, G)).permute(1, 2, 0, 3).flatten(1, 2)
            s = (q @ key.transpose(1, 2).contiguous()).unflatten(1, (G, n)) / dh ** 0.5
            if case["causal"]:
                late = torch.ones(n, m, dtype=torch.bool, device=DEV).triu(m - n + 1)
                s[..., t:].masked_fill_(late, -math.inf)
            each(b, k, n, t, m, s.flatten(1, 2), val)


def _exact_attend(st):
    """Every list by itself: softmax over its keys laid side by side."""
    Hkv = st["case"]["Hkv"]
    out = torch.zeros_like(st["q"], dtype=torch.float64)
    lse = torch.full(out.shape[:-1], -math.inf, dtype=torch.float64, device=DEV)

    def each(b, k, n, t, m, s, val):
        G = s.shape[1] // n
        out[b, k, :n] = (torch.softmax(s, -1) @ val).unflatten(1, (G, n)).permute(2, 0, 1, 3).flatten(1, 2)
        lse[b, k, :n] = torch.logsumexp(s, -1).view(Hkv, G, n).permute(2, 0, 1).flatten(1)

    _exact_lists(st, each)
    return dict(out=out, lse=lse)


def _exact_weigh(st):
    """Every list by itself: its weights added to the shared rows' and to its own."""
    K, Hkv = st["case"]["K"], st["case"]["Hkv"]
    ctx, one = st["ctx_w_out"].double(), st["own_w_out"].double()
    for x, w, lens in ((ctx, st["ctx_w"], st["ctx_len"]), (one, st["own_w"], st["own_len"])):
        for i, n in enumerate(lens.tolist()):
            x[i, :, :n] = w[i, :, :n].double()

    def each(b, k, n, t, m, s, val):
        lse = st["lse"][b, k, :n].double().unflatten(1, (Hkv, -1)).permute(1, 2, 0).flatten(1)
        p = torch.exp(s - lse[..., None]).sum(1)
        ctx[b, :, :t] += p[:, :t]
        one[b * K + k, :, :m] += p[:, t:]

    _exact_lists(st, each)
    return dict(ctx_w=ctx, own_w=one)


def _exact_evict(st):
    """One sequence and head at a time, by comparing (weight, index) pairs on the host."""
    case = st["case"]
    Hkv, keep = case["Hkv"], case["keep"]
    weights, k_out, v_out = (st[n].double() for n in ("weights_out", "k_out", "v_out"))
    for s, n in enumerate(st["len"].tolist()):
        m = min(keep, n)
        first = min(case["first"], m)
        recent = min(case["recent"], m - first)
        ws = st["weights"][s].double().cpu().tolist()
        keys, values = (_decoded(st, "table", s, n, part) for part in (0, 1))
        for h in range(Hkv):
            rest = sorted(range(first, n - recent), key=lambda i: (-ws[h][i], i))[:m - first - recent]
            rows = sorted(list(range(first)) + rest + list(range(n - recent, n)))
            at = torch.tensor(rows, device=DEV)
            weights[s, h, :m] = st["weights"][s, h, at].double()
            k_out[s, :m, h], v_out[s, :m, h] = keys[h, at], values[h, at]
    return dict(kept=None, weights=weights, len=None, k=k_out, v=v_out)

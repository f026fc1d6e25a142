"""The library's cache and shared-prefix attention calls, as cases that can be timed and checked.

A request's K lists (candidate slates, hypotheses that grow token by token) attend to one shared
context and, each, to their own rows.  `append` puts the keys and values of new rows into a paged cache, turned by
their positions; `attend` is the attention of every list over the shared rows and its own; `train`
is that attention with the gradients of the queries, keys and values.

  listed()              the cases that are always measured
  draw(rng)             one more case of the same ranges
  prepare(case, seed)   the inputs a program has in hand before the call, on the GPU
  run(state)            one pass: through the public binding where `own` is true, in plain torch otherwise
  work(case)            bytes and operations the pass cannot do without
  exact(case, seed)     the outputs in float64, list by list
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one new token of each of 128 hypotheses (8 documents x 16), the text workload's heads: launches and latency
        dict(name="append_step", kind="append", N=128, S=1, H=8, Hkv=8, dh=64, rot=64, P=16, cap=64, pair="half",
             ragged=False, dtype="bf16"),
        # the histories of a batch of long-context requests entering the cache at once
        dict(name="append_prompt", kind="append", N=16, S=2048, H=8, Hkv=8, dh=32, rot=32, P=64, cap=2304, pair="half",
             ragged=False, dtype="bf16"),
        # prompts of every length, shared key heads, a partial rotation of neighbouring pairs, odd pages, fp32
        dict(name="append_ragged_f32", kind="append", N=37, S=129, H=12, Hkv=4, dh=64, rot=48, P=7, cap=301,
             pair="neighbour", ragged=True, dtype="f32"),
        # one user's request answered online: the last element of five growing slates
        dict(name="attend_one_request", kind="attend", B=1, K=5, S=1, H=4, Hkv=4, dh=32, T=181, L=12, P=0, causal=True,
             ragged=True, dtype="bf16"),
        # the next token of 16 hypotheses for each of 8 documents, the own rows in a paged cache
        dict(name="attend_text_step", kind="attend", B=8, K=16, S=1, H=8, Hkv=8, dh=64, T=1024, L=64, P=16, causal=True,
             ragged=True, dtype="bf16"),
        # the next token of 32 continuations of a very long document, grouped heads
        dict(name="attend_long_step", kind="attend", B=4, K=32, S=1, H=32, Hkv=8, dh=128, T=32768, L=512, P=64, causal=True,
             ragged=True, dtype="bf16"),
        # scoring the 50 slates of 64 recommendation requests at once, [CLS] and ten elements each
        dict(name="attend_recsys", kind="attend", B=64, K=50, S=11, H=4, Hkv=4, dh=32, T=256, L=11, P=0, causal=False,
             ragged=False, dtype="bf16"),
        # scoring 16 whole hypotheses of 8 documents
        dict(name="attend_text", kind="attend", B=8, K=16, S=64, H=8, Hkv=8, dh=64, T=1024, L=64, P=0, causal=True,
             ragged=False, dtype="bf16"),
        # a few rows more of lists of every length, fp32, odd sizes
        dict(name="attend_ragged_f32", kind="attend", B=3, K=19, S=7, H=6, Hkv=2, dh=64, T=777, L=23, P=0, causal=True,
             ragged=True, dtype="f32"),
        # a training step's attention on a small batch of lists of every length, grouped heads
        dict(name="train_ragged", kind="train", B=2, K=9, S=37, H=8, Hkv=2, dh=128, T=333, L=37, P=0, causal=True,
             ragged=True, dtype="bf16"),
        # a training step's attention of the recommendation model on its full batch (the training step is fp32)
        dict(name="train_recsys_f32", kind="train", B=64, K=50, S=11, H=4, Hkv=4, dh=32, T=256, L=11, P=0, causal=False,
             ragged=False, dtype="f32"),
        # a training step's attention over whole hypotheses
        dict(name="train_text", kind="train", B=8, K=16, S=64, H=8, Hkv=8, dh=64, T=1024, L=64, P=0, causal=True,
             ragged=False, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One case of the listed kinds; no drawn case costs more than the largest listed one of its kind."""
    kind = rng.choice(["append", "attend", "attend", "train"])
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
        else:
            step = kind == "attend" and rng.random() < 0.5
            s = rng.choice([1, 1, 2, 5]) if step else _log(rng, 2, 100)
            l = s + _log(rng, 1, 512) if step else s
            p = rng.choice([0, 1, 16, 40]) if step else 0
            case = dict(kind=kind, B=_log(rng, 1, 64), K=_log(rng, 1, 64), S=s, H=h, Hkv=hkv, dh=dh,
                        T=_log(rng, 1, 16384 if step else 2048), L=l, P=p, causal=step or rng.random() < 0.5,
                        ragged=rng.random() < 0.6, dtype=dtype)
        if _cost(case) <= _cost(most) and (kind == "append" or _heavy(case) <= _heavy(most)):
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


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    dt, dh, H, Hkv = TYPES[case["dtype"]], case["dh"], case["H"], case["Hkv"]

    def rows(*shape):
        return torch.randn(*shape, generator=g, device=DEV, dtype=dt)

    def shuffled(values, times=None):
        v = torch.tensor(values, dtype=torch.int32, device=DEV)
        if times is None:
            return v[torch.randperm(len(values), generator=g, device=DEV)]
        order = torch.rand(times, len(values), generator=g, device=DEV).argsort(1)
        return v[order].contiguous()

    st = dict(case=case)
    if case["kind"] == "append":
        N, S, P, rot = case["N"], case["S"], case["P"], case["rot"]
        cols = -(-case["cap"] // P)
        pages = N * cols + 3
        # queries, keys and values as the column blocks of one fused projection
        qkv = rows(N, S, H + 2 * Hkv, dh)
        st.update(q=qkv[:, :, :H], k=qkv[:, :, H:H + Hkv], v=qkv[:, :, H + Hkv:],
                  k_pages=rows(pages, P, Hkv, dh), v_pages=rows(pages, P, Hkv, dh),
                  table=torch.randperm(pages, generator=g, device=DEV)[:N * cols].view(N, cols).int().contiguous(),
                  new=shuffled(_spread(1, S, N)) if case["ragged"] else torch.full((N,), S, dtype=torch.int32, device=DEV),
                  len=torch.randint(0, case["cap"] - S + 1, (N,), generator=g, device=DEV).int(),
                  # the cached rows follow a context of some length: positions count on from there
                  pos0=torch.randint(0, 100000, (N,), generator=g, device=DEV).int(),
                  freq=10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / max(1, rot)),
                  q_out=torch.zeros(N, S, H, dh, dtype=dt, device=DEV),
                  len_out=torch.empty(N, dtype=torch.int32, device=DEV))
        if own:
            from paper_2603_02565_amd import flasheval as fe
            st["cache"] = fe.PagedCache(st["k_pages"], st["v_pages"], st["table"], st["len"])
        return st
    B, K, S, T, L, P = (case[n] for n in ("B", "K", "S", "T", "L", "P"))
    ctx, q, o = _lengths(case)
    st.update(q=rows(B, K, S, H, dh), ctx_k=rows(B, T, Hkv, dh), ctx_v=rows(B, T, Hkv, dh), table=None, ctx_len=None,
              q_len=None, own_len=None)
    pages = 0
    if P:
        cols = -(-L // P)
        pages = B * K * cols + 3
        st.update(own_k=rows(pages, P, Hkv, dh), own_v=rows(pages, P, Hkv, dh),
                  table=torch.randperm(pages, generator=g, device=DEV)[:B * K * cols].view(B, K, cols).int().contiguous())
        L = cols * P
    else:
        st.update(own_k=rows(B, K, L, Hkv, dh), own_v=rows(B, K, L, Hkv, dh))
    if case["ragged"] or P:
        pair = shuffled(list(range(K)), B).long()
        st.update(ctx_len=shuffled(ctx), q_len=torch.tensor(q, dtype=torch.int32, device=DEV)[pair].contiguous(),
                  own_len=torch.tensor(o, dtype=torch.int32, device=DEV)[pair].contiguous())
    if case["kind"] == "train":
        st["dout"] = rows(B, K, S, H, dh)
    if own:
        from paper_2603_02565_amd import flasheval as fe
        st["plan"] = fe.PrefixAttention(B=B, K=K, S=S, T=T, L=L, n_heads=H, n_kv_heads=Hkv, dh=dh, dtype=case["dtype"],
                                        causal=case["causal"], page_rows=P, n_pages=pages, train=case["kind"] == "train")
    return st


# ---------------------------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------------------------

def run(state):
    kind = state["case"]["kind"]
    if own:
        return _own_append(state) if kind == "append" else _own_attend(state)
    return _plain_append(state) if kind == "append" else _plain_attend(state)


def _own_append(st):
    st["cache"].append(st["k"], st["v"], q=st["q"], q_out=st["q_out"], new_len=st["new"], pos0=st["pos0"],
                       freq=st["freq"] if st["case"]["rot"] else None, neighbours=st["case"]["pair"] == "neighbour",
                       len_out=st["len_out"])
    return dict(q=st["q_out"], k_pages=st["k_pages"], v_pages=st["v_pages"], len=st["len_out"])


def _own_attend(st):
    keys = (st["q"], st["ctx_k"], st["ctx_v"], st["own_k"], st["own_v"])
    more = dict(table=st["table"], ctx_len=st["ctx_len"], own_len=st["own_len"], q_len=st["q_len"])
    out = st["plan"].run(*keys, **more)
    if st["case"]["kind"] == "attend":
        return dict(out=out)
    dq, dck, dcv, dok, dov = st["plan"].grad(st["dout"], *keys, **more)
    return dict(out=out, dq=dq, dctx_k=dck, dctx_v=dcv, down_k=dok, down_v=dov)


def _turn(x, angle, neighbours):
    """x [rows][heads][dh] in fp32 with the pairs of its first 2 * angle.shape[1] columns turned by angle [rows][pairs]."""
    c, s = angle.cos().float()[:, None], angle.sin().float()[:, None]
    n = angle.shape[1]
    a, b = (x[..., 0:2 * n:2], x[..., 1:2 * n:2]) if neighbours else (x[..., :n], x[..., n:2 * n])
    u, w = a * c - b * s, b * c + a * s
    turned = torch.stack((u, w), -1).flatten(-2) if neighbours else torch.cat((u, w), -1)
    return torch.cat((turned, x[..., 2 * n:]), -1)


def _plain_append(st):
    case, P = st["case"], st["case"]["P"]
    i = torch.arange(case["S"], device=DEV)
    n, i = (i[None] < st["new"][:, None]).nonzero(as_tuple=True)      # the new rows: sequence, row
    j = st["len"].long()[n] + i
    angle = (st["pos0"].long()[n] + j).double()[:, None] * st["freq"]
    page, row = st["table"].long()[n, j // P], j % P
    near = case["pair"] == "neighbour"
    dt = st["k_pages"].dtype
    st["k_pages"][page, row] = _turn(st["k"][n, i].float(), angle, near).to(dt)
    st["v_pages"][page, row] = st["v"][n, i]
    st["q_out"][n, i] = _turn(st["q"][n, i].float(), angle, near).to(dt)
    torch.add(st["len"], st["new"], out=st["len_out"])
    return dict(q=st["q_out"], k_pages=st["k_pages"], v_pages=st["v_pages"], len=st["len_out"])


def _plain_attend(st):
    case = st["case"]
    B, K, S, H = st["q"].shape[:4]
    dh, Hkv, T, dt = case["dh"], case["Hkv"], case["T"], st["q"].dtype
    G, scale = H // Hkv, 1 / math.sqrt(dh)

    def heads(x):       # [B][K][S][H][dh] -> [B][Hkv][K][S * G][dh] in fp32
        return x.float().view(B, K, S, Hkv, G, dh).permute(0, 3, 1, 2, 4, 5).reshape(B, Hkv, K, S * G, dh)

    def back(x):
        return x.view(B, Hkv, K, S, G, dh).permute(0, 2, 3, 1, 4, 5).reshape(B, K, S, H, dh).to(dt)

    q = heads(st["q"])
    ck, cv = (st[n].float().permute(0, 2, 1, 3).contiguous() for n in ("ctx_k", "ctx_v"))
    if st["table"] is None:
        ok, ov = st["own_k"], st["own_v"]
    else:
        t = st["table"].long()
        ok, ov = st["own_k"][t].flatten(2, 3), st["own_v"][t].flatten(2, 3)
    ok, ov = (x.float().permute(0, 3, 1, 2, 4).contiguous() for x in (ok, ov))
    L = ok.shape[3]

    s = torch.arange(S, device=DEV)
    see_ctx = torch.ones(B, 1, 1, 1, T, dtype=torch.bool, device=DEV)
    see_own = torch.ones(B, 1, K, S, L, dtype=torch.bool, device=DEV)
    q_len = torch.full((B, K), S, device=DEV) if st["q_len"] is None else st["q_len"].long()
    own_len = torch.full((B, K), L, device=DEV) if st["own_len"] is None else st["own_len"].long()
    j = torch.arange(L, device=DEV)
    if st["ctx_len"] is not None:
        see_ctx = torch.arange(T, device=DEV) < st["ctx_len"][:, None, None, None, None]
    last = (own_len - q_len)[:, None, :, None] + s if case["causal"] else (own_len - 1)[:, None, :, None].expand(B, 1, K, S)
    see_own = see_own & (j < own_len[:, None, :, None, None]) & (j <= last[..., None])
    row = (s < q_len[:, None, :, None]).repeat_interleave(G, 3)[..., None]          # [B][1][K][S * G][1]
    see_own = see_own.repeat_interleave(G, 3)

    def shared(x):      # every list's rows of a head together, against the shared rows
        return x.reshape(B, Hkv, K * S * G, x.shape[-1])

    w_ctx = (shared(q) @ ck.transpose(-1, -2)).view(B, Hkv, K, S * G, T) * scale
    w_own = q @ ok.transpose(-1, -2) * scale
    w = torch.cat((w_ctx.masked_fill(~see_ctx, -math.inf), w_own.masked_fill(~see_own, -math.inf)), -1)
    p = torch.exp(w - w.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    p = torch.where(row, p, torch.zeros((), device=DEV))
    p_ctx, p_own = shared(p[..., :T]), p[..., T:]
    out = (p_ctx @ cv).view_as(q) + p_own @ ov
    if case["kind"] == "attend":
        return dict(out=back(out))

    do = torch.where(row, heads(st["dout"]), torch.zeros((), device=DEV))
    dp = torch.cat(((shared(do) @ cv.transpose(-1, -2)).view(B, Hkv, K, S * G, T), do @ ov.transpose(-1, -2)), -1)
    ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * scale
    ds_ctx, ds_own = shared(ds[..., :T]), ds[..., T:]
    dq = (ds_ctx @ ck).view_as(q) + ds_own @ ok
    dck, dcv = ds_ctx.transpose(-1, -2) @ shared(q), p_ctx.transpose(-1, -2) @ shared(do)
    dok, dov = ds_own.transpose(-1, -2) @ q, p_own.transpose(-1, -2) @ do
    dck, dcv = (x.permute(0, 2, 1, 3).contiguous().to(dt) for x in (dck, dcv))
    dok, dov = (x.permute(0, 2, 3, 1, 4).contiguous().to(dt) for x in (dok, dov))
    return dict(out=back(out), dq=back(dq), dctx_k=dck, dctx_v=dcv, down_k=dok, down_v=dov)


# ---------------------------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------------------------

def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    H, Hkv, dh = case["H"], case["Hkv"], case["dh"]
    if case["kind"] == "append":
        n = sum(_spread(1, case["S"], case["N"])) if case["ragged"] else case["N"] * case["S"]
        turned = n * (H + Hkv) * case["rot"]
        return {"bytes": 2 * n * (H + 2 * Hkv) * dh * e, "flops": 3 * turned}
    ctx, q, o = _lengths(case)
    B = case["B"]
    rows = B * sum(q)
    pairs = sum(ctx) * sum(q)
    for n, m in zip(q, o):
        pairs += B * (n * (m - n) + n * (n + 1) // 2 if case["causal"] else n * m)
    kv = 2 * (sum(ctx) + B * sum(o)) * Hkv * dh * e
    io = 2 * rows * H * dh * e
    if case["kind"] == "attend":
        return {"bytes": io + kv, "flops": 4 * pairs * H * dh}
    return {"bytes": 2 * (io + kv), "flops": 14 * pairs * H * dh}


# ---------------------------------------------------------------------------------------------
# The outputs in float64
# ---------------------------------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    return _exact_append(st) if case["kind"] == "append" else _exact_attend(st)


def _exact_append(st):
    """Each sequence's new rows as complex numbers times exp(i angle)."""
    case = st["case"]
    rot, P = case["rot"], case["P"]
    k_pages, v_pages, q_out = st["k_pages"].double(), st["v_pages"].double(), st["q_out"].double()

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
        j = torch.arange(length[s], length[s] + new[s], device=DEV)
        pos = (j + pos0[s]).double()
        page = st["table"][s].long()[torch.div(j, P, rounding_mode="floor")]
        k_pages[page, j % P] = turned(st["k"][s, :new[s]], pos)
        v_pages[page, j % P] = st["v"][s, :new[s]].double()
        q_out[s, :new[s]] = turned(st["q"][s, :new[s]], pos)
    return dict(q=q_out, k_pages=k_pages, v_pages=v_pages, len=None)


def _exact_attend(st):
    """Every list by itself: softmax over its keys laid side by side, gradients by differentiation."""
    case = st["case"]
    B, K, S, H = st["q"].shape[:4]
    G, train = H // case["Hkv"], case["kind"] == "train"
    lens = [None if st[n] is None else st[n].tolist() for n in ("ctx_len", "q_len", "own_len")]
    names = ("q", "ctx_k", "ctx_v") + (() if case["P"] else ("own_k", "own_v"))
    x = {n: st[n].double().requires_grad_(train) for n in names}
    out = torch.zeros_like(st["q"], dtype=torch.float64)
    for b in range(B):
        t = case["T"] if lens[0] is None else lens[0][b]
        for k in range(K):
            n = S if lens[1] is None else lens[1][b][k]
            m = case["L"] if lens[2] is None else lens[2][b][k]
            if case["P"]:
                pages = st["table"][b, k].long()
                ok, ov = (st[a][pages].flatten(0, 1)[:m].double() for a in ("own_k", "own_v"))
            else:
                ok, ov = x["own_k"][b, k, :m], x["own_v"][b, k, :m]
            key = torch.cat((x["ctx_k"][b, :t], ok)).permute(1, 2, 0)               # [Hkv][dh][t + m]
            val = torch.cat((x["ctx_v"][b, :t], ov)).permute(1, 0, 2)               # [Hkv][t + m][dh]
            q = x["q"][b, k, :n].unflatten(1, (case["Hkv"], G)).permute(1, 2, 0, 3).flatten(1, 2)
            s = (q @ key).unflatten(1, (G, n)) / case["dh"] ** 0.5
            if case["causal"]:
                late = torch.ones(n, m, dtype=torch.bool, device=DEV).triu(m - n + 1)
                s = torch.cat((s[..., :t], s[..., t:].masked_fill(late, -math.inf)), -1)
            o = (torch.softmax(s, -1).flatten(1, 2) @ val).unflatten(1, (G, n)).permute(2, 0, 1, 3).flatten(1, 2)
            out[b, k, :n] = o.detach()
            if train:
                o.backward(st["dout"][b, k, :n].double())
    if not train:
        return dict(out=out)
    return dict(out=out, dq=x["q"].grad, dctx_k=x["ctx_k"].grad, dctx_v=x["ctx_v"].grad, down_k=x["own_k"].grad,
                down_v=x["own_v"].grad)

"""The 4-bit cache on the GPU: append, read, attention, weights and eviction against tests/packed_reference.py and the
float64 attention of tests/prefix_reference.py within its bounds; bytes and kept rows have to be equal.  What lies
outside the lengths holds NaN blocks."""
import math

import numpy as np
import pytest
import torch

from paper_2603_02565_amd import PagedCache4, PrefixAttention, PrefixAttention4
from paper_2603_02565_amd import flasheval as fe
from tests import packed_reference as ref
from tests import prefix_reference as dense

pytestmark = pytest.mark.gpu

ACT = {"bf16": torch.bfloat16, "f32": torch.float32}
NAN, INF = float("nan"), float("inf")


def _say(*what):
    print(*what, flush=True)


def _i32(v):
    return None if v is None else torch.tensor(np.ascontiguousarray(v), dtype=torch.int32).cuda()


def _np(t):
    return t.double().cpu().numpy()


def _rounded(x, dtype):
    return torch.tensor(x).to(ACT[dtype]).double().numpy()


# ---------------------------------------------------------------------------------------------
# Append and read
# ---------------------------------------------------------------------------------------------

APPEND = [
    dict(dtype="bf16", N=1, S=1, H=1, Hkv=1, dh=32, rot=32, P=1, cols=1, near=False, full=True),
    dict(dtype="bf16", N=9, S=1, H=8, Hkv=8, dh=64, rot=64, P=16, cols=3, near=False),
    dict(dtype="f32", N=5, S=13, H=6, Hkv=2, dh=64, rot=48, P=7, cols=4, near=True),
    dict(dtype="bf16", N=3, S=70, H=4, Hkv=4, dh=128, rot=128, P=5, cols=20, near=False),
    dict(dtype="bf16", N=3, S=33, H=3, Hkv=1, dh=128, rot=96, P=64, cols=2, near=True),
    dict(dtype="f32", N=2, S=41, H=2, Hkv=2, dh=32, rot=16, P=3, cols=17, near=False),
    dict(dtype="bf16", N=4, S=6, H=2, Hkv=2, dh=64, rot=0, P=16, cols=2, near=False),
    dict(dtype="f32", N=2, S=130, H=0, Hkv=2, dh=64, rot=64, P=16, cols=9, near=False),
    dict(dtype="bf16", N=2, S=5, H=64, Hkv=32, dh=128, rot=128, P=4, cols=3, near=True),
]


def _append_case(dtype, N, S, H, Hkv, dh, rot, P, cols, near, full=False, seed=0, amp=1.0):
    r = np.random.default_rng(seed)
    cap = cols * P
    rnd = lambda *s: _rounded(r.standard_normal(s) * amp * np.exp2(r.integers(-3, 4, s[:-1] + (1,))), dtype)     # noqa: E731
    c = dict(q=rnd(N, S, H, dh) if H else None, k=rnd(N, S, Hkv, dh), v=rnd(N, S, Hkv, dh),
             new=np.full(N, S) if full else r.integers(0, S + 1, N), pos0=r.integers(0, 2 ** 20, N),
             freq=10000.0 ** (-np.arange(0, rot, 2) / max(1, rot)), n_pages=N * cols + 3)
    c["len"] = np.array([r.integers(0, cap - n + 1) for n in c["new"]])
    c["table"] = r.permutation(c["n_pages"])[:N * cols].reshape(N, cols)
    return c


def _append_want(c, dtype, N, Hkv, dh, rot, P, near, pages, q_out, **_):
    """Pages and q_out after the append, and q_out's bound."""
    cap = c["table"].shape[1] * P
    for s in range(N):
        for i in range(min(max(int(c["new"][s]), 0), c["k"].shape[1])):
            j = int(max(c["len"][s], 0)) + i
            pos = np.array(float(c["pos0"][s] + j))
            turn = lambda x: dense.turned(x, pos, c["freq"], near) if rot else x                         # noqa: E731
            if c["q"] is not None:
                q_out[s, i] = turn(c["q"][s, i])
            page = c["table"][s, j // P] if j < cap else -1
            if 0 <= page < pages.shape[0]:
                ref.write(pages, page, j % P, P, dh, turn(c["k"][s, i]), c["v"][s, i])
    return pages, q_out


def _append_run(c, dtype, Hkv, dh, rot, P, near, pages, q_out, **_):
    """Device pages [n][Hkv][head_bytes], q_out and the cache after the call."""
    up = lambda v: torch.tensor(v).to(ACT[dtype]).cuda()                                                  # noqa: E731
    dev = torch.tensor(pages.reshape(pages.shape[0], -1)).cuda()
    cache = PagedCache4(dev, _i32(c["table"]), P, Hkv, dh, _i32(c["len"]))
    q = None if c["q"] is None else up(c["q"])
    qo = None if q is None else up(q_out)
    cache.append(up(c["k"]), up(c["v"]), q=q, q_out=qo, new_len=_i32(c["new"]), pos0=_i32(c["pos0"]),
                 freq=torch.tensor(c["freq"]).cuda() if rot else None, neighbours=near)
    return dev.view(pages.shape[0], Hkv, -1), qo, cache


@pytest.mark.parametrize("kw", APPEND, ids=lambda k: f"{k['dtype']}-N{k['N']}-S{k['S']}-dh{k['dh']}-rot{k['rot']}-P{k['P']}")
def test_append_holds_the_nearest(kw):
    _say("append", kw)
    c = _append_case(**kw, seed=3)
    empty = np.full((c["n_pages"], kw["Hkv"], ref.head_bytes(kw["P"], kw["dh"])), 0xA5, np.uint8)
    q0 = np.full((kw["N"], kw["S"], kw["H"], kw["dh"]), 7.0)
    want, q_want = _append_want(c, pages=empty.copy(), q_out=q0.copy(), **kw)
    got, q_got, cache = _append_run(c, pages=empty, q_out=q0, **kw)
    assert np.array_equal(got.cpu().numpy(), want)                       # every other byte is left as it was
    assert (cache.status.cpu().numpy() == 0).all()
    assert np.array_equal(cache.len.cpu().numpy(), c["len"] + c["new"])
    if kw["H"]:
        # fp32 products of sines good to 2^-24, one rounding to the type
        bound = dense.turned_bound(c["q"], c["freq"], kw["near"], kw["dtype"])
        assert (np.abs(_np(q_got) - q_want) <= bound).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_of_every_kind_of_number(dtype):
    """Ties, borders, zeros, denormals, the largest numbers, infinities and NaN, as values and as keys that are not turned."""
    top = float(torch.finfo(ACT[dtype]).max)
    rows = [
        [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0] * 2 + [-0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, -6.0] * 2,
        [6.03125, 0.25, 0.75, -0.0, 0.0, 12.0, 3.0, -6.0] * 4,          # the largest is 12
        [0.0] * 16 + [-0.0] * 16,
        [top, -top, top / 2, 1.0] * 8,
        [2.0 ** -126, 2.0 ** -127, -2.0 ** -128, 0.0] * 8,
        [2.0 ** -120] + [2.0 ** -126, 3 * 2.0 ** -127] * 15 + [0.0],
        [1.0] * 31 + [INF], [-INF] + [2.0] * 31, [1.0] * 30 + [NAN, 5.0], [INF, NAN] * 16,
        [1.5 * 2.0 ** 20] + [1.0] * 31, [1.5078125 * 2.0 ** 20] + [1.0] * 31, [3 * 2.0 ** 125] * 32, [2.0 ** 127] * 32,
    ]
    x = _rounded(np.array(rows), dtype)
    c = dict(q=None, k=x[None, :, None, :], v=-x[None, :, None, :], new=np.array([len(rows)]), len=np.array([0]), pos0=np.array([0]),
             freq=np.zeros(0), table=np.array([[1, 0]]))
    empty = np.zeros((2, 1, ref.head_bytes(8, 32)), np.uint8)
    kw = dict(dtype=dtype, N=1, Hkv=1, dh=32, rot=0, P=8, near=False)
    want, _ = _append_want(c, pages=empty.copy(), q_out=None, **kw)
    got, _, _ = _append_run(c, pages=empty, q_out=None, **kw)
    assert np.array_equal(got.cpu().numpy(), want)
    # turned by nothing (position 0): the fp64 path gives the same bytes
    c["freq"] = np.zeros(16)
    with np.errstate(invalid="ignore"):
        want, _ = _append_want(c, pages=empty.copy(), q_out=None, **{**kw, "rot": 32})
    got, _, _ = _append_run(c, pages=empty, q_out=None, **{**kw, "rot": 32})
    assert np.array_equal(got.cpu().numpy(), want)


def test_append_next_to_a_border():
    """Turned keys that lie within 2^-40 of a border between two codes, on both sides."""
    borders = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    r = np.random.default_rng(0)
    N = 64
    k = np.zeros((N, 1, 1, 32))
    angle = r.uniform(0.1, 1.4, N)
    for s in range(N):
        # columns 0 .. 15 are a, 16 .. 31 b of a pair; u = a cos - b sin comes as near as fp32 inputs allow
        want = np.resize(borders, 16) * r.choice([-1, 1], 16)
        b = r.uniform(-1, 1, 16).astype(np.float32).astype(np.float64)
        a = ((want + b * np.sin(angle[s])) / np.cos(angle[s])).astype(np.float32).astype(np.float64)
        k[s, 0, 0] = np.concatenate((a, b))
    c = dict(q=None, k=k, v=np.zeros_like(k), new=np.ones(N, int), len=np.zeros(N, int), pos0=np.ones(N, int), freq=None,
             table=np.arange(N)[:, None])
    empty = np.zeros((N, 1, ref.head_bytes(1, 32)), np.uint8)
    kw = dict(dtype="f32", Hkv=1, dh=32, rot=32, P=1, near=False)
    for s in range(0, N, 8):                                             # one angle a call
        d = {n: (v[s:s + 1] if isinstance(v, np.ndarray) else v) for n, v in c.items()}
        d["freq"] = np.full(16, angle[s])
        want, _ = _append_want(d, N=1, pages=empty.copy(), q_out=None, **kw)
        got, _, _ = _append_run(d, pages=empty, q_out=None, **kw)
        assert np.array_equal(got.cpu().numpy(), want)


@pytest.mark.parametrize("S", [1, 300])
def test_append_rows_without_a_page(S):
    """Past the capacity, in pages outside the pool, lengths out of range."""
    kw = dict(dtype="bf16", N=6, S=S, H=2, Hkv=2, dh=64, rot=64, P=8, cols=3, near=False)
    c = _append_case(**{**kw, "cols": 40}, seed=5, full=True)
    c["table"] = c["table"][:, :3].copy()
    c["len"] = np.array([0, 23, 24, 5, -4, 1000])
    c["new"] = np.array([S, S, S, S + 9, 2, -3])
    c["table"][0, 0], c["table"][3, 0] = -1, c["n_pages"]
    empty = np.full((c["n_pages"], 2, ref.head_bytes(8, 64)), 0x5A, np.uint8)
    q0 = np.full((6, S, 2, 64), 7.0)
    want, q_want = _append_want(c, pages=empty.copy(), q_out=q0.copy(), **kw)
    got, q_got, cache = _append_run(c, pages=empty, q_out=q0, **kw)
    assert np.array_equal(got.cpu().numpy(), want)
    assert (np.abs(_np(q_got) - q_want) <= dense.turned_bound(c["q"], c["freq"], False, "bf16")).all()
    bad = [4, 4 if S > 1 else 0, 4, 4, 0, 0]
    assert cache.status.cpu().tolist() == bad
    assert cache.len.cpu().tolist() == [S, 23 + S, 24 + S, 5 + S, min(2, S), 1000]


def test_append_len_out_and_strides():
    """Column blocks of one projection as q, k and v, lengths into another tensor, a page stride."""
    r = np.random.default_rng(1)
    N, S, Hkv, H, dh, P = 3, 20, 2, 4, 64, 16
    qkv = torch.tensor(r.standard_normal((N, S, H + 2 * Hkv, dh))).bfloat16().cuda()
    width = PagedCache4.page_bytes(P, Hkv, dh)
    wide = torch.zeros(8, width + 64, dtype=torch.uint8, device="cuda")
    table, freq = _i32([[0, 5], [7, 2], [1, 4]]), torch.tensor(100.0 ** -(np.arange(32) / 32)).cuda()
    cache = PagedCache4(wide[:, :width], table, P, Hkv, dh)
    assert cache.cache.page_ld == width + 64
    len_out = torch.empty(3, dtype=torch.int32, device="cuda")
    q = cache.append(qkv[:, :, H:H + Hkv], qkv[:, :, H + Hkv:], q=qkv[:, :, :H], freq=freq, len_out=len_out)
    assert cache.len.tolist() == [0] * 3 and len_out.tolist() == [20] * 3
    flat = PagedCache4(torch.zeros(8, width, dtype=torch.uint8, device="cuda"), table, P, Hkv, dh)
    q2 = flat.append(qkv[:, :, H:H + Hkv].contiguous(), qkv[:, :, H + Hkv:].contiguous(), q=qkv[:, :, :H].contiguous(), freq=freq)
    assert torch.equal(wide[:, :width], flat.pages) and torch.equal(q, q2) and (wide[:, width:] == 0).all()
    assert flat.len.tolist() == [20] * 3


@pytest.mark.parametrize("dtype,dh,P", [("bf16", 32, 5), ("f32", 64, 16), ("bf16", 128, 1), ("f32", 128, 7)])
def test_read_gives_the_values_held(dtype, dh, P):
    r = np.random.default_rng(2)
    N, Hkv, cols, S = 5, 3, 4, 9
    hb = ref.head_bytes(P, dh)
    pages = r.integers(0, 256, (N * cols, Hkv, hb)).astype(np.uint8)
    for p in range(N * cols):
        for row in range(P):
            for part in (0, 1):
                s = ref.place(P, dh, part, row)[1]
                pages[p, :, s] = r.choice([2, 100, 127, 130, 200, 252, 255], (Hkv, dh // 32))
    table = r.permutation(N * cols).reshape(N, cols)
    table[3, 0] = -1
    length = np.array([0, 3, cols * P, cols * P + 5, 2])
    cache = PagedCache4(torch.tensor(pages.reshape(N * cols, -1)).cuda(), _i32(table), P, Hkv, dh, _i32(length))
    for start, count in ((None, None), (np.array([0, 1, 2, 0, cols * P - 1]), np.array([S, 0, 5, 2, S + 3])), (np.array([-4, 0, 1, 2, 3]), None)):
        k, v = (torch.full((N, S, Hkv, dh), 3.0, dtype=ACT[dtype], device="cuda") for _ in range(2))
        cache.read(k, v, start=_i32(start), count=_i32(count))
        want = np.full((2, N, S, Hkv, dh), 3.0)
        for s in range(N):
            st = 0 if start is None else max(int(start[s]), 0)
            n = min(max(int(length[s]), 0), cols * P) - st if count is None else int(count[s])
            for i in range(min(max(n, 0), S)):
                j = st + i
                page = table[s, j // P] if j < cols * P else -1
                want[:, s, i] = ref.read(pages, page, j % P, P, dh) if page >= 0 else 0.0
        for got, w in ((k, want[0]), (v, want[1])):
            assert np.array_equal(_np(got), w, equal_nan=True)
        one = torch.full((N, S, Hkv, dh), 3.0, dtype=ACT[dtype], device="cuda")
        cache.read(None, one, start=_i32(start), count=_i32(count))
        assert np.array_equal(_np(one), want[1], equal_nan=True)
    k, v = cache.read()
    assert k.shape == (N, cols * P, Hkv, dh) and (k[0] == 0).all() and v.dtype == torch.bfloat16


# ---------------------------------------------------------------------------------------------
# Attention and weights
# ---------------------------------------------------------------------------------------------

class Case:
    """A batch over two caches in one pool; rows outside the lengths, and pages of no sequence, are NaN blocks."""

    def __init__(self, dtype, B, K, S, H, Hkv, dh, T, L, P=16, causal=True, lens="ragged", seed=0, amp=1.0, scale=None, holes=0):
        r = np.random.default_rng(seed)
        self.dtype, self.P, self.causal, self.scale = dtype, P, causal, dh ** -0.5 if scale is None else scale
        self.B, self.K, self.S, self.H, self.Hkv, self.dh = B, K, S, H, Hkv, dh
        ccols, ocols = -(-T // P), -(-L // P)
        self.T, self.L = ccols * P, ocols * P
        rnd = lambda *s: ref.held_values(r.standard_normal(s) * amp) if np.prod(s) else np.zeros(s)       # noqa: E731
        self.q = _rounded(r.standard_normal((B, K, S, H, dh)) * amp, dtype)
        self.ck, self.cv, self.ok, self.ov = (rnd(B, self.T, Hkv, dh), rnd(B, self.T, Hkv, dh), rnd(B, K, self.L, Hkv, dh),
                                              rnd(B, K, self.L, Hkv, dh))
        if lens == "full":
            self.nc, self.nq, self.no = np.full(B, T), None, np.full((B, K), L)
        elif lens == "ragged":
            self.nq = r.integers(1, S + 1, (B, K))
            self.nc, self.no = r.integers(0, T + 1, B), np.minimum(self.nq + r.integers(0, L + 1, (B, K)), L)
        elif lens == "own":
            self.nq = r.integers(0, min(S, L) + 1, (B, K))
            self.nc, self.no = r.integers(0, T + 1, B), self.nq.copy()
        else:                                           # no context, no rows, no own keys, lengths out of range
            self.nq = r.choice([0, 1, S, S + 2, -1], (B, K))
            self.nc, self.no = r.choice([0, 0, 1, T, self.T + 5, -3], B), r.choice([0, 1, L, self.L + 9, -7], (B, K))
        self.n_pages = B * ccols + B * K * ocols + 3
        order = r.permutation(self.n_pages)
        self.ct = order[:B * ccols].reshape(B, ccols).copy()
        self.ot = order[B * ccols:B * ccols + B * K * ocols].reshape(B * K, ocols).copy()
        hb = ref.head_bytes(P, dh)
        self.pages = np.full((self.n_pages, Hkv, hb), 255, np.uint8)
        nc, nq, no = self.lengths()
        ok, ov = (x.reshape(B * K, -1, Hkv, dh) for x in (self.ok, self.ov)) if self.L else ([None] * (B * K),) * 2
        for t, n, k, v in ((self.ct, nc, self.ck, self.cv), (self.ot, no.reshape(-1), ok, ov)):
            for s in range(len(n)):
                if n[s]:
                    j = np.arange(n[s])
                    ref.write_rows(self.pages, t[s, j // P], j % P, P, dh, k[s][:n[s]], v[s][:n[s]])
        for b in range(B):
            for k in range(K):
                self.q[b, k, nq[b, k]:] = NAN
        # pages of no sequence, pages outside the pool
        for t in (self.ct, self.ot):
            for x in range(holes if t.size else 0):
                t[r.integers(t.shape[0]), r.integers(t.shape[1])] = r.choice([-1, self.n_pages, 2 ** 31 - 1, -2 ** 31])

    def lengths(self):
        return dense.clamp_lengths(self.B, self.K, self.S, self.T, self.L, self.nc, self.nq, self.no)

    def seen(self, t):
        """[sequences][capacity] rows whose page is in the pool."""
        return np.repeat((t >= 0) & (t < self.n_pages), self.P, 1)

    def device(self):
        self.dev = torch.tensor(self.pages.reshape(self.n_pages, -1)).cuda()
        mk = lambda t, n: PagedCache4(self.dev, _i32(t), self.P, self.Hkv, self.dh, _i32(np.asarray(n).reshape(-1)))   # noqa: E731
        self.ctx = mk(self.ct, self.nc) if self.T else None
        self.own = mk(self.ot, self.no) if self.L else None
        self.qd, self.q_len = torch.tensor(self.q).to(ACT[self.dtype]).cuda(), _i32(self.nq)
        return self

    def plan(self):
        return PrefixAttention4(B=self.B, K=self.K, S=self.S, T=self.T, L=self.L, n_heads=self.H, n_kv_heads=self.Hkv, dh=self.dh,
                                dtype=self.dtype, causal=self.causal, scale=self.scale)

    def run(self, plan=None, **kw):
        plan = plan or self.plan()
        out = plan.run(self.qd, self.ctx, self.own, q_len=self.q_len, **kw)
        return out, plan.lse

    def reference(self):
        """out and lse with bounds; shared rows of no page are taken out, request by request (their order says nothing)."""
        nc, nq, no = self.lengths()
        see, ck, cv, n = self.seen(self.ct), self.ck.copy(), self.cv.copy(), nc.copy()
        for b in range(self.B):
            rows = np.flatnonzero(see[b, :nc[b]])
            ck[b, :rows.size], cv[b, :rows.size], n[b] = ck[b, rows], cv[b, rows], rows.size
        want = dense.attend(self.q, ck, cv, self.ok, self.ov, dtype=self.dtype, causal=self.causal, scale=self.scale, ctx_len=n,
                            q_len=nq, own_len=no, seen=self.seen(self.ot).reshape(self.B, self.K, self.L) if self.L else None)
        # Held values are often 0, so a column's sum p|v| may be smaller than any fp32 number where its other keys have next to no
        # weight: what lies below 2^-126 may become 0, of a probability (at most 1) or of any of its three parts, 4 * 2^-126 |v|
        # a key, whatever the sum that the bound is relative to.
        top = max((float(np.abs(x).max()) for x in (cv, self.ov) if x.size), default=0.0)
        want["out"] = want["out"][0], want["out"][1] + 4 * (self.T + self.L) * 2.0 ** -126 * top
        return want


def _near(got, want, name):
    val, bound = want
    got = _np(got).reshape(val.shape)
    with np.errstate(invalid="ignore"):
        err = np.where((np.isneginf(val) & np.isneginf(got)) | np.isnan(bound), 0.0, np.abs(got - val))
        bad = ~((err <= bound) | np.isnan(bound))
    assert not bad.any(), (name, int(bad.sum()), float(np.nanmax(err)), float(bound[bad].max()), np.argwhere(bad)[:3].tolist())


FORWARD = [
    # the smallest: one row, one key; no key at all
    dict(dtype="bf16", B=1, K=1, S=1, H=1, Hkv=1, dh=32, T=1, L=0, P=1, lens="full"),
    dict(dtype="f32", B=1, K=1, S=1, H=1, Hkv=1, dh=32, T=0, L=1, P=1, lens="full"),
    dict(dtype="bf16", B=2, K=2, S=2, H=2, Hkv=1, dh=64, T=0, L=0, P=1, lens="full"),
    # single tokens: up to 32, up to 64 and more rows a key head
    dict(dtype="bf16", B=2, K=5, S=1, H=4, Hkv=4, dh=32, T=181, L=12),
    dict(dtype="bf16", B=2, K=16, S=1, H=8, Hkv=8, dh=64, T=200, L=64),
    dict(dtype="bf16", B=1, K=7, S=1, H=8, Hkv=2, dh=128, T=300, L=37, P=7),
    dict(dtype="bf16", B=1, K=60, S=1, H=2, Hkv=2, dh=64, T=100, L=33, P=5),
    dict(dtype="bf16", B=1, K=13, S=1, H=8, Hkv=2, dh=128, T=150, L=20, P=5),
    dict(dtype="bf16", B=1, K=45, S=1, H=2, Hkv=2, dh=32, T=150, L=20, P=48),
    dict(dtype="f32", B=2, K=3, S=1, H=6, Hkv=2, dh=64, T=65, L=33, P=1),
    dict(dtype="bf16", B=1, K=140, S=1, H=2, Hkv=1, dh=32, T=31, L=150, P=64),
    dict(dtype="bf16", B=1, K=140, S=1, H=1, Hkv=1, dh=128, T=700, L=9, P=64),
    # a few rows
    dict(dtype="bf16", B=2, K=4, S=5, H=4, Hkv=2, dh=64, T=130, L=40),
    dict(dtype="f32", B=3, K=6, S=7, H=6, Hkv=2, dh=64, T=77, L=23, P=5),
    dict(dtype="f32", B=1, K=3, S=3, H=2, Hkv=2, dh=128, T=129, L=65, P=5),
    dict(dtype="f32", B=1, K=9, S=5, H=3, Hkv=1, dh=128, T=200, L=30, P=48),
    # whole lists
    dict(dtype="bf16", B=3, K=9, S=11, H=4, Hkv=4, dh=32, T=100, L=11, P=11, causal=False, lens="full"),
    dict(dtype="bf16", B=2, K=3, S=64, H=2, Hkv=2, dh=64, T=96, L=64, lens="full"),
    dict(dtype="bf16", B=1, K=2, S=150, H=3, Hkv=1, dh=128, T=20, L=150, P=48, lens="own"),
    dict(dtype="f32", B=2, K=13, S=11, H=4, Hkv=4, dh=32, T=64, L=11, P=5, causal=False, lens="own"),
    dict(dtype="bf16", B=1, K=1, S=260, H=2, Hkv=1, dh=64, T=0, L=300, P=64, lens="ragged"),
    dict(dtype="bf16", B=1, K=1, S=50, H=1, Hkv=1, dh=128, T=70, L=80, P=16, lens="ragged"),
    # many requests of few rows: four waves a workgroup
    dict(dtype="bf16", B=64, K=2, S=1, H=8, Hkv=8, dh=32, T=40, L=9, P=4),
    dict(dtype="bf16", B=70, K=3, S=1, H=8, Hkv=8, dh=64, T=33, L=9, P=7),
    dict(dtype="bf16", B=64, K=1, S=2, H=8, Hkv=8, dh=128, T=37, L=9, P=4),
    dict(dtype="f32", B=64, K=2, S=1, H=8, Hkv=8, dh=64, T=40, L=9, P=4),
    dict(dtype="f32", B=66, K=2, S=1, H=8, Hkv=8, dh=32, T=40, L=9, P=4),
    # ranges of keys in proportion to the requests' lengths
    dict(dtype="bf16", B=8, K=34, S=1, H=4, Hkv=4, dh=32, T=16384, L=3, P=64),
    # lengths at and past their limits, rows without keys
    dict(dtype="bf16", B=6, K=5, S=3, H=4, Hkv=2, dh=32, T=40, L=9, P=4, lens="edge"),
    dict(dtype="bf16", B=6, K=5, S=9, H=4, Hkv=2, dh=64, T=140, L=70, P=10, lens="edge", causal=False),
    dict(dtype="bf16", B=6, K=3, S=9, H=4, Hkv=2, dh=128, T=140, L=70, P=10, lens="edge"),
    dict(dtype="f32", B=6, K=7, S=4, H=2, Hkv=1, dh=32, T=33, L=20, P=3, lens="edge"),
    # pages outside the pool
    dict(dtype="bf16", B=3, K=4, S=2, H=4, Hkv=2, dh=64, T=160, L=30, P=5, holes=12),
    dict(dtype="bf16", B=2, K=20, S=2, H=4, Hkv=2, dh=32, T=400, L=30, P=16, holes=12),
    dict(dtype="f32", B=2, K=50, S=1, H=4, Hkv=2, dh=128, T=160, L=30, P=8, holes=20),
    # sharp softmaxes: scores up to some hundreds
    dict(dtype="bf16", B=1, K=4, S=6, H=2, Hkv=2, dh=64, T=150, L=20, amp=6.0),
    dict(dtype="f32", B=1, K=4, S=6, H=2, Hkv=2, dh=64, T=150, L=20, amp=6.0, scale=0.3),
    dict(dtype="f32", B=1, K=4, S=6, H=2, Hkv=2, dh=32, T=50, L=20, scale=-0.4),
    dict(dtype="bf16", B=1, K=4, S=6, H=2, Hkv=2, dh=32, T=50, L=20, scale=0.0),
    # long: ranges of keys that are joined, fp32 sums
    dict(dtype="bf16", B=1, K=3, S=1, H=4, Hkv=1, dh=64, T=3000, L=100, P=64),
    dict(dtype="bf16", B=1, K=50, S=1, H=4, Hkv=1, dh=32, T=3000, L=100, P=64),
    dict(dtype="f32", B=1, K=2, S=2, H=2, Hkv=1, dh=64, T=4500, L=10, P=48),
]
IDS = lambda k: "-".join(f"{n}{v}" for n, v in k.items())                                                 # noqa: E731


@pytest.mark.parametrize("kw", FORWARD, ids=IDS)
def test_attention(kw):
    _say("attention", kw)
    c = Case(**kw, seed=1).device()
    want = c.reference()
    out, lse = c.run()
    _near(out, want["out"], "out")
    _near(lse, want["lse"], "lse")
    again, lse2 = c.run()
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("kw", FORWARD, ids=IDS)
def test_weights(kw):
    _say("weights", kw)
    c = Case(**kw, seed=2).device()
    r = np.random.default_rng(3)
    lse = c.reference()["lse"][0].astype(np.float32)
    nc, nq, no = c.lengths()
    for b in range(c.B):
        for k in range(c.K):
            lse[b, k, nq[b, k]:] = NAN                                    # not read into anything
    cw, ow = (r.random(s).astype(np.float32) for s in ((c.B, c.Hkv, c.T), (c.B, c.K, c.Hkv, c.L)))
    want = ref.weigh(c.q, c.ck, c.ok, lse, causal=c.causal, scale=c.scale, ctx_len=nc, q_len=nq, own_len=no, ctx_w=cw, own_w=ow,
                     ctx_seen=c.seen(c.ct).tolist(), own_seen=c.seen(c.ot).reshape(c.B, c.K, c.L).tolist())
    plan, lse = c.plan(), torch.tensor(lse).cuda()
    d = lambda x: torch.tensor(x).cuda() if x.size else None                                              # noqa: E731
    cd, od = d(cw), d(ow)
    co, oo = (None if t is None else torch.full_like(t, 9.0) for t in (cd, od))
    plan.weigh(c.qd, lse, c.ctx, c.own, cd, od, q_len=c.q_len, ctx_w_out=co, own_w_out=oo)
    for got, name, lens in ((co, "ctx_w", nc), (oo, "own_w", no.reshape(-1))):
        if got is None:
            continue
        _near(got, want[name], name)
        for s, n in enumerate(lens):
            assert (got.flatten(0, -3)[s, :, n:] == 9.0).all()            # entries past the length
    # in place, and one of the two alone
    if cd is not None:
        x = cd.clone()
        plan.weigh(c.qd, lse, c.ctx, c.own, ctx_w=x, q_len=c.q_len)
        for b in range(c.B):
            assert torch.equal(x[b, :, :nc[b]], co[b, :, :nc[b]]) and torch.equal(x[b, :, nc[b]:], cd[b, :, nc[b]:])
    if od is not None:
        x = od.clone()
        plan.weigh(c.qd, lse, c.ctx, c.own, own_w=x, q_len=c.q_len)
        for s, n in enumerate(no.reshape(-1)):
            y, z = (t.view(-1, c.Hkv, c.L)[s] for t in (x, oo))
            assert torch.equal(y[:, :n], z[:, :n])


@pytest.mark.parametrize("rows,dh", [(dict(K=60, S=30, H=4, Hkv=1), 32), (dict(K=2, S=700, H=2, Hkv=1), 64)])
def test_weights_of_many_rows(rows, dh):
    """Few keys and many rows: the rows are cut into ranges whose sums are added."""
    c = Case("bf16", B=1, dh=dh, T=70, L=rows["S"], P=16, lens="full", seed=4, **rows).device()
    plan = c.plan()
    assert fe.fe_packed_workspace_size(_sizes(c), True) > 0
    out, lse = c.run(plan)
    cw, ow = torch.zeros(1, 1, c.T).cuda(), torch.zeros(rows["K"], 1, c.L).cuda()
    plan.weigh(c.qd, lse, c.ctx, c.own, cw, ow)
    n = rows["K"] * rows["S"] * rows["H"]
    # the weights of a row add up to one: rows in all; each is off by its exponent's roundings and lse's (dh 2^-24 times
    # sum |q||k| scale each, at most 20 here), and by the sums' of n terms
    assert abs(float(cw.double().sum() + ow.double().sum()) - n) <= n * 2.0 ** -24 * (dh * 40 + n)
    nc, nq, no = c.lengths()
    want = ref.weigh(c.q[:, :, ::97], c.ck, c.ok, lse.cpu().numpy()[:, :, ::97], causal=False, scale=c.scale, ctx_len=nc,
                     q_len=np.full_like(nq, len(range(0, rows["S"], 97))), own_len=no * 0, ctx_w=np.zeros((1, 1, c.T)),
                     own_w=np.zeros((1, c.K, 1, c.L)))["ctx_w"]
    q = c.qd[:, :, ::97].contiguous()
    few = PrefixAttention4(B=1, K=c.K, S=q.shape[2], T=c.T, L=0, n_heads=c.H, n_kv_heads=1, dh=dh, dtype="bf16")
    x = torch.zeros(1, 1, c.T).cuda()
    few.weigh(q, lse[:, :, ::97].contiguous(), c.ctx, None, x)
    _near(x, want, "ctx_w")


def _sizes(c):
    a = fe.fe_packed_args()
    a.dtype = fe.FE_BF16 if c.dtype == "bf16" else fe.FE_F32
    a.B, a.K, a.S, a.n_heads, a.n_kv_heads, a.dh = c.B, c.K, c.S, c.H, c.Hkv, c.dh
    a.ctx = fe.fe_packed_cache(None, 0, None, None, c.B if c.T else 0, 1, c.T, 1)
    a.own = fe.fe_packed_cache(None, 0, None, None, c.B * c.K if c.L else 0, 1, c.L, 1)
    a.ctx_w = a.own_w = 1
    return a


@pytest.mark.parametrize("K,S,dh,dtype", [(5, 3, 64, "bf16"), (40, 3, 32, "bf16"), (70, 3, 128, "bf16"), (15, 3, 64, "bf16"), (15, 3, 128, "f32"),
                                          (3, 45, 32, "bf16"), (3, 70, 64, "f32"), (2, 90, 128, "bf16")])
def test_own_rows_of_nan_stay_in_their_list(K, S, dh, dtype):
    """Blocks of NaN among one list's own keys and values: the other lists keep their bits; in that list the rows that see the
    key are NaN, in all columns for a key's block and in the block's for a value's."""
    L = S + 6
    kw = dict(dtype=dtype, B=2, K=K, S=S, H=2, Hkv=2, dh=dh, T=40, L=L, P=4, lens="full", seed=6)
    clean = Case(**kw).device()
    want, lse0 = clean.run()
    for part, row in ((1, L - 2), (0, L - 2), (1, 2), (0, L // 2)):
        c = Case(**kw)
        page = c.ot[K + 1, row // 4]                                      # list 1 of request 1
        s = ref.place(4, dh, part, row % 4)[1]
        c.pages[page, 1, s.start] = 255                                   # key head 1, the first block
        got, lse = c.device().run()
        same = torch.ones_like(want, dtype=torch.bool)
        sees = [i for i in range(S) if row <= L - S + i]
        cols = slice(0, 32) if part else slice(0, dh)
        same[1, 1, sees, 1, cols] = False
        assert torch.equal(got[same], want[same])
        assert torch.isnan(got[1, 1, sees, 1, cols]).all()
        assert torch.isnan(lse[1, 1, sees, 1]).all() if part == 0 else torch.equal(lse, lse0)


def test_shared_nan_reaches_every_row_of_its_request():
    c = Case("bf16", B=2, K=3, S=2, H=2, Hkv=2, dh=64, T=40, L=9, P=4, lens="full", seed=6)
    page = c.ct[1, 3]
    c.pages[page, 0, ref.place(4, 64, 1, 2)[1].start + 1] = 255           # the second block of a value
    got, _ = c.device().run()
    assert torch.isnan(got[1, :, :, 0, 32:]).all() and torch.isfinite(got[1, :, :, 0, :32]).all()
    assert torch.isfinite(got[0]).all() and torch.isfinite(got[1, :, :, 1]).all()


def test_a_list_does_not_depend_on_the_others():
    c = Case("bf16", B=1, K=9, S=4, H=4, Hkv=2, dh=64, T=50, L=12, P=4, lens="full", seed=8).device()
    out, _ = c.run()
    d = Case("bf16", B=1, K=9, S=4, H=4, Hkv=2, dh=64, T=50, L=12, P=4, lens="full", seed=8)
    for k in range(9):
        if k != 4:
            for p in d.ot[k]:
                d.pages[p] = 255
    got, _ = d.device().run()
    assert torch.equal(got[0, 4], out[0, 4])


def test_strided_queries_and_another_stream():
    c = Case("bf16", B=2, K=3, S=4, H=4, Hkv=2, dh=64, T=50, L=12, seed=9).device()
    want, lse = c.run()
    wide = torch.full((2, 3, 4, 12, 64), NAN, dtype=torch.bfloat16, device="cuda")
    wide[..., 4:8, :] = c.qd
    plan = c.plan()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = plan.run(wide[..., 4:8, :], c.ctx, c.own, q_len=c.q_len, stream=side)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(plan.lse, lse)


def test_shared_pages_and_two_pools():
    """Requests whose tables name the same pages, and own rows in another pool with pages of another size."""
    g = torch.Generator(device="cuda").manual_seed(2)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()                               # noqa: E731
    B, K, Hkv, H, dh = 3, 4, 2, 4, 64
    pool = torch.full((9, PagedCache4.page_bytes(16, Hkv, dh)), 255, dtype=torch.uint8, device="cuda")
    other = torch.full((B * K * 3, PagedCache4.page_bytes(5, Hkv, dh)), 255, dtype=torch.uint8, device="cuda")
    one = PagedCache4(pool, _i32([[2, 7, 4]]), 16, Hkv, dh)
    one.append(rnd(1, 40, Hkv, dh), rnd(1, 40, Hkv, dh))
    ctx = PagedCache4(pool, _i32([[2, 7, 4]] * B), 16, Hkv, dh, _i32([40, 17, 33]))
    own = PagedCache4(other, torch.randperm(B * K * 3, generator=g, device="cuda").int().view(B * K, 3), 5, Hkv, dh)
    own.append(rnd(B * K, 13, Hkv, dh), rnd(B * K, 13, Hkv, dh))
    q = rnd(B, K, 2, H, dh)
    plan = PrefixAttention4(B=B, K=K, S=2, T=48, L=15, n_heads=H, n_kv_heads=Hkv, dh=dh, dtype="bf16", causal=True)
    out = plan.run(q, ctx, own)
    (ck, cv), (ok, ov) = ((_np(x) for x in c.read()) for c in (ctx, own))
    want = dense.attend(_np(q), ck, cv, ok.reshape(B, K, 15, Hkv, dh), ov.reshape(B, K, 15, Hkv, dh), dtype="bf16", causal=True,
                        ctx_len=np.array([40, 17, 33]), own_len=np.full((B, K), 13))
    _near(out, want["out"], "out")
    w = torch.zeros(B, Hkv, 48, device="cuda")
    plan.weigh(q, plan.lse, ctx, own, ctx_w=w)
    to = PagedCache4(pool, _i32([[0], [1], [3]]), 16, Hkv, dh)            # each request keeps rows of the shared pages for itself
    kept = ctx.evict(w, to, keep=9, recent=3)
    k, v = to.read()
    for b, n in enumerate((40, 17, 33)):
        for h in range(Hkv):
            rows = ref.evict_rows(w[b, h].tolist(), n, 9, 0, 3)
            assert kept[b, h].tolist() == rows
            assert np.array_equal(_np(k)[b, :9, h], ck[b, rows, h]) and np.array_equal(_np(v)[b, :9, h], cv[b, rows, h])


def test_replayed_step():
    """Append, attention, weights and eviction captured once, replayed with eager work between; every replay against eager."""
    torch.manual_seed(0)
    B, K, H, Hkv, dh, P, T, L = 2, 5, 4, 2, 64, 16, 96, 48
    g = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()                               # noqa: E731
    pages = torch.zeros(200, PagedCache4.page_bytes(P, Hkv, dh), dtype=torch.uint8, device="cuda")
    ids = torch.arange(200, device="cuda").int()
    ctx = PagedCache4(pages, ids[:12].view(B, 6).contiguous(), P, Hkv, dh)
    own = PagedCache4(pages, ids[12:42].view(B * K, 3).contiguous(), P, Hkv, dh)
    to = PagedCache4(pages, ids[42:52].view(B * K, 1).contiguous(), P, Hkv, dh)
    ctx.append(rnd(B, 90, Hkv, dh), rnd(B, 90, Hkv, dh))
    freq = torch.tensor(100.0 ** -(np.arange(32) / 32)).cuda()
    plan = PrefixAttention4(B=B, K=K, S=1, T=T, L=L, n_heads=H, n_kv_heads=Hkv, dh=dh, dtype="bf16", causal=True)
    q, k, v = rnd(B * K, 1, H, dh), rnd(B * K, 1, Hkv, dh), rnd(B * K, 1, Hkv, dh)
    own.append(rnd(B * K, 20, Hkv, dh), rnd(B * K, 20, Hkv, dh))
    q_out, lens = torch.empty_like(q), own.len.clone()
    cw, ow, two = torch.zeros(B, Hkv, T).cuda(), torch.zeros(B * K, Hkv, L).cuda(), torch.zeros(B * K, Hkv, 16).cuda()
    kept = torch.empty(B * K, Hkv, 12, dtype=torch.int32, device="cuda")

    def step():
        own.append(k, v, q=q, q_out=q_out, freq=freq)
        out = plan.run(q_out.view(B, K, 1, H, dh), ctx, own)
        plan.weigh(q_out.view(B, K, 1, H, dh), plan.lse, ctx, own, cw, ow)
        own.evict(ow, to, keep=12, first=1, recent=4, weights_out=two, kept=kept)
        return out

    def state():
        return [t.clone() for t in (plan.out, plan.lse, cw, ow, two, kept, own.len, to.len, pages)]

    def reset():
        own.len.copy_(lens)
        cw.zero_()
        ow.zero_()

    step()
    reset()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(3):
        for t in (q, k, v):
            t.copy_(rnd(*t.shape))
        reset()
        for _ in range(2):
            step()
        want = state()
        reset()
        torch.cuda.synchronize()
        for _ in range(2):
            graph.replay()
        got = state()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_far_offsets():
    """Pages more than 2^31 bytes into the pool."""
    P, Hkv, dh = 16, 2, 64
    width = PagedCache4.page_bytes(P, Hkv, dh)
    pool = torch.empty(3 * (1 << 30) + width, dtype=torch.uint8, device="cuda")
    pages = pool.as_strided((4, width), (1 << 30, 1))
    for t in range(4):
        pages[t].fill_(255)
    near = torch.zeros(4, width, dtype=torch.uint8, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v, q = (torch.randn(1, n, h, dh, generator=g, device="cuda").bfloat16() for n, h in ((30, Hkv), (30, Hkv), (1, 4)))
    got = []
    for p in (pages, near):
        ctx, to = PagedCache4(p, _i32([[3, 1]]), P, Hkv, dh), PagedCache4(p, _i32([[2]]), P, Hkv, dh)
        ctx.append(k, v)
        plan = PrefixAttention4(B=1, K=1, S=1, T=32, L=0, n_heads=4, n_kv_heads=Hkv, dh=dh, dtype="bf16")
        out = plan.run(q.view(1, 1, 1, 4, dh), ctx, None)
        w = torch.zeros(1, Hkv, 32, device="cuda")
        plan.weigh(q.view(1, 1, 1, 4, dh), plan.lse, ctx, None, w)
        kept = ctx.evict(w, to, keep=10)
        got.append([out, w, kept, *to.read(), *ctx.read()])
    for a, b in zip(*got):
        assert torch.equal(a, b)
    assert torch.isfinite(got[0][0]).all()


# ---------------------------------------------------------------------------------------------
# Eviction
# ---------------------------------------------------------------------------------------------

EVICT = [
    dict(N=1, Hkv=1, dh=32, T=1, P=1, to_P=1, keep=1, first=0, recent=0),
    dict(N=4, Hkv=2, dh=64, T=64, P=16, to_P=16, keep=48, first=2, recent=16),
    dict(N=3, Hkv=2, dh=128, T=203, P=7, to_P=5, keep=50, first=4, recent=0),
    dict(N=3, Hkv=1, dh=64, T=203, P=64, to_P=5, keep=50, first=60, recent=7),        # all first
    dict(N=3, Hkv=1, dh=32, T=203, P=64, to_P=1, keep=50, first=3, recent=90),        # all protected
    dict(N=3, Hkv=3, dh=64, T=100, P=5, to_P=16, keep=130, first=3, recent=9),        # nothing to leave out
    dict(N=2, Hkv=2, dh=64, T=3000, P=48, to_P=64, keep=1000, first=1, recent=100),
    dict(N=2, Hkv=1, dh=128, T=9001, P=64, to_P=16, keep=17, first=0, recent=1),
    dict(N=1, Hkv=1, dh=32, T=70001, P=64, to_P=64, keep=30000, first=5, recent=1000),
]


def _weights(kind, r, shape):
    if kind == "ties":
        return r.choice([0.0, -0.0, 1.0, 0.5], shape)
    if kind == "one":
        return np.full(shape, 0.25)
    if kind == "odd":
        return r.choice([NAN, INF, -INF, -1.0, 0.0, 1e-42, 2.5, 3e38], shape)
    return r.standard_normal(shape) ** 3


@pytest.mark.parametrize("kind", ["random", "ties", "one", "odd"])
@pytest.mark.parametrize("kw", EVICT, ids=IDS)
def test_evict(kw, kind):
    _say("evict", kw, kind)
    r = np.random.default_rng(11)
    N, Hkv, dh, T, P, to_P, keep = (kw[n] for n in ("N", "Hkv", "dh", "T", "P", "to_P", "keep"))
    cols, to_cols = -(-T // P), -(-keep // to_P)
    pages = torch.tensor(r.integers(0, 256, (N * cols + 1, Hkv * ref.head_bytes(P, dh))).astype(np.uint8)).cuda()
    table = r.permutation(N * cols + 1)[:N * cols].reshape(N, cols)
    to_table = r.permutation(N * to_cols + 2)[:N * to_cols].reshape(N, to_cols)
    to_pages = torch.full((N * to_cols + 2, Hkv * ref.head_bytes(to_P, dh)), 77, dtype=torch.uint8, device="cuda")
    length = r.integers(T // 2, T + 1, N)
    length[-1] = T
    if N > 2:
        length[0] = 0 if kind == "odd" else 1
    w = _weights(kind, r, (N, Hkv, cols * P)).astype(np.float32)
    frm = PagedCache4(pages, _i32(table), P, Hkv, dh, _i32(length))
    to = PagedCache4(to_pages, _i32(to_table), to_P, Hkv, dh)
    w_out = torch.full((N, Hkv, to.capacity), 5.0, device="cuda")
    kept = frm.evict(torch.tensor(w).cuda(), to, keep=keep, first=kw["first"], recent=kw["recent"], weights_out=w_out).cpu().numpy()
    want_to = np.full((N * to_cols + 2, Hkv, ref.head_bytes(to_P, dh)), 77, np.uint8)
    src = pages.cpu().numpy().reshape(-1, Hkv, ref.head_bytes(P, dh))
    w_out = w_out.cpu().numpy()
    for s in range(N):
        for h in range(Hkv):
            rows = np.array(ref.evict_rows(w[s, h], int(length[s]), keep, kw["first"], kw["recent"]), int)
            m = rows.size
            assert np.array_equal(kept[s, h, :m], rows) and (kept[s, h, m:] == -1).all()
            assert np.array_equal(w_out[s, h, :m], w[s, h, rows], equal_nan=True) and (w_out[s, h, m:] == 5).all()
            for part in (0, 1):
                for width, off, step in ((dh // 2, 0, dh // 2), (dh // 32, None, dh // 32)):
                    at = lambda P_, x: (part * P_ + x % P_) * step + (0 if off == 0 else P_ * dh)             # noqa: E731
                    d = np.arange(m)
                    span = np.arange(width)
                    want_to[to_table[s, d // to_P][:, None], h, at(to_P, d)[:, None] + span] = \
                        src[table[s, rows // P][:, None], h, at(P, rows)[:, None] + span]
    assert np.array_equal(to_pages.cpu().numpy().reshape(want_to.shape), want_to)
    assert to.len.cpu().tolist() == np.minimum(length, keep).tolist() and frm.status.cpu().tolist() == [0] * N
    assert frm.len.cpu().tolist() == length.tolist()


@pytest.mark.parametrize("keep,first,recent", [(300, 200, 150), (300, 200, 100), (300, 0, 0), (301, 10, 20), (2999, 1, 1), (1, 0, 0)])
@pytest.mark.parametrize("T", [3000, 9001, 40000])
def test_evict_where_digits_end(T, keep, first, recent):
    """Weights of which exactly as many as are kept, one more or one fewer share their upper digits; NaN and -infinity at the cut."""
    _say("evict, digits", T, keep, first, recent)
    r = np.random.default_rng(T + keep)
    w = np.full((1, 8, T), 1e-30, np.float32)
    for h, (high, low) in enumerate([(1e30, 1e-30), (1.0, 1.0 + 2.0 ** -23), (1.5, 1.25), (0.0, NAN), (-INF, NAN), (NAN, NAN), (INF, -INF),
                                     (1.0 + 2.0 ** -15, 1.0)]):
        w[0, h] = low
        w[0, h, r.permutation(T)[:max(keep - first - recent, 0) + h % 3 - 1]] = high
    pool = torch.zeros(1, PagedCache4.page_bytes(64, 8, 32), dtype=torch.uint8, device="cuda")
    cols, to_cols = -(-T // 64), -(-keep // 64)
    full = np.zeros((1, 8, cols * 64), np.float32)
    full[:, :, :T] = w
    frm = PagedCache4(pool, torch.zeros(1, cols, dtype=torch.int32, device="cuda"), 64, 8, 32, _i32([T]))
    to = PagedCache4(torch.zeros_like(pool), torch.zeros(1, to_cols, dtype=torch.int32, device="cuda"), 64, 8, 32)
    kept = frm.evict(torch.tensor(full).cuda(), to, keep=keep, first=first, recent=recent).cpu().numpy()
    for h in range(8):
        assert kept[0, h].tolist() == ref.evict_rows(w[0, h], T, keep, first, recent), h


def test_evict_rows_without_a_page():
    P, Hkv, dh = 4, 1, 32
    r = np.random.default_rng(0)
    pages = torch.tensor(r.integers(0, 256, (12, ref.head_bytes(P, dh))).astype(np.uint8)).cuda()
    to_pages = torch.zeros_like(pages)
    frm = PagedCache4(pages, _i32([[0, 1, 2], [3, 99, 4], [5, 6, 7], [8, 9, -1]]), P, Hkv, dh, _i32([12, 12, 12, 8]))
    to = PagedCache4(to_pages, _i32([[0, 1], [2, 3], [-1, 5], [6, 7]]), P, Hkv, dh)
    w = torch.tensor(r.random((4, 1, 12))).float().cuda()
    kept = frm.evict(w, to, keep=8)
    assert frm.status.tolist() == [0, 4, 4, 0] and to.len.tolist() == [8] * 4
    k, v = to.read()
    fk, fv = frm.read()
    for s in range(4):
        rows = ref.evict_rows(w[s, 0].tolist(), int(frm.len[s]), 8, 0, 0)
        assert kept[s, 0].tolist() == rows
        for i, j in enumerate(rows):
            if (s == 1 and j // 4 == 1) or (s == 2 and i // 4 == 0):      # left as it was: zeros
                assert (k[s, i] == 0).all() and (v[s, i] == 0).all()
            else:
                assert torch.equal(k[s, i].nan_to_num(7.0), fk[s, j].nan_to_num(7.0)) and torch.equal(v[s, i].nan_to_num(7.0), fv[s, j].nan_to_num(7.0))


# ---------------------------------------------------------------------------------------------
# Together
# ---------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_hypotheses_grow_over_a_document(dtype):
    """A document enters the cache, lists grow token by token, the document's rows are evicted by what they received, and the
    lists go on: against the attention over the values that the cache holds."""
    B, K, H, Hkv, dh, P, T, L = 2, 6, 4, 2, 64, 16, 160, 32
    g = torch.Generator(device="cuda").manual_seed(5)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").to(ACT[dtype])                           # noqa: E731
    pages = torch.full((100, PagedCache4.page_bytes(P, Hkv, dh)), 255, dtype=torch.uint8, device="cuda")
    ids = torch.randperm(100, generator=g, device="cuda").int()
    ctx = PagedCache4(pages, ids[:20].view(B, 10).contiguous(), P, Hkv, dh)
    own = PagedCache4(pages, ids[20:44].view(B * K, 2).contiguous(), P, Hkv, dh)
    small = PagedCache4(pages, ids[44:52].view(B, 4).contiguous(), P, Hkv, dh)
    freq = torch.tensor(1000.0 ** -(np.arange(32) / 32)).cuda()
    n = torch.tensor([150, 111]).int().cuda()
    ctx.append(rnd(B, 150, Hkv, dh), rnd(B, 150, Hkv, dh), new_len=n, freq=freq)
    pos0 = n.repeat_interleave(K)
    cw, ow = torch.zeros(B, Hkv, T, device="cuda"), torch.zeros(B * K, Hkv, L, device="cuda")
    received = np.zeros((B, Hkv, T))
    plans = {t: PrefixAttention4(B=B, K=K, S=1, T=t, L=L, n_heads=H, n_kv_heads=Hkv, dh=dh, dtype=dtype, causal=True) for t in (T, 64)}
    shared, weights = ctx, cw
    for step in range(9):
        if step == 6:
            shared = small
            weights = torch.zeros(B, Hkv, 64, device="cuda")
            kept = ctx.evict(cw, small, keep=50, first=2, recent=10, weights_out=weights)
            for b in range(B):
                for h in range(Hkv):
                    assert kept[b, h].tolist() == ref.evict_rows(cw[b, h].tolist(), int(n[b]), 50, 2, 10)
            assert small.len.tolist() == [50, 50]
            ck, cv = (x.gather(1, kept.transpose(1, 2).long()[..., None].expand(B, 50, Hkv, dh)) for x in ctx.read())
            sk, sv = small.read()
            assert torch.equal(sk[:, :50], ck) and torch.equal(sv[:, :50], cv)
        q = own.append(rnd(B * K, 1, Hkv, dh), rnd(B * K, 1, Hkv, dh), q=rnd(B * K, 1, H, dh), freq=freq, pos0=pos0)
        q = q.view(B, K, 1, H, dh)
        plan = plans[shared.capacity]
        out = plan.run(q, shared, own)
        plan.weigh(q, plan.lse, shared, own, weights, ow)
        ck, cv, ok, ov = (_np(x) for c in (shared, own) for x in c.read())
        lens = dict(ctx_len=shared.len.cpu().numpy(), q_len=None, own_len=own.len.cpu().numpy().reshape(B, K))
        want = dense.attend(_np(q), ck, cv, ok.reshape(B, K, L, Hkv, dh), ov.reshape(B, K, L, Hkv, dh), dtype=dtype, causal=True, **lens)
        _near(out, want["out"], "out")
        _near(plan.lse, want["lse"], "lse")
        # the weights of a request's rows add up to their number, step after step (each to fp32's roundings)
        if step < 6:
            total = weights.double().sum((1, 2)) + ow.double().view(B, K, Hkv, L).sum((1, 2, 3))
            assert (total - (step + 1) * K * H).abs().max() <= (step + 1) * K * H * 2.0 ** -24 * 64 * 40
    assert (own.status == 0).all() and own.len.tolist() == [9] * (B * K)


def test_the_same_values_as_the_dense_attention():
    """What the cache holds, read back, gives PrefixAttention the same result to its roundings."""
    c = Case("bf16", B=2, K=5, S=6, H=4, Hkv=2, dh=64, T=90, L=20, P=10, lens="full", seed=3).device()
    out, _ = c.run()
    ck, cv = c.ctx.read()
    ok, ov = (x.view(2, 5, 20, 2, 64) for x in c.own.read())
    full = PrefixAttention(B=2, K=5, S=6, T=90, L=20, n_heads=4, n_kv_heads=2, dh=64, dtype="bf16", causal=True)
    other = full.run(c.qd, ck, cv, ok, ov)
    want = c.reference()["out"]
    assert (np.abs(_np(out) - _np(other)) <= 2 * want[1]).all()


# ---------------------------------------------------------------------------------------------
# Refusals that need tensors on the GPU
# ---------------------------------------------------------------------------------------------

def test_refusals():
    c = Case("bf16", B=1, K=2, S=1, H=2, Hkv=1, dh=32, T=8, L=4, P=4, lens="full").device()
    plan = c.plan()
    with pytest.raises(ValueError, match="own"):
        plan.run(c.qd, c.ctx, None)
    with pytest.raises(ValueError, match="ctx"):
        plan.run(c.qd, c.own, c.own)
    with pytest.raises(ValueError, match="q"):
        plan.run(c.qd.float(), c.ctx, c.own)
    with pytest.raises(ValueError, match="ctx_w"):
        plan.weigh(c.qd, plan.lse, c.ctx, c.own, ctx_w=torch.zeros(3, device="cuda"))
    with pytest.raises(ValueError, match="pages"):
        PagedCache4(c.dev[:, :-16].contiguous(), c.ctx.table, 4, 1, 32)
    with pytest.raises(ValueError, match="to"):
        c.ctx.evict(torch.zeros(1, 1, 8, device="cuda"), c.own, keep=1)
    with pytest.raises(fe.FeError, match="capacity"):
        to = PagedCache4(c.dev, _i32([[0]]), 4, 1, 32)
        c.ctx.evict(torch.zeros(1, 1, 8, device="cuda"), to, keep=5)
    with pytest.raises(fe.FeError, match="of its own"):
        c.ctx.evict(torch.zeros(1, 1, 8, device="cuda"), c.ctx, keep=5)
    x = torch.zeros(2, 1, 1, 32, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(fe.FeError, match="q_out"):
        c.own.append(x, x, q=x, q_out=x)
    with pytest.raises(ValueError, match="k"):
        c.own.append(x.half(), x.half())
    with pytest.raises(ValueError, match="count"):
        c.own.read(x, x, count=torch.zeros(2, device="cuda"))
    assert math.isfinite(float(plan.run(c.qd, c.ctx, c.own).float().sum()))


# ---------------------------------------------------------------------------------------------
# Log sums of any strides
# ---------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kw", [
    dict(dtype="bf16", B=8, K=16, S=1, H=8, Hkv=8, dh=64, T=100, L=20),
    dict(dtype="bf16", B=2, K=5, S=3, H=4, Hkv=2, dh=128, T=70, L=20, P=7),
    dict(dtype="f32", B=3, K=4, S=6, H=4, Hkv=2, dh=32, T=50, L=16, P=5),
    dict(dtype="bf16", B=1, K=60, S=30, H=4, Hkv=1, dh=32, T=70, L=30),
    dict(dtype="f32", B=1, K=1, S=1, H=1, Hkv=1, dh=32, T=9, L=0),
], ids=IDS)
def test_weights_of_strided_log_sums(kw):
    """Log sums head by head, row by row, in a wider tensor and shared along an axis: the weights of the dense ones."""
    _say("strided log sums", kw)
    c = Case(**kw, seed=12).device()
    plan = c.plan()
    _, lse = c.run(plan)
    lse = lse.clone()

    def weights(lse):
        w = torch.zeros(c.B, c.Hkv, c.T, device="cuda"), torch.zeros(c.B * c.K, c.Hkv, c.L, device="cuda")
        plan.weigh(c.qd, lse, c.ctx, c.own, w[0] if c.T else None, w[1] if c.L else None, q_len=c.q_len)
        return w

    def wide(x):
        y = torch.full([2 * n + 1 for n in x.shape], NAN, device="cuda")[:x.shape[0], 1:1 + x.shape[1], -x.shape[2]:, :x.shape[3]]
        return y.copy_(x)

    want = weights(lse)
    by_head = lse.view(c.B, c.K, c.S, c.Hkv, -1).permute(0, 3, 1, 2, 4).contiguous()
    for got in (weights(by_head.permute(0, 2, 3, 1, 4).flatten(3, 4)), weights(lse.permute(3, 2, 1, 0).contiguous().permute(3, 2, 1, 0)),
                weights(wide(lse))):
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    one = lse[:, :1].expand(lse.shape)
    for a, b in zip(weights(one), weights(one.contiguous())):
        assert torch.equal(a, b)


def test_refusals_of_log_sums():
    c = Case("bf16", B=2, K=2, S=1, H=2, Hkv=1, dh=32, T=8, L=4, P=4, lens="full").device()
    plan = c.plan()
    w = torch.zeros(2, 1, 8, device="cuda")
    for lse in (torch.zeros(2, 2, 1, 2, device="cuda").double(), torch.zeros(2, 2, 1, 3, device="cuda")[..., :1], torch.zeros(7, device="cuda"),
                torch.zeros(2, 2, 2, 1, device="cuda").transpose(0, 2)[:, :, :, :1].expand(2, 2, 2, 2)):
        with pytest.raises(ValueError, match="lse"):
            plan.weigh(c.qd, lse, c.ctx, c.own, ctx_w=w)


# ---------------------------------------------------------------------------------------------
# Infinite scores
# ---------------------------------------------------------------------------------------------

INFINITE = [
    dict(dtype="bf16", B=1, K=1, S=1, H=1, Hkv=1, dh=32, T=1, L=0, P=1, lens="full"),
    dict(dtype="bf16", B=2, K=5, S=1, H=4, Hkv=4, dh=32, T=181, L=12),
    dict(dtype="bf16", B=64, K=1, S=2, H=8, Hkv=8, dh=128, T=37, L=9, P=4),
    dict(dtype="bf16", B=1, K=45, S=1, H=2, Hkv=2, dh=32, T=150, L=20, P=48),
    dict(dtype="bf16", B=1, K=1, S=50, H=1, Hkv=1, dh=128, T=70, L=80, P=16),
    dict(dtype="bf16", B=1, K=140, S=1, H=1, Hkv=1, dh=128, T=700, L=9, P=64),
    dict(dtype="bf16", B=1, K=2, S=150, H=3, Hkv=1, dh=128, T=20, L=150, P=48, lens="own"),
    dict(dtype="bf16", B=1, K=3, S=1, H=4, Hkv=1, dh=64, T=3000, L=100, P=64),
    dict(dtype="f32", B=1, K=2, S=2, H=2, Hkv=1, dh=64, T=4500, L=10, P=48),
    dict(dtype="f32", B=2, K=13, S=11, H=4, Hkv=4, dh=32, T=64, L=11, P=5, causal=False, lens="own"),
    # rows without keys, pages outside the pool
    dict(dtype="bf16", B=6, K=5, S=3, H=4, Hkv=2, dh=32, T=40, L=9, P=4, lens="edge"),
    dict(dtype="bf16", B=6, K=5, S=9, H=4, Hkv=2, dh=64, T=140, L=70, P=10, lens="edge", causal=False),
    dict(dtype="f32", B=6, K=7, S=4, H=2, Hkv=1, dh=32, T=33, L=20, P=3, lens="edge"),
    dict(dtype="bf16", B=3, K=4, S=2, H=4, Hkv=2, dh=64, T=10, L=10, P=5, holes=16),
    dict(dtype="f32", B=2, K=50, S=1, H=4, Hkv=2, dh=128, T=16, L=16, P=8, holes=70),
]


def _first_column(c, code):
    """Column 0 of every cached key is the 4-bit float `code` of its block's scale."""
    for r in range(c.P):
        at = ref.place(c.P, c.dh, 0, r)[0].start
        c.pages[:, :, at] = c.pages[:, :, at] & 0xF0 | code
    return c


def _sees(c):
    """[B][K][S] rows that see a key."""
    nc, nq, no = c.lengths()
    ctx, own = c.seen(c.ct), c.seen(c.ot).reshape(c.B, c.K, c.L)
    some = np.zeros((c.B, c.K, c.S), bool)
    for b in range(c.B):
        for k in range(c.K):
            for i in range(nq[b, k]):
                m = no[b, k]
                to = min(max(m - nq[b, k] + i + 1, 0), m) if c.causal else m
                some[b, k, i] = ctx[b, :nc[b]].any() or own[b, k, :to].any()
    return some


@pytest.mark.parametrize("scale", [0.125, -0.125])
@pytest.mark.parametrize("kw", INFINITE, ids=IDS)
def test_rows_whose_scores_are_all_minus_infinity_are_nan(kw, scale):
    """Queries with an infinity over keys whose column has the other sign: NaN, as softmax of such scores is, and not the zeros
    of a row that sees no key."""
    _say("all -infinity", kw, scale)
    c = _first_column(Case(**kw, scale=scale, seed=21), 2)
    live = ~np.isnan(c.q[..., 0])
    c.q[..., 0] = np.where(live, -INF if scale > 0 else INF, NAN)
    out, lse = c.device().run()
    some = torch.tensor(_sees(c)).cuda()
    assert torch.isnan(out[some]).all() and torch.isnan(lse[some]).all()
    assert (out[~some] == 0).all() and torch.isneginf(lse[~some]).all()


@pytest.mark.parametrize("kw", [k for k in INFINITE if k.get("lens") != "edge"], ids=IDS)
def test_rows_beside_one_with_infinite_scores_keep_their_bits(kw):
    c = _first_column(Case(**kw, seed=22), 2).device()
    out, lse = (t.clone() for t in c.run())
    row = (c.B - 1, c.K // 2, 0, c.H - 1)
    for value in (-INF, INF, NAN):
        c.qd[row][0] = value
        got, lse2 = c.run()
        other = torch.ones_like(lse, dtype=torch.bool)
        other[row] = False
        assert torch.equal(got[other], out[other]) and torch.equal(lse2[other], lse[other])
        if _sees(c)[row[:3]]:
            assert torch.isnan(got[row]).all() and torch.isnan(lse2[row])


@pytest.mark.parametrize("kw", [INFINITE[1], INFINITE[4], INFINITE[5], INFINITE[7], INFINITE[8]], ids=IDS)
def test_a_score_of_minus_infinity_beside_finite_ones_weighs_nothing(kw):
    """Products that overflow for some keys: the row is the softmax over the others, the bits that they give without these."""
    c = Case(**{**kw, "lens": "full"}, seed=23)
    nc, _, no = c.lengths()
    c.q[..., 0] = -2.0 ** 127
    _first_column(c, 0)                                                  # a 0 there: finite
    far = [(c.ct, b, j) for b in range(c.B) for j in range(0, nc[b], 3)] + \
          [(c.ot, s, j) for s in range(c.B * c.K) for j in range(0, no.reshape(-1)[s], 2)] if c.L else []
    for t, s, j in far:
        at, by = ref.place(c.P, c.dh, 0, j % c.P)
        c.pages[t[s, j // c.P], :, at.start] |= 7                        # 6 times a scale of 1: beyond fp32
        c.pages[t[s, j // c.P], :, by.start] = 127
    got, lse = c.device().run()
    # the same keys far below the others, by a finite query
    c.q[..., 0] = -2.0 ** 90
    want, lse2 = c.device().run()
    assert torch.isfinite(got).all() and torch.equal(got, want) and torch.equal(lse, lse2)


# ---------------------------------------------------------------------------------------------
# Turned queries
# ---------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kw", [k for k in APPEND if k["H"]], ids=lambda k: f"{k['dtype']}-N{k['N']}-S{k['S']}-dh{k['dh']}-rot{k['rot']}-P{k['P']}")
def test_append_turns_queries_to_the_nearest(kw):
    """q_out is the turned query rounded once: off by half a step of its own size, and by the fp64 products of sines good to
    2^-52, 2^-50 (|a| + |b|) in all."""
    c = _append_case(**kw, seed=31)
    empty = np.zeros((c["n_pages"], kw["Hkv"], ref.head_bytes(kw["P"], kw["dh"])), np.uint8)
    q0 = np.full((kw["N"], kw["S"], kw["H"], kw["dh"]), 7.0)
    _, want = _append_want(c, pages=empty.copy(), q_out=q0.copy(), **kw)
    _, got, _ = _append_run(c, pages=empty, q_out=q0, **kw)
    pair = dense.turned_bound(c["q"], c["freq"], kw["near"], kw["dtype"]) / (dense.HALF_STEP[kw["dtype"]] + 2.0 ** -21)
    assert (np.abs(_np(got) - want) <= dense.HALF_STEP[kw["dtype"]] * np.abs(want) + 2.0 ** -50 * pair).all()


def test_append_turns_queries_next_to_a_border():
    """Turned queries down to 2^-22 from the border between two bf16 numbers, on both sides, go to the nearer one."""
    r = np.random.default_rng(7)
    N, angle = 4000, 0.7
    b = torch.tensor(r.uniform(1, 2, (N, 16))).bfloat16().double().numpy()
    a = torch.tensor(r.uniform(1, 2, (N, 16))).bfloat16().double().numpy()
    c = dict(q=np.concatenate((a, b), -1)[:, None, None], k=np.zeros((N, 1, 1, 32)), v=np.zeros((N, 1, 1, 32)), new=np.ones(N, int),
             len=np.zeros(N, int), pos0=np.ones(N, int), freq=np.full(16, angle), table=np.arange(N)[:, None])
    kw = dict(dtype="bf16", Hkv=1, dh=32, rot=32, P=1, near=False)
    empty, q0 = np.zeros((N, 1, ref.head_bytes(1, 32)), np.uint8), np.zeros((N, 1, 1, 32))
    _, want = _append_want(c, N=N, pages=empty.copy(), q_out=q0.copy(), **kw)
    _, got, _ = _append_run(c, pages=empty, q_out=q0, **kw)
    # the smallest are about 2^-14, so fp64 products of size 2 are off by 2^-36 of them at most, 2^16 units of 2^-52: less than
    # any one's distance from a border, and the nearest bf16 number is the same by every fp64 way to it
    bits = want.view(np.int64)
    rest = (bits & ((1 << 45) - 1)) - (1 << 44)                          # to the border, in units of 2^-52 of the exponent
    assert np.abs(want).min() > 2.0 ** -15 and 1 << 24 < np.abs(rest).min() < 1 << 30
    nearest = ((bits + (1 << 44)) & ~((1 << 45) - 1)).view(np.float64)
    assert np.array_equal(_np(got), nearest)


# ---------------------------------------------------------------------------------------------
# Scales of 0 and next to it
# ---------------------------------------------------------------------------------------------

@pytest.mark.parametrize("scale", [0.0, -0.0, 2.0 ** -124, -2.0 ** -126, 2.0 ** -128])
@pytest.mark.parametrize("kw", [dict(dtype="bf16", B=2, K=3, S=2, H=2, Hkv=2, dh=32, T=60, L=12, P=4),
                                dict(dtype="f32", B=2, K=3, S=2, H=2, Hkv=2, dh=32, T=60, L=12, P=4),
                                dict(dtype="bf16", B=1, K=40, S=2, H=2, Hkv=1, dh=64, T=70, L=12, P=4),
                                dict(dtype="bf16", B=1, K=2, S=2, H=2, Hkv=1, dh=128, T=1500, L=12, P=16)], ids=IDS)
def test_scales_next_to_zero_over_large_products(kw, scale):
    """Products of queries and keys up to 2^127: a scale of 0 gives every key the same weight, one of 2^-126 the weights of that."""
    class Large(Case):
        def __init__(self, **kw):
            super().__init__(**kw)
            self.q *= 2.0 ** 98
            self.ck *= 2.0 ** 24
            self.ok *= 2.0 ** 24
            for r in range(self.P):                                       # the scale bytes of the keys
                at = ref.place(self.P, self.dh, 0, r)[1]
                self.pages[:, :, at] = np.where(self.pages[:, :, at] == 255, 255, np.minimum(self.pages[:, :, at], 230) + 24)

    c = Large(**kw, scale=scale, seed=41).device()
    want = c.reference()
    out, lse = c.run()
    _near(out, want["out"], "out")
    _near(lse, want["lse"], "lse")
    nc, nq, no = c.lengths()
    cw, ow = np.zeros((c.B, c.Hkv, c.T), np.float32), np.zeros((c.B, c.K, c.Hkv, c.L), np.float32)
    at = lse.cpu().numpy()
    weights = ref.weigh(c.q, c.ck, c.ok, at, causal=c.causal, scale=c.scale, ctx_len=nc, q_len=nq, own_len=no, ctx_w=cw, own_w=ow)
    cd, od = torch.tensor(cw).cuda(), torch.tensor(ow).cuda()
    c.plan().weigh(c.qd, lse, c.ctx, c.own, cd, od, q_len=c.q_len)
    _near(cd, weights["ctx_w"], "ctx_w")
    _near(od, weights["own_w"], "own_w")


def test_a_scale_of_zero_over_what_is_no_number():
    """0 times an infinity is no number: the row is NaN, whatever the infinity's sign; the others keep their bits."""
    c = _first_column(Case("bf16", B=2, K=3, S=2, H=2, Hkv=2, dh=64, T=60, L=12, P=4, scale=0.0, lens="full", seed=42), 2).device()
    out, lse = (t.clone() for t in c.run())
    for value in (INF, -INF, NAN):
        c.qd[1, 1, 0, 1, 0] = value
        got, lse2 = c.run()
        other = torch.ones_like(lse, dtype=torch.bool)
        other[1, 1, 0, 1] = False
        assert torch.isnan(got[1, 1, 0, 1]).all() and torch.isnan(lse2[1, 1, 0, 1])
        assert torch.equal(got[other], out[other]) and torch.equal(lse2[other], lse[other])


# ---------------------------------------------------------------------------------------------
# Two threads
# ---------------------------------------------------------------------------------------------

def _during(monkeypatch, name, other):
    """The binding's call `name` runs `other` once just before it enters the library, as another thread may."""
    real, calls = getattr(fe, name), []

    def call(args, stream=None):
        if not calls:
            calls.append(1)
            other()
        real(args, stream)

    monkeypatch.setattr(fe, name, call)


def test_reads_and_evictions_of_one_cache_from_two_threads(monkeypatch):
    """A call's arguments are its own: another thread's call on the same cache in between does not change them."""
    P, Hkv, dh, N = 8, 2, 64, 3
    g = torch.Generator(device="cuda").manual_seed(9)
    width = PagedCache4.page_bytes(P, Hkv, dh)
    pages = lambda n: torch.zeros(n, width, dtype=torch.uint8, device="cuda")                             # noqa: E731
    cache = PagedCache4(pages(N * 4), torch.arange(N * 4, device="cuda").int().view(N, 4), P, Hkv, dh)
    cache.append(*(torch.randn(N, 30, Hkv, dh, generator=g, device="cuda").bfloat16() for _ in range(2)))
    want = [t.clone() for t in cache.read()]
    new = lambda n, dt: [torch.full((N, n, Hkv, dh), 3.0, dtype=dt, device="cuda") for _ in range(2)]     # noqa: E731
    one, two = new(32, torch.bfloat16), new(7, torch.float32)
    start = _i32([5, 0, 20])
    with monkeypatch.context() as m:
        _during(m, "fe_packed_read", lambda: cache.read(*two, start=start))
        cache.read(*one)
    for a, b, w in zip(one, two, want):
        assert torch.equal(a[:, :30], w[:, :30]) and (a[:, 30:] == 3).all()
        for s, f in enumerate((5, 0, 20)):
            assert torch.equal(b[s], w[s, f:f + 7].float())
    to = [PagedCache4(pages(N * 2), torch.arange(N * 2, device="cuda").int().view(N, 2), P, Hkv, dh) for _ in range(2)]
    w = [torch.rand(N, Hkv, 32, generator=g, device="cuda") for _ in range(2)]
    got = []
    with monkeypatch.context() as m:
        _during(m, "fe_packed_evict", lambda: got.append(cache.evict(w[1], to[1], keep=5, recent=2)))
        got.insert(0, cache.evict(w[0], to[0], keep=16, first=1))
    for i, (keep, first, recent) in enumerate(((16, 1, 0), (5, 0, 2))):
        assert to[i].len.tolist() == [keep] * N
        k, _ = to[i].read()
        for s in range(N):
            for h in range(Hkv):
                rows = ref.evict_rows(w[i][s, h].tolist(), 30, keep, first, recent)
                assert got[i][s, h].tolist() == rows and torch.equal(k[s, :keep, h], want[0][s, rows, h])


def test_many_threads_read_one_cache():
    """Eight threads, each with a layout, a stream and outputs of its own."""
    import threading
    P, Hkv, dh, N = 8, 2, 32, 2
    cache = PagedCache4(torch.zeros(N * 8, PagedCache4.page_bytes(P, Hkv, dh), dtype=torch.uint8, device="cuda"),
                        torch.arange(N * 8, device="cuda").int().view(N, 8), P, Hkv, dh)
    cache.append(*(torch.randn(N, 64, Hkv, dh, device="cuda").bfloat16() for _ in range(2)))
    want = [t.clone() for t in cache.read()]
    torch.cuda.synchronize()
    bad = []

    def reads(i):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for n in range(1, 40):                                    # n + i stays below 64
                    k, v = (torch.zeros(N, n + i, Hkv, dh, dtype=torch.bfloat16, device="cuda") for _ in range(2))
                    cache.read(k, v)
                    if not (torch.equal(k, want[0][:, :n + i]) and torch.equal(v, want[1][:, :n + i])):
                        bad.append((i, n))
        except Exception as e:                                            # noqa: BLE001
            bad.append(repr(e))

    threads = [threading.Thread(target=reads, args=(i,)) for i in range(8)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad, bad[:5]


# ---------------------------------------------------------------------------------------------
# Parts of prompts over long documents: own rows in the common loop, ranges of keys that are joined
# ---------------------------------------------------------------------------------------------

PARTS = [
    dict(dtype="bf16", B=1, K=1, S=200, H=4, Hkv=2, dh=128, T=1500, L=400),
    dict(dtype="bf16", B=1, K=1, S=200, H=4, Hkv=2, dh=128, T=1500, L=400, lens="full"),
    dict(dtype="bf16", B=2, K=3, S=70, H=2, Hkv=2, dh=64, T=900, L=150, P=7),
    dict(dtype="bf16", B=1, K=1, S=60, H=2, Hkv=2, dh=32, T=2000, L=300, P=48),
    dict(dtype="bf16", B=1, K=3, S=70, H=2, Hkv=2, dh=32, T=1000, L=90, P=5, causal=False),
    dict(dtype="f32", B=1, K=1, S=150, H=2, Hkv=1, dh=64, T=1100, L=320),
    dict(dtype="f32", B=1, K=1, S=130, H=1, Hkv=1, dh=128, T=800, L=200, P=48),
    dict(dtype="f32", B=1, K=2, S=70, H=2, Hkv=2, dh=32, T=700, L=130, P=7),
    dict(dtype="bf16", B=2, K=2, S=90, H=2, Hkv=1, dh=64, T=1200, L=200, holes=20),
    # ... in proportion to the requests' lengths
    dict(dtype="bf16", B=4, K=1, S=130, H=4, Hkv=4, dh=32, T=16384, L=200, P=64),
    dict(dtype="bf16", B=2, K=2, S=66, H=8, Hkv=8, dh=64, T=16384, L=100, P=64),
]


@pytest.mark.parametrize("kw", PARTS, ids=IDS)
def test_attention_of_prompt_parts(kw):
    c = Case(**kw, seed=1)
    size = fe.fe_packed_workspace_size(_sizes(c))
    assert size > 0                                                       # several ranges of keys
    test_attention(kw)


@pytest.mark.parametrize("kw", PARTS[:9], ids=IDS)
def test_weights_of_prompt_parts(kw):
    test_weights(kw)


@pytest.mark.parametrize("kw", [dict(dtype="bf16", B=2, K=9, S=4, H=4, Hkv=2, dh=64, T=50, L=24, P=4),
                                dict(dtype="bf16", B=1, K=3, S=70, H=2, Hkv=2, dh=32, T=1000, L=90, P=5),
                                dict(dtype="f32", B=2, K=13, S=3, H=2, Hkv=1, dh=64, T=300, L=30, P=16)], ids=IDS)
def test_a_list_beside_lists_of_other_lengths(kw):
    """Other lengths of the other lists move a list's keys to other places, so that its sums may have another order, and no more."""
    c = Case(**kw, lens="full", seed=14)
    own = c.K // 2
    for others in (0, 1, 3):
        d = Case(**kw, lens="full", seed=14)
        d.nq, d.no = np.full((c.B, c.K), min(others, c.S)), np.full((c.B, c.K), others)
        d.nq[:, own], d.no[:, own] = c.S, c.no[:, own]
        d.device()
        want = d.reference()
        out, lse = d.run()
        _near(out, want["out"], "out")
        _near(lse, want["lse"], "lse")
        assert torch.isfinite(out[:, own]).all()

"""Shared-prefix attention, its gradient and the paged-cache append on the GPU against the float64 loops of
tests/prefix_reference.py, within the bounds derived there; what lies outside the lengths holds NaN."""
import numpy as np
import pytest
import torch

import gen
from paper_2603_02565_amd import flasheval as fe
from tests import prefix_reference as ref
from tests.gpu_harness import make_evaluator, upload

pytestmark = pytest.mark.gpu

ACT = {"bf16": torch.bfloat16, "f32": torch.float32}
NAN, INF = float("nan"), float("inf")


def _say(*what):
    print(*what, flush=True)


def _lens(kind, r, B, K, S, T, L, causal):
    """(ctx_len, q_len, own_len) of a kind of batch, int arrays or None."""
    if kind == "full":
        return None, None, None
    if kind == "ragged":
        q = r.integers(1, S + 1, (B, K))
        return r.integers(0, T + 1, B), q, np.minimum(q + r.integers(0, L + 1, (B, K)), L)
    if kind == "own":                                   # the own rows are the query rows
        q = r.integers(0, min(S, L) + 1, (B, K))
        return r.integers(0, T + 1, B), q, q.copy()
    assert kind == "edge"                               # no context, no rows, no own keys, fewer own keys than rows, lengths out of range
    c = r.choice([0, 0, 1, T, T + 5, -3], B)
    return c, r.choice([0, 1, S, S + 2, -1], (B, K)), r.choice([0, 1, L, L + 9, -7], (B, K))


class Case:
    def __init__(self, dtype, B, K, S, H, Hkv, dh, T, L, P=0, causal=True, lens="ragged", seed=0, amp=1.0, scale=None):
        r = np.random.default_rng(seed)
        self.dims = dict(B=B, K=K, S=S, T=T, n_heads=H, n_kv_heads=Hkv, dh=dh, dtype=dtype, causal=causal, scale=scale)
        self.dtype, self.P, self.L = dtype, P, L
        cols = -(-L // P) if P else 0
        self.Lcap = cols * P if P else L
        dt = ACT[dtype]
        rnd = lambda *s: torch.tensor(r.standard_normal(s) * amp).to(dt).double().numpy()       # noqa: E731
        self.q, self.do = rnd(B, K, S, H, dh), rnd(B, K, S, H, dh)
        self.ck, self.cv = rnd(B, T, Hkv, dh), rnd(B, T, Hkv, dh)
        self.ok, self.ov = rnd(B, K, self.Lcap, Hkv, dh), rnd(B, K, self.Lcap, Hkv, dh)
        self.ctx_len, self.q_len, self.own_len = _lens(lens, r, B, K, S, T, L, causal)
        nc, nq, no = ref.clamp_lengths(B, K, S, T, self.Lcap, self.ctx_len, self.q_len, self.own_len)
        self.nc, self.nq, self.no = nc, nq, no
        for b in range(B):
            self.ck[b, nc[b]:] = self.cv[b, nc[b]:] = NAN
            for k in range(K):
                self.q[b, k, nq[b, k]:] = self.do[b, k, nq[b, k]:] = NAN
                self.ok[b, k, no[b, k]:] = self.ov[b, k, no[b, k]:] = NAN
        self.table = None
        if P:
            self.n_pages = B * K * cols + 5
            self.table = r.permutation(self.n_pages)[:B * K * cols].reshape(B, K, cols).astype(np.int32)
            self.dims.update(page_rows=P, n_pages=self.n_pages)
        self.dims["L"] = self.Lcap

    def pages(self, own):
        t = np.full((self.n_pages, self.P) + own.shape[3:], NAN)
        t[self.table.reshape(-1)] = own.reshape(-1, self.P, *own.shape[3:])
        return t

    def device(self):
        up = lambda v: torch.tensor(v).to(ACT[self.dtype]).cuda()                               # noqa: E731
        i32 = lambda v: None if v is None else torch.tensor(np.asarray(v), dtype=torch.int32).cuda()   # noqa: E731
        own = (self.pages(self.ok), self.pages(self.ov)) if self.P else (self.ok, self.ov)
        self.keys = [up(self.q), up(self.ck), up(self.cv), up(own[0]), up(own[1])]
        self.more = dict(table=i32(self.table), ctx_len=i32(self.ctx_len), q_len=i32(self.q_len), own_len=i32(self.own_len))
        return self

    def reference(self, grad=False, seen=None):
        return ref.attend(self.q, self.ck, self.cv, self.ok, self.ov, dtype=self.dtype, causal=self.dims["causal"],
                          scale=self.dims["scale"], ctx_len=self.nc, q_len=self.nq, own_len=self.no,
                          dout=self.do if grad else None, seen=seen)


def _near(got, want, name):
    val, bound = want
    got = got.double().cpu().numpy()
    same = np.isneginf(val) & np.isneginf(got)
    with np.errstate(invalid="ignore"):
        err = np.where(same, 0.0, np.abs(got - val))
    bad = ~(err <= bound)
    assert not bad.any(), (name, int(bad.sum()), float(np.nanmax(err)), float(bound[bad].max()), np.argwhere(bad)[:3].tolist())


FORWARD = [
    # the smallest: one row, one key
    dict(dtype="bf16", B=1, K=1, S=1, H=1, Hkv=1, dh=32, T=1, L=0, lens="full"),
    dict(dtype="f32", B=1, K=1, S=1, H=1, Hkv=1, dh=32, T=0, L=1, lens="full"),
    dict(dtype="f32", B=1, K=1, S=1, H=1, Hkv=1, dh=64, T=0, L=0, lens="full"),
    # single tokens, dense and paged, odd pages, grouped heads
    dict(dtype="bf16", B=2, K=5, S=1, H=4, Hkv=4, dh=32, T=181, L=12),
    dict(dtype="bf16", B=2, K=16, S=1, H=8, Hkv=8, dh=64, T=200, L=64, P=16),
    dict(dtype="bf16", B=1, K=7, S=1, H=8, Hkv=2, dh=128, T=300, L=37, P=7),
    dict(dtype="f32", B=2, K=3, S=1, H=6, Hkv=2, dh=64, T=65, L=33, P=1),
    dict(dtype="bf16", B=1, K=70, S=1, H=2, Hkv=1, dh=32, T=31, L=150, P=64),
    # a few rows
    dict(dtype="bf16", B=2, K=4, S=5, H=4, Hkv=2, dh=64, T=130, L=40, P=16),
    dict(dtype="f32", B=3, K=6, S=7, H=6, Hkv=2, dh=64, T=77, L=23),
    dict(dtype="f32", B=1, K=3, S=3, H=2, Hkv=2, dh=128, T=129, L=65, P=5),
    # whole lists
    dict(dtype="bf16", B=3, K=9, S=11, H=4, Hkv=4, dh=32, T=100, L=11, causal=False, lens="full"),
    dict(dtype="bf16", B=2, K=3, S=64, H=2, Hkv=2, dh=64, T=96, L=64, lens="full"),
    dict(dtype="bf16", B=1, K=2, S=150, H=3, Hkv=1, dh=128, T=20, L=150, lens="own"),
    dict(dtype="f32", B=2, K=13, S=11, H=4, Hkv=4, dh=32, T=64, L=11, causal=False, lens="own"),
    # lengths at and past their limits, rows without keys
    dict(dtype="bf16", B=6, K=5, S=3, H=4, Hkv=2, dh=32, T=40, L=9, lens="edge"),
    dict(dtype="bf16", B=6, K=5, S=3, H=4, Hkv=2, dh=64, T=140, L=70, P=10, lens="edge", causal=False),
    dict(dtype="f32", B=6, K=7, S=4, H=2, Hkv=1, dh=32, T=33, L=20, lens="edge"),
    # sharp softmaxes: scores up to some hundreds
    dict(dtype="bf16", B=1, K=4, S=6, H=2, Hkv=2, dh=64, T=150, L=20, amp=6.0),
    dict(dtype="f32", B=1, K=4, S=6, H=2, Hkv=2, dh=64, T=150, L=20, amp=6.0, scale=0.3),
    dict(dtype="f32", B=1, K=4, S=6, H=2, Hkv=2, dh=32, T=50, L=20, scale=-0.4),
    # 65 to 128 rows of a key head, in one tile
    dict(dtype="bf16", B=2, K=25, S=1, H=8, Hkv=2, dh=128, T=150, L=40, P=8),
    dict(dtype="bf16", B=1, K=5, S=10, H=6, Hkv=3, dh=128, T=90, L=10, lens="own"),
    dict(dtype="bf16", B=2, K=11, S=2, H=8, Hkv=2, dh=64, T=70, L=33, P=4),
    dict(dtype="f32", B=2, K=7, S=5, H=6, Hkv=2, dh=32, T=70, L=21),
    dict(dtype="f32", B=1, K=16, S=1, H=8, Hkv=1, dh=64, T=200, L=30, P=30, lens="edge"),
    # many tiles of 128 rows
    dict(dtype="bf16", B=128, K=2, S=64, H=8, Hkv=4, dh=32, T=5, L=64, lens="own"),
    # one long list, causal, over several tiles and chunks; lists of different lengths in one tile
    dict(dtype="bf16", B=1, K=1, S=333, H=1, Hkv=1, dh=64, T=0, L=333, lens="full"),
    dict(dtype="f32", B=1, K=2, S=200, H=3, Hkv=1, dh=32, T=33, L=260),
    # groups of heads that no power of two divides
    dict(dtype="bf16", B=1, K=3, S=9, H=5, Hkv=1, dh=32, T=20, L=9, lens="own"),
    # equal weights
    dict(dtype="bf16", B=1, K=3, S=4, H=2, Hkv=2, dh=32, T=45, L=9, scale=0.0),
    # fp32 sums longer than one chain, with workgroups to spare
    dict(dtype="f32", B=8, K=1, S=1, H=8, Hkv=8, dh=32, T=4500, L=2, lens="full"),
    # few rows over many keys
    dict(dtype="bf16", B=1, K=2, S=1, H=2, Hkv=1, dh=64, T=5000, L=300, P=16),
    dict(dtype="f32", B=1, K=1, S=2, H=1, Hkv=1, dh=128, T=3001, L=3, lens="full"),
]


@pytest.mark.parametrize("i", range(len(FORWARD)))
def test_forward(i):
    kw = FORWARD[i]
    _say("forward", i, kw)
    c = Case(seed=i, **kw).device()
    p = fe.PrefixAttention(train=not c.P, **c.dims)
    out = p.run(*c.keys, **c.more)
    want = c.reference()
    _near(out, want["out"], "out")
    if not c.P:
        _near(p.lse, want["lse"], "lse")
    dead = torch.arange(c.dims["S"]) >= torch.tensor(c.nq)[..., None]
    assert torch.count_nonzero(out.cpu()[dead]) == 0
    again = p.run(*c.keys, **c.more).clone()
    assert torch.equal(again, out)                     # the same bits from call to call


# Long contexts whose key ranges follow the requests' lengths: eight requests, some of none and of all the rows; as many
# requests as share ranges that way, and one more
BY_LENGTH = [
    dict(dtype="bf16", B=8, K=3, S=2, H=8, Hkv=8, dh=32, T=12288, L=20, lens="edge", seed=3),
    dict(dtype="bf16", B=64, K=2, S=1, H=2, Hkv=1, dh=32, T=12288, L=70, P=16, seed=4),
    dict(dtype="bf16", B=65, K=2, S=1, H=1, Hkv=1, dh=32, T=12288, L=7, seed=5),
    dict(dtype="bf16", B=2, K=40, S=1, H=32, Hkv=16, dh=128, T=16384, L=30, seed=6),
]


@pytest.mark.parametrize("i", range(len(BY_LENGTH)))
def test_ranges_by_length(i):
    _say("by length", i, BY_LENGTH[i])
    c = Case(**BY_LENGTH[i]).device()
    p = fe.PrefixAttention(**c.dims)
    out = p.run(*c.keys, **c.more)
    _near(out, c.reference()["out"], "out")
    assert torch.equal(p.run(*c.keys, **c.more).clone(), out)


def test_ranges_by_length_in_a_graph():
    """A captured call replayed with other lengths: the ranges follow them, and every replay has the eager call's bits."""
    c = Case(**dict(BY_LENGTH[0], lens="full")).device()
    B, T = c.dims["B"], c.dims["T"]
    g = torch.Generator().manual_seed(9)
    lens = [torch.full((B,), T), torch.tensor([T] + [0] * (B - 1)), torch.randint(0, T + 1, (B,), generator=g)]
    lens = [n.to(torch.int32).cuda() for n in lens]
    more = dict(c.more, ctx_len=lens[0].clone())
    plan, other = fe.PrefixAttention(**c.dims), fe.PrefixAttention(**c.dims)
    eager = [plan.run(*c.keys, **dict(c.more, ctx_len=n)).clone() for n in lens]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = plan.run(*c.keys, **more)
    for i in (0, 1, 2, 1, 0):
        more["ctx_len"].copy_(lens[i])
        graph.replay()
        again = other.run(*c.keys, **dict(c.more, ctx_len=lens[i]))
        torch.cuda.synchronize()
        assert torch.equal(out, eager[i]) and torch.equal(again, eager[i]), i


GRAD = [
    dict(dtype="f32", B=1, K=1, S=1, H=1, Hkv=1, dh=32, T=1, L=1, lens="full"),
    dict(dtype="f32", B=1, K=2, S=3, H=2, Hkv=1, dh=32, T=0, L=3, lens="own"),
    dict(dtype="bf16", B=1, K=2, S=3, H=2, Hkv=1, dh=64, T=9, L=0, lens="full"),
    dict(dtype="f32", B=3, K=9, S=11, H=4, Hkv=4, dh=32, T=100, L=11, causal=False, lens="full"),
    dict(dtype="f32", B=2, K=5, S=6, H=6, Hkv=2, dh=64, T=77, L=23),
    dict(dtype="bf16", B=2, K=3, S=64, H=2, Hkv=2, dh=64, T=96, L=64, lens="full"),
    dict(dtype="bf16", B=2, K=9, S=37, H=4, Hkv=1, dh=128, T=133, L=37, lens="own"),
    dict(dtype="f32", B=1, K=3, S=20, H=2, Hkv=1, dh=128, T=70, L=20, lens="own"),
    dict(dtype="bf16", B=6, K=5, S=3, H=4, Hkv=2, dh=32, T=40, L=9, lens="edge"),
    dict(dtype="f32", B=6, K=7, S=4, H=2, Hkv=1, dh=32, T=33, L=20, lens="edge"),
    dict(dtype="bf16", B=1, K=2, S=1, H=2, Hkv=2, dh=64, T=700, L=90, causal=False),
    dict(dtype="bf16", B=1, K=40, S=5, H=4, Hkv=1, dh=32, T=65, L=5, causal=False, lens="own"),
    # one long list; own rows longer than the query rows; groups of 3 and 5; a negative scale; equal weights
    dict(dtype="bf16", B=1, K=1, S=200, H=2, Hkv=1, dh=64, T=10, L=200, lens="full"),
    dict(dtype="f32", B=1, K=2, S=30, H=3, Hkv=1, dh=32, T=20, L=150),
    dict(dtype="bf16", B=1, K=4, S=13, H=10, Hkv=2, dh=32, T=50, L=13, lens="own"),
    dict(dtype="f32", B=2, K=3, S=5, H=2, Hkv=2, dh=64, T=40, L=9, scale=-0.3),
    dict(dtype="f32", B=1, K=2, S=5, H=2, Hkv=2, dh=32, T=30, L=9, scale=0.0),
    # more rows than one fp32 chain
    dict(dtype="f32", B=1, K=60, S=20, H=2, Hkv=1, dh=32, T=70, L=20, causal=False, lens="own"),
    dict(dtype="bf16", B=2, K=30, S=20, H=4, Hkv=1, dh=128, T=20, L=20, lens="own"),
]
NAMES = ("dq", "dck", "dcv", "dok", "dov")


@pytest.mark.parametrize("i", range(len(GRAD)))
def test_grad(i):
    kw = GRAD[i]
    _say("grad", i, kw)
    c = Case(seed=100 + i, **kw).device()
    p = fe.PrefixAttention(train=True, **c.dims)
    out = p.run(*c.keys, **c.more)
    dout = torch.tensor(c.do).to(ACT[c.dtype]).cuda()
    grads = p.grad(dout, *c.keys, **c.more)
    want = c.reference(grad=True)
    _near(out, want["out"], "out")
    for name, g in zip(NAMES, grads):
        _near(g, want[name], name)
    first = [g.clone() for g in grads]
    for g in p.grad(dout, *c.keys, **c.more), :
        assert all(torch.equal(a, b) for a, b in zip(first, g))


def test_grad_without_the_rest_of_out():
    """Without out_rest the gradient takes dout . out from the rounded out (the bound covers both)."""
    c = Case(dtype="bf16", B=2, K=3, S=9, H=4, Hkv=2, dh=64, T=40, L=9, lens="own", seed=77).device()
    p = fe.PrefixAttention(train=True, **c.dims)
    p.run(*c.keys, **c.more)
    dout = torch.tensor(c.do).bfloat16().cuda()
    kept = [g.clone() for g in p.grad(dout, *c.keys, **c.more)]
    p.args.out_rest = None
    want = c.reference(grad=True)
    differs = False
    for name, g, k in zip(NAMES, p.grad(dout, *c.keys, **c.more), kept):
        _near(g, want[name], name)
        differs |= not torch.equal(g, k)
    assert differs


def test_two_calls_at_once():
    """Two objects on two streams, many calls in flight: each keeps its own outputs and workspace."""
    cases = [Case(dtype="bf16", B=1, K=4, S=1, H=4, Hkv=2, dh=64, T=3000, L=48, P=16, seed=s).device() for s in (41, 42)]
    plans = [fe.PrefixAttention(**c.dims) for c in cases]
    want = [p.run(*c.keys, **c.more).clone() for p, c in zip(plans, cases)]
    streams = [torch.cuda.Stream() for _ in plans]
    torch.cuda.synchronize()
    for _ in range(20):
        for p, c, s in zip(plans, cases, streams):
            p.run(*c.keys, stream=s, **c.more)
    torch.cuda.synchronize()
    assert all(torch.equal(p.out, w) for p, w in zip(plans, want))


def test_first_call_on_a_given_stream():
    """Outputs, workspace and q_out that a call allocates itself are good for the stream that it is given."""
    c = Case(dtype="bf16", B=1, K=4, S=1, H=4, Hkv=2, dh=64, T=3000, L=48, P=16, seed=43).device()
    want = fe.PrefixAttention(**c.dims).run(*c.keys, **c.more).clone()
    ac = AppendCase(seed=44, **APPEND[0])
    (k, v), kw = ac.device()
    for side in (torch.cuda.Stream(), torch.cuda.default_stream()):
        p = fe.PrefixAttention(**c.dims)
        torch.cuda.synchronize()
        got = p.run(*c.keys, stream=side, **c.more)
        side.synchronize()
        assert torch.equal(got, want)
    side = torch.cuda.Stream()
    q_out = ac.cache.append(k, v, stream=side, **kw)
    side.synchronize()
    ac.check(q_out)


def _busy():
    """Some milliseconds of work on the current stream."""
    a = torch.ones(4096, 4096, device="cuda")
    for _ in range(10):
        a = a @ a * 2.0 ** -12
    return a


def test_own_tensors_on_a_given_stream():
    """Lengths that the cache starts at zero itself, and outputs allocated ahead, while their own stream is still busy with what
    their memory held before."""
    ac = AppendCase(seed=45, **APPEND[0])
    (k, v), kw = ac.device()
    ac.len[:] = 0
    c = Case(dtype="bf16", B=1, K=4, S=1, H=4, Hkv=2, dh=64, T=3000, L=48, P=16, seed=46).device()
    want = fe.PrefixAttention(**c.dims).run(*c.keys, **c.more).clone()
    p = fe.PrefixAttention(**c.dims)
    before = [torch.empty(ac.len.shape, dtype=torch.int32, device="cuda") for _ in range(2)]
    old = [torch.empty_like(want), torch.empty(p.ws_bytes, dtype=torch.uint8, device="cuda")]
    torch.cuda.synchronize()
    kept = _busy()
    for t in before + old:
        t.fill_(77)
    del before, old
    ac.cache = fe.PagedCache(ac.cache.k_pages, ac.cache.v_pages, ac.cache.table)
    p.allocate()
    side = torch.cuda.Stream()
    q_out = ac.cache.append(k, v, stream=side, **kw)
    got = p.run(*c.keys, stream=side, **c.more)
    torch.cuda.synchronize()
    ac.check(q_out)
    assert torch.equal(got, want) and bool(torch.isfinite(kept).all())


def test_lists_do_not_depend_on_each_other():
    """The same list beside other lists of the same lengths: the same bits."""
    c = Case(dtype="bf16", B=1, K=12, S=7, H=4, Hkv=2, dh=64, T=100, L=15, seed=61).device()
    p = fe.PrefixAttention(**c.dims)
    want = p.run(*c.keys, **c.more).clone()
    other = [t.clone() for t in c.keys]
    keep = [0, 5, 11]
    for i in (0, 3, 4):                                  # queries, own keys, own values of the other lists
        new = torch.randn(other[i].shape, device="cuda").bfloat16() * 3
        new[:, keep] = other[i][:, keep]
        other[i] = new
    got = p.run(*other, **c.more)
    assert torch.equal(got[:, keep], want[:, keep])


def test_grad_matches_differences():
    """The kernel's gradients against central differences of the kernel's own forward, along random directions:
    the loss sum(out * dout) in float64; fp32 outputs are off by about 1e-6 relative, so a step of 2^-6 leaves the
    difference good to about 1e-4 plus its own third-order term of step^2."""
    kw = dict(dtype="f32", B=2, K=3, S=4, H=4, Hkv=2, dh=32, T=21, L=9)
    c = Case(seed=5, **kw).device()
    for t in c.keys:
        t.nan_to_num_(0.0)
    p = fe.PrefixAttention(train=True, **c.dims)
    dout = torch.tensor(np.nan_to_num(c.do)).float().cuda()
    p.run(*c.keys, **c.more)
    grads = [g.double() for g in p.grad(dout, *c.keys, **c.more)]
    gen_ = torch.Generator(device="cuda").manual_seed(1)
    for i, g in enumerate(grads):
        d = torch.randn(c.keys[i].shape, generator=gen_, device="cuda")
        d /= d.norm()
        f = []
        for step in (2.0 ** -6, -(2.0 ** -6)):
            keys = list(c.keys)
            keys[i] = keys[i] + step * d
            f.append(float((p.run(*keys, **c.more).double() * dout.double()).sum()))
        diff, want = (f[0] - f[1]) * 2.0 ** 5, float((g * d.double()).sum())
        assert abs(diff - want) <= 2e-3 * max(1.0, abs(want)), (NAMES[i], diff, want)


def test_gradients_handed_to_autograd():
    """Queries, keys and values that a model computed: run() returns no history, and the gradients go on into the model."""
    c = Case(dtype="f32", B=2, K=3, S=4, H=4, Hkv=2, dh=32, T=21, L=4, lens="full", seed=8).device()
    weights = [torch.full((32,), 0.5 + i, device="cuda", requires_grad=True) for i in range(5)]
    made = [x * w for x, w in zip(c.keys, weights)]
    p = fe.PrefixAttention(train=True, **c.dims)
    dout = torch.tensor(c.do).float().cuda()
    assert not p.run(*made, **c.more).requires_grad
    grads = p.grad(dout, *made, **c.more)
    torch.autograd.backward(made, grads)
    for w, x, g in zip(weights, c.keys, grads):
        want, size = ((x * g).double().flatten(0, -2).sum(0), (x * g).double().abs().flatten(0, -2).sum(0))
        n = x.numel() // 32                              # fp32 sums of n products, in an order of torch's
        assert ((w.grad.double() - want).abs() <= (n + 1) * 2.0 ** -24 * size).all()


def test_strided_inputs():
    """Queries as a column block of a fused projection, the shared rows as one layer of a context cache."""
    c = Case(dtype="bf16", B=2, K=3, S=4, H=4, Hkv=2, dh=32, T=50, L=10, seed=7).device()
    want = fe.PrefixAttention(**c.dims).run(*c.keys, **c.more).clone()
    q, ck, cv, ok, ov = c.keys
    wide = torch.full((2, 3, 4, 11, 32), NAN, dtype=torch.bfloat16, device="cuda")
    wide[:, :, :, 3:7] = q
    cache = torch.full((3, 2, 2, 50, 2, 32), NAN, dtype=torch.bfloat16, device="cuda")       # [layer][key, value][B][T][..]
    cache[1, 0], cache[1, 1] = ck, cv
    own = torch.full((2, 3, 10, 7, 32), NAN, dtype=torch.bfloat16, device="cuda")
    own[..., 1:3, :], own[..., 4:6, :] = ok, ov
    got = fe.PrefixAttention(**c.dims).run(wide[:, :, :, 3:7], cache[1, 0], cache[1, 1], own[..., 1:3, :], own[..., 4:6, :], **c.more)
    assert torch.equal(got, want)
    wide = torch.full((2, 3, 4, 11, 32), NAN, dtype=torch.bfloat16, device="cuda")
    wide[:, :, :, 2:6] = torch.tensor(c.do).bfloat16().cuda()
    p = fe.PrefixAttention(train=True, **c.dims)
    p.run(*c.keys, **c.more)
    a = [g.clone() for g in p.grad(wide[:, :, :, 2:6].contiguous(), *c.keys, **c.more)]
    assert all(torch.equal(x, y) for x, y in zip(a, p.grad(wide[:, :, :, 2:6], *c.keys, **c.more)))


def test_pages_outside_the_pool_do_not_count():
    c = Case(dtype="bf16", B=2, K=4, S=2, H=2, Hkv=2, dh=64, T=20, L=40, P=8, lens="full", causal=False, seed=9)
    seen = np.ones((2, 4, 40), bool)
    good = c.table.copy()
    for b, k, col, page in ((0, 0, 0, -1), (0, 1, 4, c.n_pages), (1, 2, 2, 2 ** 31 - 1), (1, 3, 1, -2 ** 31)):
        c.table[b, k, col] = page
        seen[b, k, col * 8:col * 8 + 8] = False
    bad, c.table = c.table, good
    c.device()
    c.more["table"] = torch.tensor(bad).cuda()
    _near(fe.PrefixAttention(**c.dims).run(*c.keys, **c.more), c.reference(seen=seen)["out"], "out")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_list_keeps_its_infinities_to_itself(dtype):
    """Infinite and NaN values of one list, and of own rows that a causal row does not see yet, reach only the rows
    that see them."""
    c = Case(dtype=dtype, B=1, K=6, S=5, H=2, Hkv=1, dh=32, T=30, L=5, lens="full", seed=11).device()
    p = fe.PrefixAttention(**c.dims)
    want = p.run(*c.keys, **c.more).clone()
    c.keys[4][0, 2, 3, 0, 7] = float("inf")
    c.keys[4][0, 4, 1, 0, 0] = NAN
    c.keys[3][0, 5, 2, 0, 1] = NAN
    got = p.run(*c.keys, **c.more)
    hit = torch.zeros_like(want, dtype=torch.bool)
    hit[0, 2, 3:, :, 7] = True
    hit[0, 4, 1:, :, 0] = True
    hit[0, 5, 2:] = True
    assert torch.isinf(got[0, 2, 3:, :, 7]).all() and torch.isnan(got[0, 4, 1:, :, 0]).all() and torch.isnan(got[0, 5, 2:]).all()
    # the same rows summed in another order: two roundings of the type and of a sum of 35 fp32 terms of size at most 4
    tol = 2 * ref.HALF_STEP[dtype] * want.abs().float() + 35 * 2.0 ** -24 * 4
    assert (((got - want).abs().float() <= tol) | hit).all()


@pytest.mark.parametrize("kw", [
    dict(dtype="bf16"), dict(dtype="bf16", train=True), dict(dtype="bf16", T=300, train=True), dict(dtype="bf16", P=2, dh=64),
    dict(dtype="f32"), dict(dtype="f32", dh=64, P=2), dict(dtype="bf16", dh=128, train=True)])
def test_infinities_leave_the_neighbours_bits(kw):
    """Infinite and NaN own values of some lists: every output that sees none of them keeps its bits, and what out's rounding
    cut as well."""
    kw = dict(dict(T=30, dh=32, train=False), **kw)
    train = kw.pop("train")
    c = Case(B=1, K=9, S=5, H=2, Hkv=1, L=6, lens="full", seed=14, **kw).device()
    p = fe.PrefixAttention(train=train, **c.dims)
    want = p.run(*c.keys, **c.more).clone()
    rest = p.out_rest.clone() if p.out_rest is not None else None
    hit = torch.zeros(want.shape, dtype=torch.bool, device="cuda")
    for k, j, col, value in ((2, 3, 7, INF), (4, 2, 0, NAN), (6, 0, 31, -INF), (6, 5, 8, INF)):
        if c.P:
            c.keys[4][int(c.table[0, k, j // c.P]), j % c.P, 0, col] = value
        else:
            c.keys[4][0, k, j, 0, col] = value
        hit[0, k, max(0, j - 1):, :, col] = True            # causal: row i sees j <= i + 1
    got = p.run(*c.keys, **c.more)
    assert (got[0, 2, 2:, :, 7] == INF).all() and torch.isnan(got[0, 4, 1:, :, 0]).all()
    assert (got[0, 6, :, :, 31] == -INF).all() and (got[0, 6, 4:, :, 8] == INF).all()
    assert torch.equal(got[~hit], want[~hit])
    assert rest is None or torch.equal(p.out_rest[~hit], rest[~hit])


@pytest.mark.parametrize("dh,T,train", [(32, 70, False), (32, 70, True), (64, 70, True), (128, 200, True), (32, 400, True)])
def test_infinite_shared_values(dh, T, train):
    """bf16: an infinite shared value makes its column infinite in every row of its request, and nothing else."""
    c = Case(dtype="bf16", B=2, K=4, S=6, H=2, Hkv=2, dh=dh, T=T, L=6, lens="full", seed=15).device()
    p = fe.PrefixAttention(train=train, **c.dims)
    want = p.run(*c.keys, **c.more).clone()
    c.keys[2][1, T - 4, 1, 5] = INF
    c.keys[2][1, 3, 0, 9] = -INF
    c.keys[2][1, 35, 0, 31] = NAN
    got = p.run(*c.keys, **c.more)
    hit = torch.zeros(want.shape, dtype=torch.bool, device="cuda")
    hit[1, :, :, 1, 5] = hit[1, :, :, 0, 9] = hit[1, :, :, 0, 31] = True
    assert (got[1, :, :, 1, 5] == INF).all() and (got[1, :, :, 0, 9] == -INF).all() and torch.isnan(got[1, :, :, 0, 31]).all()
    assert torch.equal(got[~hit], want[~hit])


@pytest.mark.parametrize("dh,T,train", [(32, 70, False), (32, 70, True), (64, 70, True), (128, 200, True), (32, 400, True)])
def test_infinite_shared_values(dh, T, train):
    """bf16: an infinite shared value makes its column infinite in every row of its request, and nothing else."""
    c = Case(dtype="bf16", B=2, K=4, S=6, H=2, Hkv=2, dh=dh, T=T, L=6, lens="full", seed=15).device()
    p = fe.PrefixAttention(train=train, **c.dims)
    want = p.run(*c.keys, **c.more).clone()
    c.keys[2][1, T - 4, 1, 5] = INF
    c.keys[2][1, 3, 0, 9] = -INF
    c.keys[2][1, 35, 0, 31] = NAN
    got = p.run(*c.keys, **c.more)
    hit = torch.zeros(want.shape, dtype=torch.bool, device="cuda")
    hit[1, :, :, 1, 5] = hit[1, :, :, 0, 9] = hit[1, :, :, 0, 31] = True
    assert (got[1, :, :, 1, 5] == INF).all() and (got[1, :, :, 0, 9] == -INF).all() and torch.isnan(got[1, :, :, 0, 31]).all()
    assert torch.equal(got[~hit], want[~hit])


@pytest.mark.parametrize("payload", [0x7f800001, -0x7fffff, 0x7fc00000])
@pytest.mark.parametrize("which", range(5))
def test_a_nan_of_any_payload_gives_nan(which, payload):
    """fp32: a NaN whose first sixteen bits are those of an infinity is a NaN in every output that sees it."""
    c = Case(dtype="f32", B=1, K=3, S=4, H=2, Hkv=2, dh=32, T=40, L=6, lens="full", causal=False, seed=16).device()
    p = fe.PrefixAttention(train=True, **c.dims)
    want = p.run(*c.keys, **c.more).clone()
    at = ((0, 1, 2, 1, 3), (0, 17, 1, 3), (0, 17, 1, 3), (0, 1, 5, 1, 3), (0, 1, 5, 1, 3))[which]
    c.keys[which].view(torch.int32)[at] = payload
    assert torch.isnan(c.keys[which][at])
    got = p.run(*c.keys, **c.more)
    hit = torch.zeros(want.shape, dtype=torch.bool, device="cuda")
    hit[((0, 1, 2, 1), (0, slice(None), slice(None), 1), (0, slice(None), slice(None), 1, 3), (0, 1, slice(None), 1),
         (0, 1, slice(None), 1, 3))[which]] = True
    assert torch.isnan(got[hit]).all()
    assert torch.equal(got[~hit], want[~hit])


@pytest.mark.parametrize("T", [40, 3000])                # whole, and in ranges that are joined
def test_a_nan_query_gives_nan(T):
    """A row whose scores are all NaN is not a row without keys; the other rows keep their bits."""
    c = Case(dtype="bf16", B=1, K=3, S=2, H=2, Hkv=2, dh=32, T=T, L=6, lens="full", seed=13).device()
    p = fe.PrefixAttention(train=True, **c.dims)
    want, lse = p.run(*c.keys, **c.more).clone(), p.lse.clone()
    c.keys[0][0, 1, 0, 1, 3] = NAN
    got = p.run(*c.keys, **c.more)
    hit = torch.zeros(want.shape[:4], dtype=torch.bool)
    hit[0, 1, 0, 1] = True
    assert torch.isnan(got[hit.cuda()]).all() and torch.isnan(p.lse[hit.cuda()]).all()
    assert torch.equal(got[~hit.cuda()], want[~hit.cuda()]) and torch.equal(p.lse[~hit.cuda()], lse[~hit.cuda()])


def test_streams_and_graphs():
    """On a stream of its own; captured once and replayed with other lengths, queries and pages, eager work in between."""
    cases = [Case(dtype="bf16", B=2, K=4, S=1, H=4, Hkv=2, dh=64, T=900, L=48, P=16, seed=s).device() for s in (21, 22, 23)]
    eager = [fe.PrefixAttention(**c.dims).run(*c.keys, **c.more).clone() for c in cases]
    st = torch.cuda.Stream()
    p = fe.PrefixAttention(**cases[0].dims)
    p.allocate()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        on_stream = p.run(*cases[0].keys, **cases[0].more).clone()
    st.synchronize()
    assert torch.equal(on_stream, eager[0])
    keys = [t.clone() for t in cases[0].keys]
    more = {n: None if t is None else t.clone() for n, t in cases[0].more.items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = p.run(*keys, **more)
    for i in (0, 1, 2, 1, 0):
        for dst, src in zip(keys, cases[i].keys):
            dst.copy_(src)
        for n, dst in more.items():
            dst.copy_(cases[i].more[n])
        graph.replay()
        other = fe.PrefixAttention(**cases[i].dims).run(*cases[i].keys, **cases[i].more)
        torch.cuda.synchronize()
        assert torch.equal(out, eager[i]) and torch.equal(other, eager[i]), i


def test_grad_in_a_graph():
    c = Case(dtype="bf16", B=2, K=3, S=9, H=4, Hkv=2, dh=64, T=70, L=9, lens="own", seed=31).device()
    dout = torch.tensor(c.do).bfloat16().cuda()
    p = fe.PrefixAttention(train=True, **c.dims)
    p.run(*c.keys, **c.more)
    want = [g.clone() for g in p.grad(dout, *c.keys, **c.more)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.run(*c.keys, **c.more)
        grads = p.grad(dout, *c.keys, **c.more)
    for _ in range(3):
        for g in grads:
            g.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, grads))


def _forward_cases():
    return [dict(seed=i, **kw) for i, kw in enumerate(FORWARD)] + BY_LENGTH


@pytest.mark.parametrize("i", range(len(FORWARD) + len(BY_LENGTH)))
def test_forward_repeats_itself(i):
    """The same bits from a second call, whatever the outputs and the workspace held before it."""
    kw = _forward_cases()[i]
    _say("repeats", i, kw)
    c = Case(**kw).device()
    p = fe.PrefixAttention(train=not c.P, **c.dims)
    first = p.run(*c.keys, **c.more).clone()
    lse = None if c.P else p.lse.clone()
    p.ws.fill_(255)                                     # as floats: NaN
    p.out.fill_(NAN)
    if lse is not None:
        p.lse.fill_(NAN)
    p.run(*c.keys, **c.more)
    assert torch.equal(p.out, first)
    assert lse is None or torch.equal(p.lse, lse)


def test_two_calls_at_once_write_their_outputs():
    """Two objects on two streams, many calls in flight, over outputs that hold something else before."""
    cases = [Case(dtype="bf16", B=1, K=4, S=1, H=4, Hkv=2, dh=64, T=3000, L=48, P=16, seed=s).device() for s in (41, 42)]
    plans = [fe.PrefixAttention(**c.dims) for c in cases]
    want = [p.run(*c.keys, **c.more).clone() for p, c in zip(plans, cases)]
    streams = [torch.cuda.Stream() for _ in plans]
    for p in plans:
        p.out.fill_(NAN)
        p.ws.fill_(255)
    torch.cuda.synchronize()
    for _ in range(20):
        for p, c, s in zip(plans, cases, streams):
            p.run(*c.keys, stream=s, **c.more)
    torch.cuda.synchronize()
    assert all(torch.equal(p.out, w) for p, w in zip(plans, want))


# Where the header says 16 bits: up to 256 keys, and the own keys' gradients over more
PRECISE = [
    dict(dtype="bf16", B=2, K=3, S=11, H=4, Hkv=2, dh=64, T=60, L=20, amp=0.5),
    dict(dtype="bf16", B=1, K=7, S=5, H=4, Hkv=4, dh=32, T=200, L=56, causal=False),
    dict(dtype="bf16", B=1, K=2, S=40, H=2, Hkv=1, dh=128, T=9, L=40, lens="own"),
    dict(dtype="bf16", B=1, K=3, S=30, H=2, Hkv=2, dh=64, T=400, L=30, lens="own"),
    dict(dtype="bf16", B=1, K=64, S=1, H=1, Hkv=1, dh=32, T=0, L=3, causal=False, lens="full"),
]


@pytest.mark.parametrize("i", range(len(PRECISE)))
def test_second_products(i):
    """bf16 with out_rest: over at most 256 keys the probabilities of out have 16 bits, D is that of out with its rest, and
    own keys' gradients take p and ds at 16 bits.  The plain roundings lie outside these bounds
    (tests/test_prefix_host.py: test_precise_bounds_tell_the_roundings_apart)."""
    kw = PRECISE[i]
    _say("precise", i, kw)
    c = Case(seed=200 + i, **kw).device()
    p = fe.PrefixAttention(train=True, **c.dims)
    out = p.run(*c.keys, **c.more)
    dout = torch.tensor(c.do).bfloat16().cuda()
    grads = p.grad(dout, *c.keys, **c.more)
    want = ref.attend(c.q, c.ck, c.cv, c.ok, c.ov, dtype="bf16", causal=c.dims["causal"], ctx_len=c.nc, q_len=c.nq,
                      own_len=c.no, dout=c.do, up_out=ref.TWO_PARTS if c.dims["T"] + c.L <= 256 else None,
                      up_own=ref.TWO_PARTS, u_rest=ref.REST)
    _near(out, want["out"], "out")
    for name, g in zip(NAMES, grads):
        _near(g, want[name], name)


# -- the cache -----------------------------------------------------------------------------------

APPEND = [
    dict(dtype="bf16", N=1, S=1, H=1, Hkv=1, dh=32, rot=32, P=1, cols=1),
    dict(dtype="bf16", N=9, S=1, H=8, Hkv=8, dh=64, rot=64, P=16, cols=4),
    dict(dtype="f32", N=5, S=9, H=6, Hkv=2, dh=64, rot=48, P=7, cols=5, near=True),
    dict(dtype="bf16", N=4, S=33, H=0, Hkv=2, dh=128, rot=128, P=5, cols=20),
    dict(dtype="f32", N=3, S=70, H=4, Hkv=1, dh=32, rot=0, P=64, cols=3),
    dict(dtype="bf16", N=3, S=150, H=4, Hkv=4, dh=128, rot=16, P=16, cols=20, near=True),
    dict(dtype="f32", N=2, S=200, H=1, Hkv=1, dh=32, rot=32, P=3, cols=100),
]


class AppendCase:
    def __init__(self, dtype, N, S, H, Hkv, dh, rot, P, cols, near=False, seed=0, far=False):
        r = np.random.default_rng(seed)
        dt = ACT[dtype]
        self.dtype, self.near = dtype, near
        rnd = lambda *s: torch.tensor(r.standard_normal(s)).to(dt).double().numpy()             # noqa: E731
        self.k, self.v = rnd(N, S, Hkv, dh), rnd(N, S, Hkv, dh)
        self.q = rnd(N, S, H, dh) if H else None
        pages = N * cols + 3
        self.kp, self.vp = rnd(pages, P, Hkv, dh), rnd(pages, P, Hkv, dh)
        self.table = r.permutation(pages)[:N * cols].reshape(N, cols).astype(np.int32)
        self.len = r.integers(0, max(1, cols * P - S + 1), N)
        self.new = r.integers(0, S + 1, N)
        self.new[0], self.len[0] = S, max(0, cols * P - S)          # one that fills its last page
        self.pos0 = r.integers(0, 2 ** 31 - 1, N) if far else r.integers(0, 5000, N)
        self.freq = 10000.0 ** (-np.arange(rot // 2) / max(1, rot // 2))

    def device(self):
        up = lambda v: None if v is None else torch.tensor(v).to(ACT[self.dtype]).cuda()        # noqa: E731
        i32 = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32).cuda()                   # noqa: E731
        self.cache = fe.PagedCache(up(self.kp), up(self.vp), i32(self.table), i32(self.len))
        return (up(self.k), up(self.v)), dict(q=up(self.q), new_len=i32(self.new), pos0=i32(self.pos0), neighbours=self.near,
                                              freq=torch.tensor(self.freq).cuda() if len(self.freq) else None)

    def check(self, got_q):
        kp, vp, qo, st = ref.append(self.k, self.v, self.q, self.kp, self.vp, self.table, self.len, self.new, self.pos0,
                                    self.freq, self.near)
        c, down = self.cache, lambda t: t.double().cpu().numpy()
        assert np.array_equal(down(c.v_pages), vp)
        wrote = (vp != self.vp).any(-1, keepdims=True)              # rows that were not written keep their bits
        err = np.abs(down(c.k_pages) - kp)
        # a turned pair's size is that of its pair before the turn: |a| + |b| <= sqrt(2) times the turned one's norm, itself <= the sum
        bound = 1.5 * ref.turned_bound(kp, self.freq, self.near, self.dtype)
        assert (err <= np.where(wrote, bound, 0.0)).all(), float(err.max())
        if self.q is not None:
            left = np.isnan(qo)
            err = np.abs(down(got_q) - qo)
            assert ((err <= ref.turned_bound(self.q, self.freq, self.near, self.dtype)) | left).all()
        assert np.array_equal(c.status.cpu().numpy(), st)
        assert np.array_equal(c.len.cpu().numpy(), np.maximum(self.len, 0) + np.clip(self.new, 0, self.k.shape[1]))
        return qo


@pytest.mark.parametrize("i", range(len(APPEND)))
def test_append(i):
    _say("append", i, APPEND[i])
    c = AppendCase(seed=i, **APPEND[i])
    (k, v), kw = c.device()
    q_out = None if c.q is None else torch.full_like(kw["q"], 5.0)
    got = c.cache.append(k, v, q_out=q_out, **kw)
    qo = c.check(got)
    if qo is not None:                                  # query rows past the new ones are left as they were
        assert (got.double().cpu().numpy()[np.isnan(qo)] == 5.0).all()


def test_append_far_positions():
    """Positions up to 2^31 keep their angles: each is formed and reduced in fp64."""
    c = AppendCase(dtype="f32", N=7, S=5, H=2, Hkv=1, dh=64, rot=64, P=4, cols=6, seed=50, far=True)
    (k, v), kw = c.device()
    c.check(c.cache.append(k, v, **kw))


def test_append_queries_in_place_and_fused():
    """Queries, keys and values as column blocks of one projection, the queries turned in place."""
    c = AppendCase(dtype="bf16", N=4, S=3, H=4, Hkv=2, dh=32, rot=32, P=8, cols=2, seed=51)
    (k, v), kw = c.device()
    fused = torch.cat((kw["q"], k, v), 2)
    q = fused[:, :, :4]
    got = c.cache.append(fused[:, :, 4:6], fused[:, :, 6:], **{**kw, "q": q, "q_out": q})
    c.check(got)
    assert torch.equal(fused[:, :, 4:6], k) and torch.equal(fused[:, :, 6:], v)


def test_append_refuses_rows_without_pages():
    """Past the table, bad pages, negative lengths: the cache keeps what it held there, status says so."""
    c = AppendCase(dtype="f32", N=6, S=10, H=2, Hkv=2, dh=32, rot=32, P=4, cols=5, seed=52)
    c.len[:] = (0, 15, 25, -9, 3, 2 ** 31 - 1)
    c.new[:] = (10, 10, 4, 10, 0, 0)
    c.table[0, 1], c.table[3, 2] = -1, 1 << 30
    c.table[4, :] = -5                                   # no new rows: its pages are not looked at
    (k, v), kw = c.device()
    c.check(c.cache.append(k, v, **kw))
    assert c.cache.status.tolist() == [fe.FE_DEV_BAD_PAGE] * 4 + [0, 0]


def test_append_lengths_beside():
    """len_out beside len leaves len alone; without new_len every row is new; a second call repeats the first."""
    c = AppendCase(dtype="bf16", N=3, S=40, H=4, Hkv=4, dh=64, rot=64, P=16, cols=4, seed=53)
    c.new[:] = 40
    (k, v), kw = c.device()
    kw["new_len"] = None
    after = torch.zeros(3, dtype=torch.int32, device="cuda")
    for _ in range(2):
        got = c.cache.append(k, v, len_out=after, **kw)
        assert c.cache.len.tolist() == c.len.tolist()
        assert after.tolist() == (c.len + 40).tolist()
    c.cache.len.copy_(after)
    c.check(got)


def test_append_in_a_graph():
    """A captured step appends one row per replay, the lengths advancing on the device."""
    c = AppendCase(dtype="bf16", N=5, S=1, H=2, Hkv=2, dh=32, rot=32, P=4, cols=3, seed=54)
    c.len[:] = (0, 1, 2, 3, 4)
    (k, v), kw = c.device()
    kw["new_len"] = None
    q_out = torch.empty_like(kw["q"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.cache.append(k, v, q_out=q_out, **kw)
    kp, vp = c.kp, c.vp
    for step in range(5):
        kn, vn, qn = (torch.randn(t.shape, device="cuda").bfloat16() for t in (k, v, kw["q"]))
        k.copy_(kn), v.copy_(vn), kw["q"].copy_(qn)
        graph.replay()
        torch.cuda.synchronize()
        c.k, c.v, c.q = (t.double().cpu().numpy() for t in (kn, vn, qn))
        c.new = np.ones(5, int)
        c.kp, c.vp = kp, vp
        c.check(q_out)
        kp, vp = c.cache.k_pages.double().cpu().numpy(), c.cache.v_pages.double().cpu().numpy()
        c.len = c.len + 1


def test_offsets_past_32_bits():
    """A pool of pages of more than 2^31 elements: rows at its end are written and read there."""
    P, hkv, dh = 64, 8, 128
    pages = (1 << 31) // (P * hkv * dh) + 40
    kp = torch.zeros(pages, P, hkv, dh, dtype=torch.bfloat16, device="cuda")
    vp = torch.zeros_like(kp)
    table = torch.tensor([[pages - 1, 5], [3, pages - 2]], dtype=torch.int32, device="cuda")
    cache = fe.PagedCache(kp, vp, table)
    g = torch.Generator(device="cuda").manual_seed(3)
    k, v = (torch.randn(2, 100, hkv, dh, generator=g, device="cuda").bfloat16() for _ in range(2))
    cache.append(k, v)
    assert torch.equal(kp[pages - 1], k[0, :64]) and torch.equal(vp[pages - 2, :36], v[1, 64:])
    q = torch.randn(1, 2, 1, 16, dh, generator=g, device="cuda").bfloat16()
    dims = dict(B=1, K=2, S=1, T=0, n_heads=16, n_kv_heads=hkv, dh=dh, dtype="bf16", causal=True)
    empty = torch.empty(1, 0, hkv, dh, dtype=torch.bfloat16, device="cuda")
    got = fe.PrefixAttention(L=128, page_rows=P, n_pages=pages, **dims).run(q, empty, empty, kp, vp, table=table.view(1, 2, 2),
                                                                         own_len=cache.len.view(1, 2)).clone()
    want = ref.attend(*(t.double().cpu().numpy() for t in (q, empty, empty, k[None], v[None])), dtype="bf16", causal=True)
    _near(got, want["out"], "out")


# -- together ------------------------------------------------------------------------------------

def test_lists_grow_over_an_encoded_context():
    """The calls as a program uses them: a request's context encoded once, its lists grown token by token through
    a paged cache, each step attending to the context's cache and the list so far; the same lists scored whole."""
    c = gen.config(1, B=2, K=3, T=70)
    W = gen.make_weights(c)
    I = gen.make_inputs(c)
    ev = make_evaluator(c, W)
    d = upload(c, I)
    b = ev.allocate(2, 70, c.M, 3, c.L)
    fe.fe_encode_context(ev.handle, 2, 70, d["x"], d["ctx_ids"], b["kv"], b["ws"])
    H, dh, steps, B, K = c.n_heads, c.dh, 5, 2, 3
    kv = b["kv"][1].view(2, B, 70, H, dh)               # the second item layer's keys and values
    g = torch.Generator(device="cuda").manual_seed(4)
    q, k, v = (torch.randn(B * K, steps, H, dh, generator=g, device="cuda").bfloat16() for _ in range(3))
    P, cols = 4, 2
    kp, vp = (torch.full((B * K * cols, P, H, dh), NAN, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.randperm(B * K * cols, generator=g, device="cuda").int().view(B * K, cols)
    cache = fe.PagedCache(kp, vp, table)
    freq = torch.tensor(100.0 ** -(np.arange(dh // 2) / (dh // 2))).cuda()
    pos0 = torch.full((B * K,), 70, dtype=torch.int32, device="cuda")
    step = fe.PrefixAttention(B=B, K=K, S=1, T=70, L=P * cols, n_heads=H, n_kv_heads=H, dh=dh, dtype="bf16", causal=True,
                              page_rows=P, n_pages=B * K * cols)
    outs = []
    for t in range(steps):
        qt = cache.append(k[:, t:t + 1], v[:, t:t + 1], q=q[:, t:t + 1], pos0=pos0, freq=freq)
        outs.append(step.run(qt.view(B, K, 1, H, dh), kv[0], kv[1], kp, vp, table=table.view(B, K, cols), own_len=cache.len).clone())
    got = torch.cat(outs, 2)
    assert cache.status.tolist() == [0] * 6 and cache.len.tolist() == [steps] * 6

    # the reference starts from the turned rows as the cache holds them (turning has its own tests)
    own = [p[table.long()].flatten(1, 2)[:, :steps].reshape(B, K, steps, H, dh) for p in (kp, vp)]
    qr = torch.tensor(ref.turned(q.double().cpu().numpy(), 70.0 + np.arange(steps)[None].repeat(B * K, 0), freq.cpu().numpy(), False)).bfloat16()
    ctx = kv.double().cpu().numpy()
    want = ref.attend(qr.double().numpy().reshape(B, K, steps, H, dh), ctx[0], ctx[1], *(o.double().cpu().numpy() for o in own),
                      dtype="bf16", causal=True)
    val, bound = want["out"]
    # a query that the two sides round to neighbouring bf16 values moves a score by at most 2^-7 |q||k| over its dh columns;
    # probabilities of scores that near move by twice that
    kmax = max(float(np.abs(ctx[0]).max()), float(own[0].abs().max()))
    vmax = max(float(np.abs(ctx[1]).max()), float(own[1].abs().max()))
    extra = 2 * 2.0 ** -7 * float(qr.abs().max()) * kmax * 2 * dh ** -0.5 * vmax
    _near(got, (val, bound + extra), "steps")

    qt, kt = (torch.stack([x.view(B * K, steps, H, dh)[:, t] for t in range(steps)], 1) for x in (qr.cuda().view(B * K, steps, H, dh), own[0]))
    whole = fe.PrefixAttention(B=B, K=K, S=steps, T=70, L=steps, n_heads=H, n_kv_heads=H, dh=dh, dtype="bf16", causal=True)
    _near(whole.run(qt.view(B, K, steps, H, dh), kv[0], kv[1], kt.view(B, K, steps, H, dh), own[1].contiguous()), want["out"], "whole")
    ev.close()

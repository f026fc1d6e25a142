"""Shared-prefix attention and paged-cache append without a GPU: the argument checks of the C calls and the
binding, workspace sizes, and the float64 reference that the GPU tests compare with."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2603_02565_amd import flasheval as fe
from tests import prefix_reference as ref

A16 = 4096          # a placeholder address: every call below is refused before anything touches it


def _args(**kw):
    a = fe.fe_prefix_args()
    base = dict(dtype=fe.FE_BF16, B=2, K=3, S=2, n_heads=4, n_kv_heads=2, dh=64, T=10, L=8, page_rows=0, n_pages=0,
                causal=1, scale=0.125, q_ld=256, ctx_ld=128, own_ld=128, out_ld=256, q=A16, ctx_k=A16, ctx_v=A16,
                own_k=A16, own_v=A16, table=None, ctx_len=None, q_len=None, own_len=None, out=A16, lse=A16, ws=A16,
                ws_bytes=1 << 30)
    for k, v in {**base, **kw}.items():
        setattr(a, k, v)
    return a


BAD_SIZES = [
    (dict(dtype=2), fe.FE_EINVAL), (dict(B=0), fe.FE_EINVAL), (dict(K=0), fe.FE_EINVAL), (dict(S=0), fe.FE_EINVAL),
    (dict(T=-1), fe.FE_EINVAL), (dict(L=-1), fe.FE_EINVAL), (dict(n_heads=3), fe.FE_EINVAL), (dict(n_kv_heads=0), fe.FE_EINVAL),
    (dict(dh=48), fe.FE_EUNSUPPORTED), (dict(dh=256), fe.FE_EUNSUPPORTED), (dict(page_rows=3, n_pages=4), fe.FE_EINVAL),
    (dict(page_rows=4, n_pages=0), fe.FE_EINVAL), (dict(page_rows=-1), fe.FE_EINVAL), (dict(T=(1 << 22) + 1), fe.FE_EUNSUPPORTED),
    (dict(L=1 << 23), fe.FE_EUNSUPPORTED), (dict(B=1 << 20, K=1 << 10), fe.FE_EUNSUPPORTED),
    (dict(B=1 << 16, T=1 << 15), fe.FE_EUNSUPPORTED), (dict(B=1 << 24, K=1, S=1, T=1, L=1), fe.FE_EUNSUPPORTED),
]
BAD_CALLS = [
    (dict(scale=float("nan")), "scale"), (dict(scale=float("inf")), "scale"), (dict(q=None), "NULL"), (dict(out=None), "NULL"),
    (dict(ctx_k=None), "ctx"), (dict(own_v=None), "own"), (dict(q=A16 + 8), "aligned"), (dict(own_k=A16 + 4), "aligned"),
    (dict(q_len=A16 + 2), "aligned"), (dict(q_ld=192), "stride"), (dict(q_ld=260), "stride"), (dict(ctx_ld=64), "stride"),
    (dict(own_ld=129), "stride"), (dict(out_ld=8), "stride"), (dict(page_rows=4, n_pages=4), "table"),
]


@pytest.mark.parametrize("kw,status", BAD_SIZES)
def test_prefix_sizes_are_checked(kw, status):
    lib, n = fe.load_library(), ctypes.c_size_t()
    a = _args(**kw)
    assert lib.fe_prefix_workspace_size(ctypes.byref(a), 0, ctypes.byref(n)) == status
    assert lib.fe_prefix_attention(ctypes.byref(a), None) == status
    assert lib.fe_prefix_attention_grad(ctypes.byref(a), None, None) == status
    assert lib.fe_last_error()


@pytest.mark.parametrize("kw,word", BAD_CALLS)
def test_prefix_calls_are_checked(kw, word):
    lib, a, g = fe.load_library(), _args(**kw), fe.fe_prefix_grads()
    assert lib.fe_prefix_attention(ctypes.byref(a), None) == fe.FE_EINVAL
    assert word in lib.fe_last_error().decode()
    assert lib.fe_prefix_attention_grad(ctypes.byref(a), ctypes.byref(g), None) == fe.FE_EINVAL


def _grads(**kw):
    g = fe.fe_prefix_grads()
    base = dict(dout=A16, dout_ld=256, dq_ld=256, dctx_ld=128, down_ld=128, dq=A16, dctx_k=A16, dctx_v=A16, down_k=A16, down_v=A16)
    for k, v in {**base, **kw}.items():
        setattr(g, k, v)
    return g


@pytest.mark.parametrize("kw,gkw,status", [
    ({}, dict(dout=None), fe.FE_EINVAL), ({}, dict(dq=None), fe.FE_EINVAL), ({}, dict(dctx_v=None), fe.FE_EINVAL),
    ({}, dict(down_k=None), fe.FE_EINVAL), ({}, dict(dout_ld=250), fe.FE_EINVAL), ({}, dict(dctx_ld=64), fe.FE_EINVAL),
    ({}, dict(dq=A16 + 2), fe.FE_EINVAL), (dict(lse=None), {}, fe.FE_EINVAL), (dict(ws=None), {}, fe.FE_EINVAL),
    (dict(ws_bytes=16), {}, fe.FE_EINVAL), (dict(page_rows=4, n_pages=9, table=A16), {}, fe.FE_EUNSUPPORTED),
])
def test_prefix_grad_is_checked(kw, gkw, status):
    lib, a, g = fe.load_library(), _args(**kw), _grads(**gkw)
    assert lib.fe_prefix_attention_grad(ctypes.byref(a), ctypes.byref(g), None) == status


def test_null_structures():
    lib, n = fe.load_library(), ctypes.c_size_t()
    assert lib.fe_prefix_workspace_size(None, 0, ctypes.byref(n)) == fe.FE_EINVAL
    assert lib.fe_prefix_workspace_size(ctypes.byref(_args()), 0, None) == fe.FE_EINVAL
    assert lib.fe_prefix_attention(None, None) == fe.FE_EINVAL
    assert lib.fe_prefix_attention_grad(ctypes.byref(_args()), None, None) == fe.FE_EINVAL
    assert lib.fe_cache_append(None, None) == fe.FE_EINVAL


def test_prefix_workspace():
    """A few rows over many keys are split over workgroups and need room for the partial sums; the call refuses less."""
    a = _args(B=1, K=1, S=1, T=8192)
    need = fe.fe_prefix_workspace_size(a)
    assert need > 0
    a.ws_bytes = need - 1
    assert fe.load_library().fe_prefix_attention(ctypes.byref(a), None) == fe.FE_EINVAL
    assert b"workspace" in fe.load_library().fe_last_error()
    assert fe.fe_prefix_workspace_size(a, True) >= 4 * a.n_heads
    with pytest.raises(fe.FeError):
        fe.fe_prefix_workspace_size(_args(page_rows=4, n_pages=2), True)


def test_gradient_grid():
    """2^28 shared keys of 4096 rows in two ranges: 2^26 workgroups of partial sums, more than a launch holds."""
    a = _args(dtype=fe.FE_F32, B=1, K=1, S=4096, n_heads=64, n_kv_heads=64, dh=128, T=1 << 22, L=0)
    fe.fe_prefix_workspace_size(a)
    with pytest.raises(fe.FeError, match="too large for the gradient"):
        fe.fe_prefix_workspace_size(a, True)


def test_row_stride_above_int32():
    t = torch.empty_strided((1, 2, 1, 32), (1 << 33, 1 << 32, 32, 1), dtype=torch.float32, device="meta")
    with pytest.raises(ValueError, match="int32"):
        fe._row_stride(t, "k", (1, 2, 1, 32), torch.float32)


def _append_args(**kw):
    a = fe.fe_append_args()
    base = dict(dtype=fe.FE_F32, N=3, S=2, n_heads=4, n_kv_heads=2, dh=32, rot=32, neighbours=0, page_rows=4, n_pages=9, table_cols=3,
                q_ld=128, k_ld=64, v_ld=64, q_out_ld=128, page_ld=64, q=A16, k=A16, v=A16, q_out=A16, freq=A16, table=A16,
                len=A16, new_len=None, pos0=None, k_pages=A16, v_pages=A16, len_out=None, status=None)
    for k, v in {**base, **kw}.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=3), fe.FE_EINVAL), (dict(N=0), fe.FE_EINVAL), (dict(S=0), fe.FE_EINVAL), (dict(n_kv_heads=0), fe.FE_EINVAL),
    (dict(n_heads=0), fe.FE_EINVAL), (dict(page_rows=0), fe.FE_EINVAL), (dict(n_pages=0), fe.FE_EINVAL), (dict(table_cols=0), fe.FE_EINVAL),
    (dict(dh=40), fe.FE_EUNSUPPORTED), (dict(rot=-2), fe.FE_EINVAL), (dict(rot=34), fe.FE_EINVAL), (dict(rot=15), fe.FE_EINVAL),
    (dict(rot=8), fe.FE_EUNSUPPORTED), (dict(k=None), fe.FE_EINVAL), (dict(v_pages=None), fe.FE_EINVAL), (dict(table=None), fe.FE_EINVAL),
    (dict(len=None), fe.FE_EINVAL), (dict(q=None), fe.FE_EINVAL), (dict(q_out=None), fe.FE_EINVAL), (dict(freq=None), fe.FE_EINVAL),
    (dict(k=A16 + 8), fe.FE_EINVAL), (dict(freq=A16 + 4), fe.FE_EINVAL), (dict(status=A16 + 2), fe.FE_EINVAL),
    (dict(k_ld=62), fe.FE_EINVAL), (dict(page_ld=66), fe.FE_EINVAL), (dict(q_ld=124), fe.FE_EINVAL), (dict(q_out_ld=64), fe.FE_EINVAL),
    (dict(N=1 << 20, S=1 << 12), fe.FE_EINVAL), (dict(table_cols=1 << 30), fe.FE_EINVAL), (dict(N=1 << 20, S=1 << 6), fe.FE_EUNSUPPORTED),
])
def test_append_is_checked(kw, status):
    a = _append_args(**kw)
    assert fe.load_library().fe_cache_append(ctypes.byref(a), None) == status
    assert fe.load_library().fe_last_error()


def test_binding_checks_layouts():
    """The binding hands raw pointers on: a wrong type, shape or layout is refused before any call."""
    p = fe.PrefixAttention(B=2, K=3, S=4, T=5, L=6, n_heads=4, n_kv_heads=2, dh=32, dtype="f32")
    q, c, o = torch.zeros(2, 3, 4, 4, 32), torch.zeros(2, 5, 2, 32), torch.zeros(2, 3, 6, 2, 32)
    for name, bad in dict(q=q.bfloat16(), ctx_k=c[:, :4], own_k=o.transpose(1, 2)).items():
        t = dict(q=q, ctx_k=c, ctx_v=c, own_k=o, own_v=o, **{})
        t[name] = bad
        with pytest.raises(ValueError, match=name):
            p.run(**t)
    with pytest.raises(ValueError, match="stride"):                      # values with another row stride than the keys
        p.run(q, c, torch.zeros(2, 5, 4, 32)[:, :, :2], o, o)
    with pytest.raises(ValueError, match="strides"):                     # every second row of a longer list: uneven from list to list
        p.run(q, c, c, torch.zeros(2, 3, 13, 2, 32)[:, :, 1::2], o)
    with pytest.raises(ValueError, match="table"):
        p.run(q, c, c, o, o, table=torch.zeros(2, 3, 1, dtype=torch.int32))
    with pytest.raises(ValueError, match="ctx_len"):
        p.run(q, c, c, o, o, ctx_len=torch.zeros(2))
    with pytest.raises(ValueError, match="device"):                      # everything else in order: the tensors are not on a GPU
        p.run(q, c, c, o, o)
    with pytest.raises(ValueError, match="train"):
        p.grad(q, q, c, c, o, o)
    with pytest.raises(ValueError, match="dtype"):
        fe.PrefixAttention(B=1, K=1, S=1, T=1, L=1, n_heads=1, n_kv_heads=1, dh=32, dtype="f16")
    with pytest.raises(fe.FeError):
        fe.PrefixAttention(B=1, K=1, S=1, T=1, L=1, n_heads=3, n_kv_heads=2, dh=32, dtype="f32")
    pages, table = torch.zeros(4, 8, 2, 32), torch.zeros(3, 2, dtype=torch.int32)
    with pytest.raises(ValueError, match="v_pages"):
        fe.PagedCache(pages, pages[:3], table)
    with pytest.raises(ValueError, match="table"):
        fe.PagedCache(pages, pages, table.long())
    with pytest.raises(ValueError, match="device"):
        fe.PagedCache(pages, pages, table)


def test_remembered_layouts_are_few():
    """Ever new lengths: what is remembered of them stays bounded, and what is asked again is right all the same."""
    known, asked = fe._Layouts(), []
    wide = lambda t: asked.append(1) or t.shape[1]                                      # noqa: E731
    for n in list(range(1, 2001)) + [2000, 1, 1, 2000]:
        assert known.of(wide, torch.empty(1, n, device="meta")) == n
    assert len(known.known) <= 256 and len(asked) == 2001
    bad = lambda t: (_ for _ in ()).throw(ValueError("no"))                             # noqa: E731
    for _ in range(2):                                                                  # a refusal is not remembered
        with pytest.raises(ValueError):
            known.of(bad, torch.empty(5, 5, device="meta"))


class _Stream:
    def __init__(self, handle):
        self.cuda_stream = handle


def test_current_stream_without_the_short_way(monkeypatch):
    """A torch without the private function that names a device's current stream serves every call all the same."""
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: _Stream(70 + a[0]))
    assert fe._stream(None) == 73 and fe._stream_on(2, None) == 72
    assert fe._stream(5) == fe._stream_on(2, 5) == fe._stream_on(2, _Stream(5)) == 5


def _without_a_gpu(monkeypatch):
    """The binding on CPU tensors, current stream 7, no library call; returns the list of (stream, tensors) handed over."""
    handed = []
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: _Stream(7))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(fe, "_on_device", lambda tensors: 0)
    monkeypatch.setattr(fe, "_allocated_for", lambda stream, *t, **kw: handed.append((stream, t)))
    for name in ("fe_cache_append", "fe_prefix_attention", "fe_prefix_attention_grad"):
        monkeypatch.setattr(fe, name, lambda *a: None)
    return handed


def _same(got, want):
    return any(g is want for g in got)


def test_a_caches_own_tensors_are_handed_to_a_given_stream(monkeypatch):
    """The first append on a stream waits for the zeros of the lengths and of status that the cache made itself."""
    handed = _without_a_gpu(monkeypatch)
    pages, table, k = torch.zeros(4, 8, 2, 32), torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, 1, 2, 32)
    cache = fe.PagedCache(pages, pages, table)
    for stream in (7, 11, 11, 13):
        cache.append(k, k, stream=stream)
    streams = [s for s, t in handed if _same(t, cache.len) and _same(t, cache.status)]
    assert streams == [11, 13]
    del handed[:]
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    cache.append(k, k, stream=17)                             # captured on the tensors' own stream: the wait is captured too
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: _Stream(19))
    cache.append(k, k, stream=19)                             # on another: it cannot wait for what is outside the capture
    assert [s for s, _ in handed] == [17]
    del handed[:]
    monkeypatch.undo()
    handed = _without_a_gpu(monkeypatch)
    cache.append(k, k, stream=17)                             # a capture says nothing about later calls
    assert [s for s, _ in handed] == [17]
    del handed[:]
    mine = torch.zeros(3, dtype=torch.int32)                  # lengths of the caller's are the caller's to order
    cache = fe.PagedCache(pages, pages, table, mine)
    cache.append(k, k, stream=11)
    assert [s for s, t in handed if _same(t, cache.status)] == [11] and not any(_same(t, mine) for _, t in handed)


def test_outputs_are_handed_to_every_stream(monkeypatch):
    """Outputs and workspace of an explicit allocate(), or of a call on another stream, as well."""
    handed = _without_a_gpu(monkeypatch)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    p = fe.PrefixAttention(B=1, K=2, S=3, T=4, L=3, n_heads=2, n_kv_heads=1, dh=32, dtype="f32", train=True)
    with monkeypatch.context() as m:
        m.setattr(torch, "device", lambda *a: "cpu")
        p.allocate()
    p.out.get_device = lambda: 0
    q, c, o = torch.zeros(1, 2, 3, 2, 32), torch.zeros(1, 4, 1, 32), torch.zeros(1, 2, 3, 1, 32)
    for stream in (7, 11, 11):
        p.run(q, c, c, o, o, stream=stream)
    p.grad(q, q, c, c, o, o, stream=13)
    streams = [s for s, t in handed if all(_same(t, x) for x in (p.out, p.lse, p.ws, *p.grads))]
    assert streams == [11, 13]


@pytest.mark.parametrize("shape,view,ld", [
    ((2, 3, 4, 32), lambda: torch.zeros(2, 3, 4, 32), 128),
    ((2, 3, 4, 32), lambda: torch.zeros(2, 3, 12, 32)[:, :, 4:8], 384),           # a column block of a fused projection
    ((1, 3, 4, 32), lambda: torch.zeros(5, 3, 4, 32)[2:3], 128),
    ((3, 1, 4, 32), lambda: torch.zeros(3, 7, 4, 32)[:, 2:3], 7 * 128),           # one row of every list
    ((1, 1, 1, 32), lambda: torch.zeros(1, 1, 9, 32)[:, :, 3:4], 32),
    ((3, 2, 4, 32), lambda: torch.zeros(3, 7, 4, 32)[:, 2:4], None),              # two rows of every list: not evenly spaced
    ((2, 3, 4, 32), lambda: torch.zeros(2, 3, 4, 64)[..., ::2], None),
    ((2, 3, 4, 32), lambda: torch.zeros(2, 3, 4, 64)[..., :32], None),
    ((2, 3, 4, 32), lambda: torch.zeros(2, 1, 4, 32).expand(2, 3, 4, 32), None),
])
def test_row_stride(shape, view, ld):
    if ld is None:
        with pytest.raises(ValueError):
            fe._row_stride(view(), "x", shape, torch.float32)
    else:
        assert fe._row_stride(view(), "x", shape, torch.float32) == ld


# -- the reference -------------------------------------------------------------------------------

def _case(causal, seed=0):
    r = np.random.default_rng(seed)
    B, K, S, T, L, H, Hkv, dh = 2, 3, 4, 5, 6, 4, 2, 8
    x = [r.standard_normal(s) for s in ((B, K, S, H, dh), (B, T, Hkv, dh), (B, T, Hkv, dh), (B, K, L, Hkv, dh), (B, K, L, Hkv, dh))]
    lens = dict(ctx_len=[5, 2], q_len=[[4, 2, 0], [1, 4, 3]], own_len=[[6, 2, 3], [0, 4, 1]])
    return x, dict(causal=causal, **lens), r.standard_normal((B, K, S, H, dh))


@pytest.mark.parametrize("causal", [False, True])
def test_reference_matches_differentiation_and_differences(causal):
    """out against torch's softmax over one masked row of all keys; gradients against reverse-mode differentiation and
    against central differences."""
    x, kw, do = _case(causal)
    got = ref.attend(*x, dtype="f32", dout=do, **kw)
    t = [torch.tensor(v, requires_grad=True) for v in x]
    q, ck, cv, ok, ov = t
    B, K, S, H, dh = q.shape
    T, L, G = ck.shape[1], ok.shape[2], H // ck.shape[2]
    nc, nq, no = (torch.tensor(kw[n]) for n in ("ctx_len", "q_len", "own_len"))
    j = torch.arange(L)
    own = (j < no[..., None, None]).expand(B, K, S, L)
    if causal:
        own = own & (j <= (no - nq)[..., None, None] + torch.arange(S)[:, None])
    see = torch.cat(((torch.arange(T) < nc[:, None, None, None]).expand(B, K, S, T), own), -1)
    see = see & (torch.arange(S) < nq[..., None])[..., None]
    keys = torch.cat((ck[:, None].expand(B, K, *ck.shape[1:]), ok), 2).repeat_interleave(G, 3)
    vals = torch.cat((cv[:, None].expand(B, K, *cv.shape[1:]), ov), 2).repeat_interleave(G, 3)
    s = (q[:, :, :, None] * keys[:, :, None]).sum(-1) * dh ** -0.5                     # [B][K][S][T + L][H]
    s = s.masked_fill(~see[..., None], -1e300)
    p = torch.softmax(s, 3) * see.any(-1)[..., None, None]
    out = (p[..., None] * vals[:, :, None]).sum(3)
    assert np.abs(out.detach().numpy() - got["out"][0]).max() < 1e-13
    (out * torch.tensor(do)).sum().backward()
    for name, v in zip(("dq", "dck", "dcv", "dok", "dov"), t):
        assert np.abs(v.grad.numpy() - got[name][0]).max() < 1e-12, name
    r = np.random.default_rng(1)
    for i, name in enumerate(("dq", "dck", "dcv", "dok", "dov")):
        for _ in range(4):
            at = tuple(r.integers(0, n) for n in x[i].shape)
            f = []
            for step in (1e-5, -1e-5):
                y = [v.copy() for v in x]
                y[i][at] += step
                f.append((ref.attend(*y, dtype="f32", **kw)["out"][0] * do).sum())
            assert abs((f[0] - f[1]) / 2e-5 - got[name][0][at]) < 1e-8, name


def test_reference_ignores_what_lies_outside():
    x, kw, do = _case(True)
    want = ref.attend(*x, dtype="bf16", dout=do, **kw)
    nc, nq, no = ref.clamp_lengths(2, 3, 4, 5, 6, kw["ctx_len"], kw["q_len"], kw["own_len"])
    for b in range(2):
        x[1][b, nc[b]:] = x[2][b, nc[b]:] = np.nan
        for k in range(3):
            x[0][b, k, nq[b, k]:] = do[b, k, nq[b, k]:] = np.nan
            x[3][b, k, no[b, k]:] = x[4][b, k, no[b, k]:] = np.nan
    got = ref.attend(*x, dtype="bf16", dout=do, **kw)
    for n in want:
        assert np.array_equal(want[n][0], got[n][0]) and np.array_equal(want[n][1], got[n][1])


def test_reference_turn_keeps_differences_of_positions():
    """Two vectors turned by their positions: their product depends on the difference of the positions alone."""
    r = np.random.default_rng(3)
    a, b, f = r.standard_normal((1, 16)), r.standard_normal((1, 16)), 100.0 ** -(np.arange(8) / 8)
    for near in (False, True):
        dots = [float((ref.turned(a, np.array(p + 5.0), f, near) * ref.turned(b, np.array(p * 1.0), f, near)).sum()) for p in (0, 7, 1000)]
        assert max(dots) - min(dots) < 1e-10
        assert abs(np.linalg.norm(ref.turned(a, np.array(3.0), f, near)) - np.linalg.norm(a)) < 1e-12


def _bf16(v):
    return torch.tensor(v).bfloat16().double().numpy()


def _two(v):
    return _bf16(v) + _bf16(v - _bf16(v))


def _cut(v):
    """The first 16 bits of the significand."""
    step = 2.0 ** (np.floor(np.log2(np.abs(v))) - 15)
    return np.trunc(v / step) * step


@pytest.mark.parametrize("K,S,L,dh", [(1, 40, 120, 64), (64, 1, 3, 32)])     # long sums; few terms, where D matters
def test_precise_bounds_tell_the_roundings_apart(K, S, L, dh):
    """The kernel's sums in float64, with p and ds rounded to one bf16 or as two, D from the rounded out or from out with its
    rest: the bounds at 16 bits hold what has 16 bits, and not the others."""
    r = np.random.default_rng(12)
    q, k, v, do = (_bf16(r.standard_normal((1, K, n, 1, dh))) for n in (S, L, L, S))
    none = np.zeros((1, 0, 1, dh))
    fine = ref.attend(q, none, none, k, v, dtype="bf16", causal=False, dout=do, up_out=ref.TWO_PARTS, up_own=ref.TWO_PARTS,
                      u_rest=ref.REST)

    def inside(name, got):
        val, bound = (x[0, :, :, 0] for x in fine[name])
        return bool((np.abs(_bf16(got) - val) <= bound).all())

    Q, K_, V, D = (x[0, :, :, 0] for x in (q, k, v, do))
    T = lambda x: x.transpose(0, 2, 1)                                                  # noqa: E731
    s = Q @ T(K_) * dh ** -0.5
    e = np.exp(s - s.max(-1, keepdims=True))
    l = e.sum(-1, keepdims=True)
    out = _two(e) @ V / l
    assert inside("out", out) and not inside("out", _bf16(e) @ V / l)
    p, dp = e / l, D @ T(V)
    dk = lambda f, o: T(f(p * (dp - (D * o).sum(-1, keepdims=True)))) @ Q * dh ** -0.5  # noqa: E731
    assert inside("dok", dk(_two, _cut(out))) and inside("dov", T(_two(p)) @ D)
    assert not inside("dok", dk(_bf16, _cut(out))) and not inside("dov", T(_bf16(p)) @ D)
    if L < 8:
        assert not inside("dok", dk(_two, _bf16(out)))

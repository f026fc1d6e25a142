"""The 4-bit cache without a GPU: the argument checks of the C calls, workspace and page sizes, and the reference that the
GPU tests compare with."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2603_02565_amd import flasheval as fe
from tests import packed_reference as ref

A16 = 4096          # a placeholder address: every call below is refused before anything touches it


def _cache(**kw):
    base = dict(pages=A16, page_ld=1 << 16, table=A16, len=A16, N=2, cols=3, page_rows=16, n_pages=9)
    return fe.fe_packed_cache(**{**base, **kw})


def _fill(a, base, kw):
    for k, v in {**base, **kw}.items():
        setattr(a, k, v)
    return a


def _append(**kw):
    return _fill(fe.fe_packed_append_args(), dict(
        cache=_cache(), dtype=fe.FE_BF16, S=4, n_heads=4, n_kv_heads=2, dh=64, rot=64, neighbours=0, q_ld=256, k_ld=128, v_ld=128,
        q_out_ld=256, q=A16, k=A16, v=A16, q_out=2 * A16, freq=A16, new_len=None, pos0=None, len_out=A16, status=A16), kw)


def _read(**kw):
    return _fill(fe.fe_packed_read_args(), dict(cache=_cache(), dtype=fe.FE_BF16, S=4, n_kv_heads=2, dh=64, k_ld=128, v_ld=128, k=A16,
                                                v=A16), kw)


def _attend(**kw):
    return _fill(fe.fe_packed_args(), dict(
        ctx=_cache(), own=_cache(N=6), dtype=fe.FE_BF16, B=2, K=3, S=2, n_heads=4, n_kv_heads=2, dh=64, causal=1, scale=0.125,
        q_ld=256, out_ld=256, q=A16, q_len=None, out=A16, lse=A16, ctx_w=A16, own_w=A16, ctx_w_out=A16, own_w_out=A16, ws=A16,
        ws_bytes=1 << 30), kw)


def _evict(**kw):
    return _fill(fe.fe_packed_evict_args(), dict(from_=_cache(), to=_cache(table=2 * A16, len=2 * A16), n_kv_heads=2, dh=64, keep=8, first=1,
                                                 recent=2, weight=A16, weight_out=2 * A16, kept=A16, status=A16), kw)


CACHE = [  # what every call checks of a cache
    (dict(N=0), fe.FE_EINVAL), (dict(cols=0), fe.FE_EINVAL), (dict(page_rows=0), fe.FE_EINVAL), (dict(n_pages=0), fe.FE_EINVAL),
    (dict(pages=None), fe.FE_EINVAL), (dict(table=None), fe.FE_EINVAL), (dict(len=None), fe.FE_EINVAL),
    (dict(pages=A16 + 8), fe.FE_EINVAL), (dict(table=A16 + 2), fe.FE_EINVAL), (dict(len=A16 + 1), fe.FE_EINVAL),
    (dict(page_ld=2 * 1088 - 16), fe.FE_EINVAL), (dict(page_ld=2 * 1088 + 8), fe.FE_EINVAL), (dict(page_ld=-16), fe.FE_EINVAL),
    (dict(cols=1 << 20, page_ld=1 << 20), fe.FE_EUNSUPPORTED), (dict(page_rows=1 << 23, page_ld=1 << 40), fe.FE_EUNSUPPORTED),
]


@pytest.mark.parametrize("kw,status", CACHE)
def test_caches_are_checked(kw, status):
    lib = fe.load_library()
    assert lib.fe_packed_append(ctypes.byref(_append(cache=_cache(**kw))), None) == status
    assert lib.fe_packed_read(ctypes.byref(_read(cache=_cache(**kw))), None) == status
    assert lib.fe_packed_evict(ctypes.byref(_evict(from_=_cache(**kw))), None) == status
    for name in ("ctx", "own"):
        if "N" in kw:
            kw = dict(N=5)                  # 0 is no cache there
        a = _attend(**{name: _cache(**{**dict(N=2 if name == "ctx" else 6), **kw})})
        assert lib.fe_packed_attention(ctypes.byref(a), None) == status
        assert lib.fe_packed_weights(ctypes.byref(a), None) == status
    assert lib.fe_last_error()


@pytest.mark.parametrize("kw,word,status", [
    (dict(dtype=5), "dtype", fe.FE_EINVAL), (dict(S=0), "S", fe.FE_EINVAL), (dict(n_kv_heads=0), "heads", fe.FE_EINVAL),
    (dict(n_heads=0), "heads", fe.FE_EINVAL), (dict(dh=96), "width", fe.FE_EUNSUPPORTED), (dict(rot=66), "rot", fe.FE_EINVAL),
    (dict(rot=-16), "rot", fe.FE_EINVAL), (dict(rot=24), "multiple", fe.FE_EUNSUPPORTED), (dict(k=None), "NULL", fe.FE_EINVAL),
    (dict(v=None), "NULL", fe.FE_EINVAL), (dict(q=None), "together", fe.FE_EINVAL), (dict(q_out=None), "together", fe.FE_EINVAL),
    (dict(q_out=A16), "q_out", fe.FE_EINVAL), (dict(freq=None), "freq", fe.FE_EINVAL), (dict(k=A16 + 8), "aligned", fe.FE_EINVAL),
    (dict(freq=A16 + 4), "aligned", fe.FE_EINVAL), (dict(pos0=A16 + 1), "aligned", fe.FE_EINVAL), (dict(k_ld=64), "stride", fe.FE_EINVAL),
    (dict(q_ld=260), "stride", fe.FE_EINVAL), (dict(q_out_ld=8), "stride", fe.FE_EINVAL), (dict(S=1 << 24), "rows", fe.FE_EUNSUPPORTED),
    (dict(n_kv_heads=1 << 26, k_ld=1 << 30, v_ld=1 << 30), "", fe.FE_EINVAL),
])
def test_append_is_checked(kw, word, status):
    lib = fe.load_library()
    assert lib.fe_packed_append(ctypes.byref(_append(**kw)), None) == status
    assert word in lib.fe_last_error().decode()


@pytest.mark.parametrize("kw,word,status", [
    (dict(dtype=5), "dtype", fe.FE_EINVAL), (dict(S=0), "S", fe.FE_EINVAL), (dict(k=None, v=None), "NULL", fe.FE_EINVAL),
    (dict(k=A16 + 8), "aligned", fe.FE_EINVAL), (dict(start=A16 + 2), "aligned", fe.FE_EINVAL), (dict(v_ld=120), "stride", fe.FE_EINVAL),
    (dict(dh=16), "width", fe.FE_EUNSUPPORTED),
])
def test_read_is_checked(kw, word, status):
    lib = fe.load_library()
    assert lib.fe_packed_read(ctypes.byref(_read(**kw)), None) == status
    assert word in lib.fe_last_error().decode()


@pytest.mark.parametrize("kw,word,status", [
    (dict(dtype=2), "dtype", fe.FE_EINVAL), (dict(B=0), "B", fe.FE_EINVAL), (dict(K=0), "K", fe.FE_EINVAL), (dict(S=0), "S", fe.FE_EINVAL),
    (dict(n_heads=3), "multiple", fe.FE_EINVAL), (dict(n_kv_heads=0), "heads", fe.FE_EINVAL), (dict(dh=48), "width", fe.FE_EUNSUPPORTED),
    (dict(B=3), "sequences", fe.FE_EINVAL), (dict(K=2), "sequences", fe.FE_EINVAL), (dict(q=None), "NULL", fe.FE_EINVAL),
    (dict(scale=float("nan")), "scale", fe.FE_EINVAL), (dict(q=A16 + 4), "aligned", fe.FE_EINVAL), (dict(ws=A16 + 8), "aligned", fe.FE_EINVAL),
    (dict(q_len=A16 + 2), "aligned", fe.FE_EINVAL), (dict(q_ld=192), "stride", fe.FE_EINVAL), (dict(q_ld=257), "stride", fe.FE_EINVAL),
    (dict(S=1 << 28), "large", fe.FE_EUNSUPPORTED), (dict(S=1 << 26, n_kv_heads=1, n_heads=1), "workgroups", fe.FE_EUNSUPPORTED),
])
def test_attention_and_weights_are_checked(kw, word, status):
    lib = fe.load_library()
    for call in (lib.fe_packed_attention, lib.fe_packed_weights):
        assert call(ctypes.byref(_attend(**kw)), None) == status
        assert word in lib.fe_last_error().decode()


@pytest.mark.parametrize("call,kw,word", [
    ("attention", dict(out=None), "out"), ("attention", dict(out=A16 + 8), "aligned"), ("attention", dict(out_ld=192), "stride"),
    ("weights", dict(lse=None), "lse"), ("weights", dict(ctx_w=None), "together"), ("weights", dict(own_w_out=None), "together"),
    ("weights", dict(own_w=A16 + 2), "aligned"), ("weights", dict(ctx=_cache(N=0)), "without"),
])
def test_attention_or_weights_are_checked(call, kw, word):
    lib = fe.load_library()
    assert getattr(lib, "fe_packed_" + call)(ctypes.byref(_attend(**kw)), None) == fe.FE_EINVAL
    assert word in lib.fe_last_error().decode()


@pytest.mark.parametrize("kw,word,status", [
    (dict(to=_cache(N=3, table=2 * A16, len=2 * A16)), "sequences", fe.FE_EINVAL), (dict(to=_cache(len=2 * A16)), "of its own", fe.FE_EINVAL),
    (dict(to=_cache(table=2 * A16)), "of its own", fe.FE_EINVAL), (dict(keep=0), "keep", fe.FE_EINVAL), (dict(keep=49), "capacity", fe.FE_EINVAL),
    (dict(first=-1), "first", fe.FE_EINVAL), (dict(recent=-1), "recent", fe.FE_EINVAL), (dict(weight=None), "NULL", fe.FE_EINVAL),
    (dict(kept=None), "NULL", fe.FE_EINVAL), (dict(weight=A16 + 2), "aligned", fe.FE_EINVAL), (dict(dh=20), "width", fe.FE_EUNSUPPORTED),
    (dict(to=_cache(pages=None, table=2 * A16, len=2 * A16)), "NULL", fe.FE_EINVAL),
    (dict(weight_out=A16), "overlaps", fe.FE_EINVAL), (dict(weight_out=A16 + 2 * 2 * 48 * 4 - 4), "overlaps", fe.FE_EINVAL),
    (dict(weight=A16 + 2 * 2 * 16 * 4 - 4, weight_out=A16, to=_cache(cols=1, table=2 * A16, len=2 * A16)), "overlaps", fe.FE_EINVAL),
])
def test_evict_is_checked(kw, word, status):
    lib = fe.load_library()
    assert lib.fe_packed_evict(ctypes.byref(_evict(**kw)), None) == status
    assert word in lib.fe_last_error().decode()


def test_null_arguments():
    lib, n = fe.load_library(), ctypes.c_size_t()
    for call in (lib.fe_packed_append, lib.fe_packed_read, lib.fe_packed_attention, lib.fe_packed_weights, lib.fe_packed_evict):
        assert call(None, None) == fe.FE_EINVAL
    assert lib.fe_packed_workspace_size(None, 0, ctypes.byref(n)) == fe.FE_EINVAL
    assert lib.fe_packed_workspace_size(ctypes.byref(_attend()), 0, None) == fe.FE_EINVAL
    assert lib.fe_packed_page_bytes(16, 2, 64, None) == fe.FE_EINVAL


def test_workspaces_are_checked_and_go_by_the_capacity():
    lib = fe.load_library()
    long = dict(ctx=_cache(cols=1 << 14, page_ld=1 << 16), B=2, K=3)
    need = fe.fe_packed_workspace_size(_attend(**long))
    assert need > 0
    a = _attend(ws_bytes=need - 1, **long)
    assert lib.fe_packed_attention(ctypes.byref(a), None) == fe.FE_EINVAL and "workspace" in lib.fe_last_error().decode()
    pages = dict(ctx=_cache(cols=1, page_rows=1 << 18), B=2, K=3)
    assert fe.fe_packed_workspace_size(_attend(**pages)) == need
    many = dict(K=3000, S=40, own=_cache(N=6000))
    need = fe.fe_packed_workspace_size(_attend(**many), True)
    assert need > 0
    a = _attend(ws=None, **many)
    assert lib.fe_packed_weights(ctypes.byref(a), None) == fe.FE_EINVAL and "workspace" in lib.fe_last_error().decode()


@pytest.mark.parametrize("P,Hkv,dh", [(1, 1, 32), (16, 8, 64), (7, 3, 128), (5, 2, 32)])
def test_page_bytes(P, Hkv, dh):
    assert fe.fe_packed_page_bytes(P, Hkv, dh) == Hkv * ref.head_bytes(P, dh)
    k, v = ref.place(P, dh, 0, 0), ref.place(P, dh, 1, P - 1)
    assert k[0].start == 0 and v[1].stop <= ref.head_bytes(P, dh) and v[0].stop == k[1].start


def test_page_bytes_are_checked():
    for args, status in (((0, 1, 64), fe.FE_EINVAL), ((4, 0, 64), fe.FE_EINVAL), ((4, 1, 48), fe.FE_EUNSUPPORTED)):
        with pytest.raises(fe.FeError) as e:
            fe.fe_packed_page_bytes(*args)
        assert e.value.status == status


# ---------------------------------------------------------------------------------------------
# The reference
# ---------------------------------------------------------------------------------------------

def test_reference_holds_what_it_can():
    """Every number that a block can hold, at every scale, is held as itself."""
    sizes = np.array(ref.SIZES)
    x = np.concatenate((sizes, -sizes, sizes, -sizes))
    for e in range(2, 253):
        codes, scales = ref.hold(x * 2.0 ** (e - 127))
        assert scales.tolist() == [e] and np.array_equal(ref.values(codes, scales), x * 2.0 ** (e - 127))


def test_reference_rounds_to_the_nearest():
    """Borders go to the even code, a step beside them to the nearer one."""
    for a, b, border, even in ((0, .5, .25, 0), (.5, 1, .75, 1), (1, 1.5, 1.25, 1), (1.5, 2, 1.75, 2), (2, 3, 2.5, 2), (3, 4, 3.5, 4), (4, 6, 5, 4)):
        for x, want in ((border, even), (border * (1 - 2e-16), a), (border * (1 + 3e-16), b), (a, a), (b, b)):
            for sign in (1, -1):
                row = np.zeros(32)
                row[:2] = sign * x, 6.0
                assert ref.held_values(row)[0] == sign * want


def test_reference_scale_is_the_smallest_that_holds():
    r = np.random.default_rng(0)
    x = r.standard_normal((500, 32)) * np.exp2(r.integers(-100, 100, (500, 1)))
    _, scales = ref.hold(x)
    unit = 2.0 ** (scales[:, 0].astype(float) - 127)
    top = np.abs(x).max(-1)
    assert (top <= 6 * unit).all() and (top > 3 * unit).all()
    step = np.abs(ref.held_values(x) - x)
    assert (step <= unit[:, None]).all()                                  # half of the widest step, 4 to 6
    assert ref.hold(np.full(32, 2.0 ** 127))[1] == 252 and ref.hold(np.zeros(32))[1] == 2
    assert np.isnan(ref.held_values(np.array([1.0] * 31 + [np.inf]))).all()


def test_reference_pages_keep_rows_apart():
    r = np.random.default_rng(1)
    for P, dh in ((3, 32), (5, 128)):
        pages = np.zeros((2, 2, ref.head_bytes(P, dh)), np.uint8)
        x = r.standard_normal((2, P, 2, 2, dh))
        for p in (0, 1):
            for row in range(P):
                ref.write(pages, p, row, P, dh, x[p, row, 0], x[p, row, 1])
        many = np.zeros_like(pages)
        for p in (0, 1):
            ref.write_rows(many, np.full(P, p), np.arange(P), P, dh, x[p, :, 0], x[p, :, 1])
        assert np.array_equal(many, pages)
        for p in (0, 1):
            for row in range(P):
                k, v = ref.read(pages, p, row, P, dh)
                assert np.array_equal(k, ref.held_values(x[p, row, 0])) and np.array_equal(v, ref.held_values(x[p, row, 1]))


def test_reference_weights_of_a_row_add_up_to_one():
    from tests import prefix_reference as dense
    r = np.random.default_rng(2)
    q, ck, ok = r.standard_normal((1, 2, 3, 4, 32)), r.standard_normal((1, 9, 2, 32)), r.standard_normal((1, 2, 5, 2, 32))
    kw = dict(causal=True, scale=0.2, ctx_len=np.array([7]), q_len=np.array([[3, 2]]), own_len=np.array([[5, 4]]))
    lse = dense.attend(q, ck, ck, ok, ok, dtype="f32", **kw)["lse"][0]
    w = ref.weigh(q, ck, ok, lse, ctx_w=np.zeros((1, 2, 9)), own_w=np.zeros((1, 2, 2, 5)), **kw)
    total = w["ctx_w"][0].sum() + w["own_w"][0].sum()
    assert abs(total - 4 * (3 + 2)) < 1e-12
    assert w["own_w"][0][0, 0, :, 4].max() < w["own_w"][0][0, 0, :, 2].max() + 3   # only the last row sees the last key
    assert (w["own_w"][0][0, 1, :, 4] == 0).all() and (w["ctx_w"][0][:, :, 7:] == 0).all()


def test_reference_eviction():
    w = [5.0, 1.0, 3.0, 3.0, float("nan"), 9.0, 0.0, 3.0]
    assert ref.evict_rows(w, 8, 4, 0, 0) == [0, 2, 3, 5]                 # of the three 3.0 the lower indices
    assert ref.evict_rows(w, 8, 4, 2, 1) == [0, 1, 5, 7]
    assert ref.evict_rows(w, 8, 8, 2, 1) == ref.evict_rows(w, 8, 20, 0, 0) == list(range(8))
    assert ref.evict_rows(w, 8, 7, 0, 0) == [0, 1, 2, 3, 5, 6, 7]         # NaN after every number
    assert ref.evict_rows(w, 8, 3, 5, 5) == [0, 1, 2] and ref.evict_rows(w, 8, 3, 1, 5) == [0, 6, 7]
    assert ref.evict_rows(w, 0, 3, 1, 1) == []


def test_held_values_are_exact_in_bf16():
    """What a block stands for has no more bits than bf16 keeps."""
    x = np.random.default_rng(3).standard_normal((7, 64))
    v = ref.held_values(x)
    assert np.array_equal(torch.tensor(v).bfloat16().double().numpy(), v)


# ---------------------------------------------------------------------------------------------
# Log sums of any strides
# ---------------------------------------------------------------------------------------------

@pytest.mark.parametrize("ld,word,status", [
    ((24, 8, 4, -1), "negative", fe.FE_EINVAL), ((-24, 8, 4, 1), "negative", fe.FE_EINVAL),
    ((1, 1 << 30, 4, 1), "apart", fe.FE_EUNSUPPORTED), ((1, 8, 1 << 31, 1), "apart", fe.FE_EUNSUPPORTED),
    ((1 << 50, 8, 4, 1), "apart", fe.FE_EUNSUPPORTED), ((1, 1 << 62, 1 << 62, 1 << 62), "apart", fe.FE_EUNSUPPORTED),
])
def test_strides_of_log_sums_are_checked(ld, word, status):
    lib = fe.load_library()
    st = lib.fe_packed_weights_strided(ctypes.byref(_attend()), (ctypes.c_int64 * 4)(*ld), None)
    assert st == status and word in lib.fe_last_error().decode()


def test_strided_weights_check_what_the_dense_ones_do():
    lib, ld = fe.load_library(), (ctypes.c_int64 * 4)(24, 8, 4, 1)
    assert lib.fe_packed_weights_strided(ctypes.byref(_attend()), None, None) == fe.FE_EINVAL
    assert lib.fe_packed_weights_strided(None, ld, None) == fe.FE_EINVAL
    for kw, word in ((dict(lse=None), "lse"), (dict(ctx_w=None), "together"), (dict(n_heads=3), "multiple")):
        assert lib.fe_packed_weights_strided(ctypes.byref(_attend(**kw)), ld, None) == fe.FE_EINVAL
        assert word in lib.fe_last_error().decode()
    # the axes of one element: their stride is not looked at, and the workspace is the next thing that is missing
    many = _attend(K=3000, S=40, own=_cache(N=6000), ws=None)
    for n in (dict(), dict(B=1, ctx=_cache(N=1), own=_cache(N=3000))):
        a = _fill(many, {}, n)
        st = lib.fe_packed_weights_strided(ctypes.byref(a), (ctypes.c_int64 * 4)(-5 if n else 1, 1, 0, 7), None)
        assert st == fe.FE_EINVAL and "workspace" in lib.fe_last_error().decode()


def test_reference_weights_keep_to_the_mask():
    """The last own key is seen by the last query row alone, the first by all; without the mask by all of them."""
    from tests import prefix_reference as dense
    r = np.random.default_rng(4)
    q, ck, ok = r.standard_normal((1, 2, 3, 4, 32)), r.standard_normal((1, 9, 2, 32)), r.standard_normal((1, 2, 5, 2, 32))
    kw = dict(scale=0.2, ctx_len=np.array([7]), q_len=np.array([[3, 2]]), own_len=np.array([[5, 4]]))
    zero = dict(ctx_w=np.zeros((1, 2, 9)), own_w=np.zeros((1, 2, 2, 5)))
    for causal in (True, False):
        lse = dense.attend(q, ck, ck, ok, ok, dtype="f32", causal=causal, **kw)["lse"][0]
        w = ref.weigh(q, ck, ok, lse, causal=causal, **kw, **zero)
        for k, (n, m) in enumerate(((3, 5), (2, 4))):
            for g in range(2):
                for j in range(m):
                    rows = [i for i in range(n) if not causal or j <= m - n + i]
                    want = sum(np.exp(0.2 * (q[0, k, i, h] @ ok[0, k, j, g]) - lse[0, k, i, h]) for i in rows for h in (2 * g, 2 * g + 1))
                    assert abs(w["own_w"][0][0, k, g, j] - want) < 1e-13
        lse[0, 0, 2] = -np.inf                                            # the last row of list 0 gives nothing
        w = ref.weigh(q, ck, ok, lse, causal=causal, **kw, **zero)
        assert ((w["own_w"][0][0, 0, :, 4] == 0) == causal).all() and (w["own_w"][0][0, 0, :, 3] > 0).all()

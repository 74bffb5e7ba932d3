"""Host-side checks of the serving entry points: what they refuse before they touch a device, and the test forms themselves."""
import ctypes

import numpy as np
import pytest

import _serving as ref

P = ctypes.c_void_p(0x10000)      # never dereferenced: every call below is refused on the host
ODD = ctypes.c_void_p(0x10004)    # not 16-byte aligned
OK, NULL, SHAPE, DTYPE, ALIGN, WORKSPACE, UNSUPPORTED = 0, 1, 2, 3, 4, 5, 6


@pytest.fixture(scope="module")
def ec():
    import paper_2603_18489_b200 as ec
    return ec


def paged(ec, **kw):
    d = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, dtype=ec.EC_BF16, page_size=16, n_pages=10, max_pages=5, mask_block=1)
    d.update(kw)
    return ec.make_paged_desc(**d)


BAD_PAGED = [(dict(batch=0), SHAPE), (dict(n_pages=0), SHAPE), (dict(max_pages=0), SHAPE), (dict(mask_block=-1), SHAPE),
             (dict(n_q_heads=7), SHAPE), (dict(scale=-1.0), SHAPE), (dict(scale=float("nan")), SHAPE), (dict(dtype=7), DTYPE),
             (dict(head_dim=96), UNSUPPORTED), (dict(page_size=8), UNSUPPORTED), (dict(page_size=48), UNSUPPORTED),
             (dict(batch=1025), UNSUPPORTED), (dict(n_q_heads=129, n_kv_heads=1), UNSUPPORTED)]


def attend(ec, d, q=P, ro=P, kl=P, n_rows=4, max_rows=2, pt=P, k=P, v=P, out=P, ws=P, ws_bytes=1 << 40, status=None):
    f = ec.lib.ec_attend_paged
    f.restype = ctypes.c_int32
    f.argtypes = [ctypes.c_void_p] * 4 + [ctypes.c_int32] * 2 + [ctypes.c_void_p] * 5 + [ctypes.c_size_t] + [ctypes.c_void_p] * 2
    return f(ctypes.byref(d) if d is not None else None, q, ro, kl, n_rows, max_rows, pt, k, v, out, ws, ws_bytes, status, None)


def test_attend_paged_refuses(ec):
    for kw, code in BAD_PAGED:
        d = paged(ec, **kw)
        assert attend(ec, d) == code, kw
        assert ec.ec_attend_paged_workspace_bytes(d, 2) == 0 and ec.ec_attend_paged_kernel_name(d, 2) == ""
    d = paged(ec)
    d.flags = 1
    assert attend(ec, d) == UNSUPPORTED
    d = paged(ec)
    assert attend(ec, None) == NULL
    assert attend(ec, d, n_rows=-1) == SHAPE and attend(ec, d, max_rows=0) == SHAPE
    assert attend(ec, d, n_rows=0, q=None) == OK
    for name in ("q", "ro", "kl", "pt", "k", "v", "out"):
        assert attend(ec, d, **{name: None}) == NULL, name
    for name in ("q", "k", "v", "out", "ws"):
        assert attend(ec, d, **{name: ODD}) == ALIGN, name
    assert attend(ec, d, status=ctypes.c_void_p(0x10001)) == ALIGN
    need = ec.ec_attend_paged_workspace_bytes(d, 2)
    assert need > 0 and attend(ec, d, ws_bytes=need - 1) == WORKSPACE and attend(ec, d, ws=None) == WORKSPACE


def test_which_paged_kernel(ec):
    rows, tiles = "attend_paged_rows_kernel", "attend_paged_tiles_kernel"
    assert ec.ec_attend_paged_kernel_name(paged(ec, max_pages=100000), 4) == rows           # 16 packed rows
    assert ec.ec_attend_paged_kernel_name(paged(ec, max_pages=100000), 5) == tiles
    assert ec.ec_attend_paged_kernel_name(paged(ec, max_pages=8), 34) == rows               # few keys
    assert ec.ec_attend_paged_kernel_name(paged(ec, dtype=ec.EC_F32, max_pages=100000), 500) == rows
    assert ec.ec_attend_paged_kernel_name(paged(ec, n_pages=2 ** 30 + 1, max_pages=100000), 500) == rows   # beyond a tensor map


def rope(ec, d, q=P, qs=1024, k=P, ks=256, qw=None, kw=None, pos=P, f=P, n=4, qo=P, ko=P):
    g = ec.lib.ec_qk_norm_rope
    g.restype = ctypes.c_int32
    vp, i64 = ctypes.c_void_p, ctypes.c_int64
    g.argtypes = [vp, vp, i64, vp, i64, vp, vp, vp, vp, ctypes.c_int32, vp, vp, vp]
    return g(ctypes.byref(d) if d is not None else None, q, qs, k, ks, qw, kw, pos, f, n, qo, ko, None)


def test_rope_refuses(ec):
    good = dict(n_q_heads=8, n_kv_heads=2, head_dim=128, dtype=ec.EC_BF16, rot_dim=128)
    for kw, code in [(dict(n_q_heads=0), SHAPE), (dict(head_dim=80), UNSUPPORTED), (dict(dtype=5), DTYPE), (dict(rot_dim=8), SHAPE),
                     (dict(rot_dim=144), SHAPE), (dict(rot_dim=-16), SHAPE), (dict(eps=-1.0), SHAPE), (dict(eps=float("nan")), SHAPE),
                     (dict(n_q_heads=5000), UNSUPPORTED)]:
        assert rope(ec, ec.make_rope_desc(**{**good, **kw})) == code, kw
    d = ec.make_rope_desc(**good)
    d.flags = 2
    assert rope(ec, d) == UNSUPPORTED
    d = ec.make_rope_desc(**good)
    assert rope(ec, None) == NULL and rope(ec, d, n=-1) == SHAPE and rope(ec, d, n=0, q=None) == OK
    for name in ("q", "k", "pos", "f", "qo", "ko"):
        assert rope(ec, d, **{name: None}) == NULL, name
    assert rope(ec, d, qw=P) == NULL and rope(ec, d, kw=P) == NULL
    assert rope(ec, d, qs=1016) == SHAPE and rope(ec, d, ks=128) == SHAPE       # rows that would overlap
    assert rope(ec, d, qs=1028) == ALIGN and rope(ec, d, q=ODD) == ALIGN and rope(ec, d, ko=ODD) == ALIGN
    assert rope(ec, d, qw=ODD, kw=P) == ALIGN and rope(ec, d, pos=ctypes.c_void_p(0x10002)) == ALIGN


def test_rope_paged_refuses(ec):
    f = ec.lib.ec_qk_norm_rope_paged
    f.restype = ctypes.c_int32
    vp, i64 = ctypes.c_void_p, ctypes.c_int64
    f.argtypes = [vp, vp, vp, i64, vp, i64, vp, i64, vp, vp, vp, vp, vp, ctypes.c_int32, vp, vp, vp, vp, vp, vp]

    def call(d, g, v=P, vs=256, ro=P, pt=P, vp_=P, n=4):
        return f(ctypes.byref(d), ctypes.byref(g), P, 1024, P, 256, v, vs, None, None, ro, P, P, n, pt, P, P, vp_, None, None)

    d = ec.make_rope_desc(8, 2, 128, ec.EC_BF16, 128)
    for kw, code in BAD_PAGED:
        assert call(d, paged(ec, **kw)) == code, kw
    g = paged(ec)
    assert call(d, paged(ec, n_q_heads=6)) == SHAPE and call(d, paged(ec, head_dim=64)) == SHAPE
    assert call(d, paged(ec, dtype=ec.EC_F32)) == DTYPE
    assert call(d, g, v=None) == NULL and call(d, g, ro=None) == NULL and call(d, g, pt=None) == NULL and call(d, g, vp_=None) == NULL
    assert call(d, g, vs=100) == SHAPE and call(d, g, v=ODD) == ALIGN and call(d, g, vp_=ODD) == ALIGN
    assert call(d, g, n=0, v=None) == OK


def test_sample_refuses(ec):
    f = ec.lib.ec_sample
    f.restype = ctypes.c_int32
    vp, i32 = ctypes.c_void_p, ctypes.c_int32
    f.argtypes = [vp, i32, i32, i32, ctypes.c_int64, vp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]

    def call(logits=P, dtype=ec.EC_BF16, n=3, vocab=1000, stride=1000, u=P, t=None, token=P, ws=P, ws_bytes=1 << 20):
        return f(logits, dtype, n, vocab, stride, u, t, None, None, None, token, None, None, ws, ws_bytes, None)

    assert call(dtype=9) == DTYPE and call(n=-1) == SHAPE and call(vocab=0) == SHAPE and call(stride=999) == SHAPE
    assert call(vocab=(1 << 20) + 1, stride=1 << 21) == UNSUPPORTED
    assert call(logits=None) == NULL and call(u=None) == NULL and call(token=None) == NULL and call(n=0, logits=None) == OK
    assert call(logits=ODD) == ALIGN and call(vocab=1001, stride=1001) == ALIGN and call(t=ctypes.c_void_p(0x10002)) == ALIGN
    assert call(ws=None) == WORKSPACE and call(ws_bytes=0) == WORKSPACE
    assert ec.ec_sample_workspace_bytes(3, 1000) > 0 and ec.ec_sample_workspace_bytes(3, 0) == 0
    assert ec.ec_sample_workspace_bytes(3, (1 << 20) + 1) == 0


class pages_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("batch", "max_pages", "n_pages", "page_size")]


def test_pages_refuse(ec):
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    fork, reserve, release, compact, copy = (getattr(ec.lib, "ec_pages_" + n) for n in ("fork", "reserve", "release", "compact", "copy"))
    fork.argtypes = [vp] * 6 + [i32, vp, vp]
    reserve.argtypes = [vp] * 8 + [i32, vp, vp, sz, vp, vp]
    release.argtypes = [vp] * 6
    compact.argtypes = [vp] * 6 + [i32, vp, vp, sz, vp]
    copy.argtypes = [vp, vp, i64, i32, i32, i64, vp, vp, i32, vp, vp, vp]
    calls = dict(fork=lambda d, t=P, n=1: fork(d, t, P, P, P, P, n, None, None),
                 reserve=lambda d, t=P, cap=1, ws=P, size=1 << 30: reserve(d, t, P, P, P, P, P, P, cap, P, ws, size, None, None),
                 release=lambda d, t=P: release(d, t, P, P, P, None),
                 compact=lambda d, t=P, cap=100, ws=P, size=1 << 30: compact(d, t, P, P, P, P, cap, P, ws, size, None))
    good = pages_desc(4, 8, 20, 16)
    for call in calls.values():
        assert call(None) == NULL and call(ctypes.byref(good), None) == NULL
        assert call(ctypes.byref(good), ctypes.c_void_p(0x10002)) == ALIGN
        for bad, code in ((pages_desc(0, 8, 20, 16), SHAPE), (pages_desc(4, 0, 20, 16), SHAPE), (pages_desc(4, 8, 0, 16), SHAPE),
                          (pages_desc(4, 8, 20, 0), SHAPE), (pages_desc(1025, 8, 20, 16), UNSUPPORTED),
                          (pages_desc(4, 2 ** 28, 20, 16), UNSUPPORTED)):
            assert call(ctypes.byref(bad)) == code
    # entries that 32 bits cannot count (reserve adds up what its sequences need)
    many = pages_desc(1024, 2 ** 21, 20, 1)
    for call in calls.values():
        assert call(ctypes.byref(many)) == UNSUPPORTED
    g = ctypes.byref(good)
    assert calls["fork"](g, n=-1) == SHAPE and calls["fork"](g, n=5) == SHAPE and calls["fork"](g, n=0) == OK
    assert calls["reserve"](g, cap=-1) == SHAPE and calls["reserve"](g, size=79) == WORKSPACE and calls["reserve"](g, ws=ODD) == ALIGN
    assert calls["compact"](g, cap=9) == SHAPE and calls["compact"](g, size=79) == WORKSPACE
    assert ec.ec_pages_workspace_bytes(20) == 80 and ec.ec_pages_workspace_bytes(0) == 0

    def cp(k=P, page=1024, n_pages=20, layers=1, layer=0, src=P, cap=3):
        return copy(k, P, page, n_pages, layers, layer, src, P, cap, None, None, None)

    assert cp(page=0) == SHAPE and cp(n_pages=0) == SHAPE and cp(layers=0) == SHAPE and cp(cap=-1) == SHAPE
    assert cp(layers=2, layer=20 * 1024 - 16) == SHAPE            # layers that would overlap
    assert cp(k=None) == NULL and cp(src=None) == NULL and cp(cap=0, k=None) == OK
    assert cp(page=1000) == ALIGN and cp(k=ODD) == ALIGN


def test_binding_refuses_host_tensors_and_wrong_shapes(ec):
    torch = pytest.importorskip("torch")
    x = torch.zeros(2, 8)
    with pytest.raises(ValueError, match="CUDA tensor"):
        ec.ec_sample(x, 8, torch.zeros(2), token_out=torch.zeros(2, dtype=torch.int32), prob_out=torch.zeros(2),
                     kept_out=torch.zeros(2, dtype=torch.int32), workspace=torch.zeros(16, dtype=torch.uint8))
    with pytest.raises(ValueError, match="CUDA tensor"):
        ec.ec_pages_release(*ec.new_pages(2, 3, 8, device="cpu"), torch.zeros(2, dtype=torch.int32), 16)
    with pytest.raises(TypeError):
        ec.make_paged_desc(1, 1, 1, 64, torch.float16, 16, 1, 1)
    with pytest.raises(ValueError):
        ec.ec_pages_copy(torch.zeros(3), torch.zeros(3), None, None)


# ---- the forms that the GPU tests compare with -----------------------------------------------------------------------
def test_sampling_form_by_hand():
    x = np.array([0.0, 2.0, 2.0, -np.inf, 1.0])
    w = np.exp([0.0, 0.0, -1.0, -2.0])            # tokens 1, 2, 4, 0
    s = w.sum()
    assert ref.sample(x, 0.0) == (1, w[0] / s, 4)
    assert ref.sample(x, float(w[0] / s) - 1e-9)[0] == 1 and ref.sample(x, float(w[0] / s) + 1e-9)[0] == 2
    assert ref.sample(x, 0.999999)[0] == 0
    assert ref.sample(x, 0.9, top_k=2) == (2, 0.5, 2)
    assert ref.sample(x, 0.9, top_p=0.5)[2] == 2 and ref.sample(x, 0.9, top_p=0.0)[2] == 1
    assert ref.sample(x, 0.9, min_p=0.2)[2] == 3 and ref.sample(x, 0.9, min_p=2.0)[2] == 1
    assert ref.sample(x, 0.9, temperature=0.0) == (1, 1.0, 1)
    assert ref.sample(np.full(3, -np.inf), 0.5) == (-1, 0.0, 0)


def test_visible_keys_by_hand():
    assert ref.visible(3, 10, 0).tolist() == [10, 10, 10]
    assert ref.visible(3, 10, 1).tolist() == [8, 9, 10]
    assert ref.visible(4, 10, 4).tolist() == [8, 8, 10, 10]
    assert ref.visible(5, 3, 1).tolist() == [0, 0, 1, 2, 3]


def test_rotation_form_turns_by_the_angle():
    x = np.zeros((1, 1, 64))
    x[0, 0, 3] = 1.0
    y, _ = ref.norm_rope(x, None, 0.0, np.array([2]), np.full(16, 0.25), 32, False)
    assert np.isclose(y[0, 0, 3], np.cos(0.5)) and np.isclose(y[0, 0, 19], np.sin(0.5))
    y, _ = ref.norm_rope(x, None, 0.0, np.array([2]), np.full(16, 0.25), 32, True)
    assert np.isclose(y[0, 0, 3], np.cos(0.5)) and np.isclose(y[0, 0, 2], -np.sin(0.5))


def test_page_form_by_hand():
    p = ref.Pages(np.array([[4, 1, -1], [-1, -1, -1]], np.int32), np.array([20, 0], np.int32), np.array([0, 1, 0, 0, 1], np.int32), 16)
    assert not p.fork([0], [1]) and p.refs.tolist() == [0, 2, 0, 0, 2]
    assert p.reserve(np.array([20, 20]), np.array([21, 40]), 9) == [(1, 0), (1, 2)]
    assert p.table.tolist() == [[4, 0, -1], [4, 2, 3]] and p.refs.tolist() == [1, 0, 1, 1, 2]
    p.release(np.array([0, 16]))
    assert p.refs.tolist() == [0, 0, 0, 0, 1] and p.compact() == [(4, 0)] and p.table[1, 0] == 0

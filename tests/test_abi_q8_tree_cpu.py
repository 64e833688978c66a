"""Refusals of the 8-bit cache's and the tree's entry points, before the device is
touched (fake aligned pointers; validation fails before any use)."""
import os

import pytest
import torch

from paper_2608_19920_amd import h2o as H

P, MIS = 0x10000, 0x10004
EINVAL, ESHAPE, EDTYPE, EALIGN, EWS = (H.H2O_EINVAL, H.H2O_ESHAPE, H.H2O_EDTYPE, H.H2O_EALIGN,
                                       H.H2O_EWORKSPACE)


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(H.LIB_PATH):
        pytest.skip("libh2o.so not built")
    return H.lib()


SIZES = dict(B=1, Hq=4, Hkv=2, T=8, M=16, d=64)


def _quant(L, fn, **kw):
    a = dict(src=P, v=P, idx=None, kc=P, ks=P, vc=P, vs=P, B=1, Hkv=2, M=16, k=8, d=64, dt=1)
    a.update(kw)
    sizes = (a["B"], a["Hkv"], a["M"], a["k"], a["d"], a["dt"], None)
    cache = (a["kc"], a["ks"], a["vc"], a["vs"])
    if fn == "h2o_kv_quantize":
        return L.h2o_kv_quantize(a["src"], a["v"], a["idx"], *cache, *sizes)
    return L.h2o_kv_dequantize(*cache, a["idx"], a["src"], a["v"], *sizes)


@pytest.mark.parametrize("fn", ["h2o_kv_quantize", "h2o_kv_dequantize"])
@pytest.mark.parametrize("kw,code", [
    (dict(dt=2), EDTYPE), (dict(d=96), ESHAPE), (dict(B=0), ESHAPE), (dict(M=0, k=0), ESHAPE),
    (dict(k=17), ESHAPE), (dict(k=-1), ESHAPE), (dict(B=1 << 20, Hkv=1, M=512, k=512), ESHAPE),
    (dict(src=None), EINVAL), (dict(v=None), EINVAL), (dict(kc=None), EINVAL),
    (dict(ks=None), EINVAL), (dict(vc=None), EINVAL), (dict(vs=None), EINVAL),
    (dict(src=MIS), EALIGN), (dict(v=MIS), EALIGN), (dict(idx=MIS), EALIGN),
    (dict(kc=MIS), EALIGN), (dict(ks=MIS), EALIGN), (dict(vc=MIS), EALIGN), (dict(vs=MIS), EALIGN),
], ids=str)
def test_quantize_rejects(L, fn, kw, code):
    assert _quant(L, fn, **kw) == code and H.lib().h2o_last_error()


def _attend(L, **kw):
    a = dict(SIZES, q=P, kc=P, ks=P, vc=P, vs=P, kn=P, vn=P, out=P, lse=P, wsum=P, ws=P,
             wsb=1 << 40, scale=0.125, dt=1)
    a.update(kw)
    return L.h2o_sdpa_chunk_q8(*(a[n] for n in ("q", "kc", "ks", "vc", "vs", "kn", "vn", "out",
                                                "lse", "wsum", "ws", "wsb", "B", "Hq", "Hkv", "T",
                                                "M", "d", "scale", "dt")), None)


SHAPE_REFUSALS = [
    (dict(dt=7), EDTYPE), (dict(Hq=5), ESHAPE), (dict(d=32), ESHAPE), (dict(Hkv=0), ESHAPE),
    (dict(T=0), EINVAL), (dict(M=-1), EINVAL), (dict(M=1 << 24), ESHAPE),
    (dict(B=32768, Hq=8, Hkv=4), ESHAPE),
    (dict(scale=0.0), EINVAL), (dict(scale=float("nan")), EINVAL), (dict(scale=-1.0), EINVAL),
    (dict(M=4096, wsb=0), EWS), (dict(M=4096, ws=None), EWS),
]


@pytest.mark.parametrize("kw,code", SHAPE_REFUSALS + [
    (dict([(n, None)]), EINVAL) for n in ("q", "kc", "ks", "vc", "vs", "kn", "vn", "out", "lse", "wsum")
] + [(dict([(n, MIS)]), EALIGN) for n in ("q", "kc", "ks", "vc", "vs", "kn", "vn", "out", "lse",
                                          "wsum", "ws")], ids=str)
def test_attend_rejects(L, kw, code):
    assert _attend(L, **kw) == code


def _evict(L, **kw):
    a = dict(B=1, Hkv=2, M=16, T=8, d=64, k=8, kc=P, ks=P, vc=P, vs=P, sc=P, tp=P, kn=P, vn=P,
             wsum=P, idx=P, dt=1, policy=0, ws=None, wsb=0)
    a.update(kw)
    return L.h2o_evict_insert_q8(*(a[n] for n in ("kc", "ks", "vc", "vs", "sc", "tp", "kn", "vn",
                                                  "wsum", "idx", "B", "Hkv", "M", "T", "d", "k")),
                                 0, a["dt"], a["policy"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(dt=3), EDTYPE), (dict(k=7), EINVAL), (dict(T=0, k=0), EINVAL), (dict(M=7), EINVAL),
    (dict(policy=3), EINVAL), (dict(policy=1, tp=None), EINVAL), (dict(policy=1), EWS),
    (dict(policy=2, ws=P, wsb=16), EWS), (dict(policy=2, ws=MIS, wsb=1 << 20), EALIGN),
    (dict(d=65), ESHAPE),
] + [(dict([(n, None)]), EINVAL) for n in ("kc", "ks", "vc", "vs", "sc", "kn", "vn", "wsum", "idx")] +
    [(dict([(n, MIS)]), EALIGN) for n in ("kc", "ks", "vc", "vs", "sc", "tp", "kn", "vn", "wsum",
                                          "idx")], ids=str)
def test_evict_rejects(L, kw, code):
    assert _evict(L, **kw) == code


def _step(L, **kw):
    a = dict(SIZES, q=P, kc=P, ks=P, vc=P, vs=P, sc=P, tp=P, kn=P, vn=P, out=P, lse=P, wsum=P,
             idx=P, ws=P, wsb=1 << 40, scale=0.125, dt=1, policy=0)
    a.update(kw)
    return L.h2o_chunk_step_q8(*(a[n] for n in ("q", "kc", "ks", "vc", "vs", "sc", "tp", "kn", "vn",
                                                "out", "lse", "wsum", "idx", "ws", "wsb", "B", "Hq",
                                                "Hkv", "T", "M", "d", "scale")),
                               0, a["dt"], a["policy"], None)


@pytest.mark.parametrize("kw,code", SHAPE_REFUSALS + [
    (dict(T=17), EINVAL), (dict(policy=-1), EINVAL), (dict(policy=1, tp=None), EINVAL),
] + [(dict([(n, None)]), EINVAL) for n in ("q", "kc", "ks", "vc", "vs", "sc", "kn", "vn", "out",
                                           "lse", "wsum", "idx")] +
    [(dict([(n, MIS)]), EALIGN) for n in ("q", "kc", "vs", "sc", "tp", "out", "idx", "ws")], ids=str)
def test_step_rejects(L, kw, code):
    if kw == dict(M=-1):
        code = EINVAL
    assert _step(L, **kw) == code


def test_policy_scratch_is_part_of_the_step(L):
    n = [L.h2o_q8_workspace_bytes(2, 4, 2, 8, 64, 64, 1, p) for p in range(3)]
    assert 0 <= n[0] < n[2] < n[1]
    assert _step(L, B=2, M=64, policy=1, wsb=n[1] - 1) == EWS
    assert L.h2o_q8_workspace_bytes(2, 4, 2, 8, 64, 64, 1, 3) == 0
    assert L.h2o_q8_workspace_bytes(2, 4, 2, 8, 64, 64, 5, 0) == 0
    assert L.h2o_q8_workspace_bytes(2, 5, 2, 8, 64, 64, 1, 0) == 0
    assert L.h2o_tree_workspace_bytes(2, 5, 2, 8, 64, 64, 1) == 0
    assert L.h2o_tree_workspace_bytes(2, 4, 2, 8, 64, 64, 9) == 0


def _tree(L, **kw):
    a = dict(SIZES, q=P, kc=P, ks=None, vc=P, vs=None, kn=P, vn=P, par=P, out=P, lse=P, ws=P,
             wsb=1 << 40, scale=0.125, dt=1)
    a.update(kw)
    return L.h2o_sdpa_tree(*(a[n] for n in ("q", "kc", "ks", "vc", "vs", "kn", "vn", "par", "out",
                                            "lse", "ws", "wsb", "B", "Hq", "Hkv", "T", "M", "d",
                                            "scale", "dt")), None)


@pytest.mark.parametrize("kw,code", SHAPE_REFUSALS + [
    (dict(ks=P), EINVAL), (dict(vs=P), EINVAL),
] + [(dict([(n, None)]), EINVAL) for n in ("q", "kc", "vc", "kn", "vn", "par", "out", "lse")] +
    [(dict([(n, MIS)]), EALIGN) for n in ("q", "kc", "vc", "kn", "vn", "par", "out", "lse", "ws")] +
    [(dict(ks=MIS, vs=P), EALIGN), (dict(ks=P, vs=MIS), EALIGN)], ids=str)
def test_tree_rejects(L, kw, code):
    assert _tree(L, **kw) == code


def _accept(L, **kw):
    a = dict(SIZES, A=3, q=P, kc=P, ks=None, kn=P, vn=P, lse=P, path=P, ka=P, va=P, wsum=P, ws=P,
             wsb=1 << 40, scale=0.125, dt=1)
    a.update(kw)
    return L.h2o_tree_accept(*(a[n] for n in ("q", "kc", "ks", "kn", "vn", "lse", "path", "ka", "va",
                                              "wsum", "ws", "wsb", "B", "Hq", "Hkv", "T", "M", "A",
                                              "d", "scale", "dt")), None)


@pytest.mark.parametrize("kw,code", SHAPE_REFUSALS + [
    (dict(A=0), EINVAL), (dict(A=9), EINVAL),
] + [(dict([(n, None)]), EINVAL) for n in ("q", "kc", "kn", "vn", "lse", "path", "ka", "va", "wsum")] +
    [(dict([(n, MIS)]), EALIGN) for n in ("q", "kc", "ks", "kn", "vn", "lse", "path", "ka", "va",
                                          "wsum", "ws")], ids=str)
def test_accept_rejects(L, kw, code):
    assert _accept(L, **kw) == code


@pytest.mark.skipif(torch.cuda.is_available(), reason="a device is visible")
def test_no_device_is_reported(L):
    for rc in (_quant(L, "h2o_kv_quantize"), _quant(L, "h2o_kv_dequantize"), _attend(L), _evict(L),
               _step(L), _tree(L), _tree(L, ks=P, vs=P), _accept(L)):
        assert rc == H.H2O_ENODEVICE


def test_binding_checks_shapes_and_types():
    z = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt)
    k8, sc, rows = z(1, 2, 16, 64, dt=torch.int8), z(1, 2, 16), z(1, 2, 8, 64)
    with pytest.raises(TypeError):
        H.h2o_kv_quantize(rows, rows, z(1, 2, 16, 64), sc, k8, sc)
    with pytest.raises(ValueError):
        H.h2o_kv_quantize(rows, rows, k8, z(1, 2, 15), k8, sc)
    with pytest.raises(ValueError):
        H.h2o_kv_quantize(rows, rows, k8, sc, k8, sc, idx=z(1, 2, 8, dt=torch.int64))
    with pytest.raises(ValueError):
        H.h2o_kv_dequantize(k8, sc, k8, sc, rows, z(1, 2, 8, 64, dt=torch.bfloat16))
    q, out, lse = z(1, 4, 8, 64), z(1, 4, 8, 64), z(1, 4, 8)
    par, ws = z(1, 8, dt=torch.int32), z(1 << 20, dt=torch.uint8)
    with pytest.raises(TypeError):       # codes without scales
        H.h2o_sdpa_tree(q, k8, k8, rows, rows, par, out, lse, ws)
    with pytest.raises(ValueError):
        H.h2o_sdpa_tree(q, k8, k8, rows, rows, par, out, lse, ws, k_scales=sc)
    with pytest.raises(ValueError):
        H.h2o_sdpa_tree(q, k8, k8, rows, rows, z(1, 7, dt=torch.int32), out, lse, ws, k_scales=sc,
                        v_scales=sc)
    with pytest.raises(ValueError):
        H.h2o_tree_accept(q, k8, rows, rows, lse, par[:, :3], z(1, 2, 3, 64), z(1, 2, 3, 64),
                          z(1, 2, 18), ws, k_scales=sc)
    with pytest.raises(ValueError):      # host tensors
        H.h2o_kv_quantize(rows, rows, k8, sc, k8, sc)


class _Elsewhere:
    """A stand-in for a contiguous tensor on a device (-1: the host)."""

    def __init__(self, device, contiguous=True):
        self.device, self.contiguous = device, contiguous

    def get_device(self):
        return self.device

    def is_contiguous(self):
        return self.contiguous

    def data_ptr(self):
        return 16 + self.device


def test_binding_refuses_other_devices_and_strides(monkeypatch):
    monkeypatch.setattr(H, "_device_number", lambda: 1)
    assert H._devs((_Elsewhere(1), "a"), (None, "b"), (_Elsewhere(1), "c")) == [17, None, 17]
    for bad, what in (((_Elsewhere(1), _Elsewhere(0)), "device 0"), ((_Elsewhere(2),), "device 2"),
                      ((_Elsewhere(-1),), "device tensor"), ((_Elsewhere(1), _Elsewhere(-1)), "device tensor"),
                      ((_Elsewhere(1, False),), "contiguous")):
        with pytest.raises(ValueError, match=what):
            H._devs(*((t, "x") for t in bad))

"""The insert after an accepted path: its definition, and its refusals before the device
is touched."""
import os

import numpy as np
import pytest
import torch

import oracle
from paper_2608_19920_amd import h2o as H

P, MIS = 0x10000, 0x10004
POLICIES = ("h2o", "h2o_norm", "h2o_orig")


def _state(seed, B=3, Hkv=2, M=20, A=5, d=8):
    rng = np.random.default_rng(seed)
    f = lambda *s: rng.standard_normal(s).astype(np.float32)
    return dict(k_cache=f(B, Hkv, M, d), v_cache=f(B, Hkv, M, d),
                scores=rng.permutation(B * Hkv * M).reshape(B, Hkv, M).astype(np.float32),
                token_pos=rng.integers(0, 50, (B, Hkv, M)).astype(np.int32),
                k_acc=f(B, Hkv, A, d), v_acc=f(B, Hkv, A, d),
                wsum=rng.random((B, Hkv, M + A)).astype(np.float32))


@pytest.mark.parametrize("policy", POLICIES)
def test_full_paths_are_the_plain_insert(policy):
    x = _state(1)
    path = np.tile(np.arange(5, dtype=np.int32), (3, 1))
    got = oracle.tree_insert(**x, path=path, pos0=np.full(3, 60), T=9, policy=policy)
    want = oracle.evict_insert(x["k_cache"], x["v_cache"], x["scores"], x["token_pos"], x["k_acc"],
                               x["v_acc"], x["wsum"], 5, 60, policy)
    for g, w in zip(got, want):
        np.testing.assert_array_equal(g, w)


@pytest.mark.parametrize("policy", POLICIES)
def test_ragged_paths(policy):
    """Two of five, none, and four of five tokens."""
    x = _state(2)
    path = np.array([[3, -1, 7, -1, 9], [-1, 9, 100, -5, 2 ** 31 - 1], [0, 1, 2, 3, -1]], np.int32)
    pos0 = np.array([60, 70, 80])
    kc, vc, sc, tp, idx = oracle.tree_insert(**x, path=path, pos0=pos0, T=9, policy=policy)
    for n, after in (("k_cache", kc), ("v_cache", vc), ("scores", sc), ("token_pos", tp)):
        np.testing.assert_array_equal(x[n][1], after[1])
        assert ((x[n] != after).reshape(3, 2, 20, -1).any(-1).sum(-1) <= [[2], [0], [4]]).all()
    assert (idx[0, :, [1, 3, 4]] == -1).all() and (idx[1] == -1).all() and (idx[2, :, 4] == -1).all()
    for h in range(2):
        a, c = idx[0, h, 0], idx[0, h, 2]
        assert 0 <= a < c
        assert tp[0, h, a] == 60 and tp[0, h, c] == 61 and tp[2, h, idx[2, h, 3]] == 83
        np.testing.assert_array_equal(kc[0, h, c], x["k_acc"][0, h, 2])
        assert sc[0, h, c] == x["wsum"][0, h, 20 + 2]
        if policy == "h2o":
            np.testing.assert_array_equal([a, c], np.sort(np.argsort(x["scores"][0, h])[:2]))


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(H.LIB_PATH):
        pytest.skip("libh2o.so not built")
    return H.lib()


def _insert(L, **kw):
    a = dict(kc=P, ks=None, vc=P, vs=None, sc=P, tp=P, ka=P, va=P, wsum=P, path=P, pos0=P, idx=P,
             B=1, Hkv=2, M=16, T=8, A=3, d=64, dt=1, policy=0, ws=None, wsb=0)
    a.update(kw)
    return L.h2o_tree_insert(*a.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(dt=2), H.H2O_EDTYPE), (dict(d=96), H.H2O_ESHAPE), (dict(B=0), H.H2O_ESHAPE),
    (dict(T=0), H.H2O_EINVAL), (dict(A=0), H.H2O_EINVAL), (dict(A=9), H.H2O_EINVAL),
    (dict(M=2), H.H2O_EINVAL), (dict(policy=3), H.H2O_EINVAL),
    (dict(policy=1, tp=None), H.H2O_EINVAL), (dict(pos0=None), H.H2O_EINVAL),
    (dict(ks=P), H.H2O_EINVAL), (dict(vs=P), H.H2O_EINVAL), (dict(policy=1), H.H2O_EWORKSPACE),
    (dict(policy=2, ws=P, wsb=16), H.H2O_EWORKSPACE), (dict(policy=2, ws=MIS, wsb=1 << 20), H.H2O_EALIGN),
    (dict(B=1 << 20, M=512, T=256, A=256), H.H2O_ESHAPE), (dict(B=32768, Hkv=2), H.H2O_ESHAPE),
] + [(dict([(n, None)]), H.H2O_EINVAL) for n in ("kc", "vc", "sc", "ka", "va", "wsum", "path", "idx")]
    + [(dict([(n, MIS)]), H.H2O_EALIGN) for n in ("kc", "vc", "sc", "tp", "ka", "va", "wsum", "path",
                                                  "pos0", "idx")]
    + [(dict(ks=MIS, vs=P), H.H2O_EALIGN), (dict(ks=P, vs=MIS), H.H2O_EALIGN)], ids=str)
def test_insert_rejects(L, kw, code):
    assert _insert(L, **kw) == code


@pytest.mark.skipif(torch.cuda.is_available(), reason="a device is visible")
def test_no_device_is_reported(L):
    assert _insert(L) == H.H2O_ENODEVICE
    assert _insert(L, tp=None, pos0=None) == H.H2O_ENODEVICE
    assert _insert(L, ks=P, vs=P) == H.H2O_ENODEVICE


def test_binding_checks_shapes_and_types():
    z = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt)
    i = lambda *s: z(*s, dt=torch.int32)
    good = dict(k_cache=z(2, 1, 16, 64), v_cache=z(2, 1, 16, 64), scores=z(2, 1, 16),
                token_pos=i(2, 1, 16), k_acc=z(2, 1, 3, 64), v_acc=z(2, 1, 3, 64), wsum=z(2, 1, 19),
                path=i(2, 3), pos0=i(2), evict_idx=i(2, 1, 3), T=8)
    for kw, err in ((dict(path=i(1, 3)), ValueError), (dict(path=z(2, 3)), ValueError),
                    (dict(pos0=i(1)), ValueError), (dict(pos0=z(2)), ValueError),
                    (dict(evict_idx=i(2, 1, 4)), ValueError), (dict(wsum=z(2, 1, 18)), ValueError),
                    (dict(v_acc=z(2, 1, 2, 64)), ValueError), (dict(scores=z(2, 1, 15)), ValueError),
                    (dict(k_scales=z(2, 1, 16)), ValueError),
                    (dict(k_scales=z(2, 1, 16), v_scales=z(2, 1, 16)), TypeError),
                    (dict(v_cache=z(2, 1, 15, 64)), ValueError),
                    (dict(k_acc=z(2, 1, 3, 64, dt=torch.bfloat16)), TypeError),
                    (dict(), ValueError)):                   # host tensors
        with pytest.raises(err):
            H.h2o_tree_insert(**{**good, **kw})

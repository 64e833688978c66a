"""The 8-bit cache where weights and values differ by many powers of two: what a query
hardly attends costs what it does attend no accuracy.

The values enter as codes, exactly. Their weights are rounded, each on its own, by at
most 2^-11 of their size (small ones by 2^-11 of the largest together), the output by at
most 2^-8 of its size: 2^-8 + 2^-11 normwise, by query head; scores are off by 2^-16 here."""
import numpy as np
import pytest
import torch

import oracle
from paper_2608_19920_amd import h2o as H
import _gpu as U
from _q8tree import close, dev, dev_cache, inputs

pytestmark = pytest.mark.gpu

TOL = 2.0 ** -8 + 2.0 ** -11
BF = torch.bfloat16


def _weights(x, log2_weights):
    """Cache keys whose scores are, in log2 units and for every query, those given [M]
    (plus a spread of about a unit): the queries share a direction."""
    d = x["q"].shape[-1]
    u = np.zeros(d, np.float32)
    u[0] = 8.0
    x["q"] *= np.float32(0.25)
    x["q"][..., 0] = u[0]
    x["k_cache"] = (0.5 * x["k_cache"]).astype(np.float32)
    x["k_cache"][..., 0] = 0.0
    x["k_new"][..., 0] = 0.0
    q = x["q"].reshape(*x["k_cache"].shape[:2], -1, d)
    # the other elements' part of the score is small against what is asked for
    need = np.asarray(log2_weights, np.float64) * np.log(2) / (float(x["scale"]) * 8.0)
    x["k_cache"][..., 0] = need.astype(np.float32)
    assert q.shape[1] == x["k_cache"].shape[1]


def _coded(x):
    x["q"] = torch.from_numpy(x["q"]).to(BF).float().numpy()
    for n in "kv":
        x[n + "_new"] = torch.from_numpy(x[n + "_new"]).to(BF).float().numpy()
        x[n + "_codes"], x[n + "_scales"] = oracle.quantize(x[n + "_cache"])
        x[n + "_values"] = oracle.dequantize(x[n + "_codes"], x[n + "_scales"])


def _attend(x, what):
    B, Hq, T, d = x["q"].shape
    Hkv, M = x["k_cache"].shape[1:3]
    args = (x["q"], x["k_values"], x["v_values"], x["k_new"], x["v_new"])
    new = [dev(x[n], BF) for n in ("q", "k_new", "v_new")]
    b = H.alloc_step(B, Hq, Hkv, T, M, d, BF, q8=True)
    b["workspace"].fill_(255)
    U.say("attend", what)
    H.h2o_sdpa_chunk_q8(new[0], *dev_cache(x), *new[1:], b["out"], b["lse"], b["wsum"],
                        b["workspace"], float(x["scale"]))
    torch.cuda.synchronize()
    o, l, w = oracle.sdpa_chunk(*args, x["scale"])
    close("bf16", what, lse=(b["lse"], l), wsum=(b["wsum"], w))
    e = oracle.rel_err(U.to_np(b["out"]), o, (-2, -1))
    U.say(f"  {what} out {e:.2e} (tol {TOL:.2e})")
    assert e <= TOL, f"{what}: out error {e:.3e}"
    if 1 < T <= 64:                # the same chunk as a chain of nodes
        parents = np.tile(np.arange(-1, T - 1, dtype=np.int32), (B, 1))
        c = dev_cache(x)
        out, lse = torch.empty_like(b["out"]), torch.empty_like(b["lse"])
        ws = torch.full((max(16, H.h2o_tree_workspace_bytes(B, Hq, Hkv, T, M, d, BF)),), 255,
                        dtype=torch.uint8, device=U.DEV)
        H.h2o_sdpa_tree(new[0], c[0], c[2], *new[1:], dev(parents), out, lse, ws, float(x["scale"]),
                        k_scales=c[1], v_scales=c[3])
        e = oracle.rel_err(U.to_np(out), o, (-2, -1))
        U.say(f"  {what} tree {e:.2e}")
        assert e <= TOL, f"{what}: tree error {e:.3e}"


SHAPES = [  # B, Hq, Hkv, d, M, T
    (1, 8, 2, 128, 2048, 1), (2, 7, 1, 64, 1501, 1), (1, 8, 2, 128, 2048, 9), (1, 4, 2, 64, 700, 40),
    (1, 16, 4, 64, 900, 150), (1, 8, 2, 128, 1100, 300),
]


@pytest.mark.parametrize("where", ["first", "middle", "last"])
@pytest.mark.parametrize("log2_size", [8, 14, 20, 60])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_a_large_value_row_of_next_to_no_weight(shape, log2_size, where):
    """One value row 2^n times the others, at a weight of 2^-(n + 30) of theirs."""
    B, Hq, Hkv, d, M, T = shape
    x = inputs(*shape, "bf16", seed=log2_size)
    at = {"first": 0, "middle": M // 2 + 5, "last": M - 1}[where]
    s = np.zeros(M)
    s[at] = -(log2_size + 30)
    _weights(x, s)
    x["v_cache"][:, :, at] *= np.float32(2.0 ** log2_size)
    _coded(x)
    _attend(x, f"{shape} 2^{log2_size} {where}")


@pytest.mark.parametrize("rows", [(0, 64), (640, 704), (-64, None)])
@pytest.mark.parametrize("log2_base,log2_size,log2_score", [(0, 60, -90), (0, 20, -120), (70, 6, -100),
                                                            (70, 8, -300)])
@pytest.mark.parametrize("shape", SHAPES + [(1, 2, 1, 64, 5000, 2)], ids=lambda s: "-".join(map(str, s)))
def test_tiles_of_large_values_that_nobody_attends(shape, log2_base, log2_size, log2_score, rows):
    """Rows of 2^base, and a run of rows 2^size larger."""
    x = inputs(*shape, "bf16", seed=-log2_score)
    s = np.zeros(shape[4])
    s[slice(*rows)] = log2_score
    _weights(x, s)
    x["v_cache"] *= np.float32(2.0 ** log2_base)
    x["v_cache"][:, :, slice(*rows)] *= np.float32(2.0 ** log2_size)
    _coded(x)
    _attend(x, f"{shape} 2^{log2_base} 2^{log2_size} at 2^{log2_score} {rows}")


@pytest.mark.parametrize("where", [0, -1])
@pytest.mark.parametrize("log2_weight", [16, 24, 32])
@pytest.mark.parametrize("shape", SHAPES[:4] + [(1, 4, 1, 64, 40000, 1), (1, 4, 1, 128, 20000, 20)],
                         ids=lambda s: "-".join(map(str, s)))
def test_a_sink(shape, log2_weight, where):
    """A slot that takes nearly all the weight and has no value: the output is what the
    others add at 2^-n each."""
    B, Hq, Hkv, d, M, T = shape
    x = inputs(*shape, "bf16", seed=log2_weight)
    s = np.zeros(M)
    s[where] = log2_weight
    _weights(x, s)
    x["v_cache"][:, :, where] = 0.0
    x["v_new"] *= np.float32(2.0 ** -log2_weight)
    _coded(x)
    _attend(x, f"{shape} sink 2^{log2_weight} at {where}")


@pytest.mark.slow
@pytest.mark.parametrize("log2_weight", [18, 22, 26])
@pytest.mark.parametrize("shape", [(1, 4, 1, 64, 60000, 1), (1, 2, 1, 128, 60000, 9), (1, 4, 1, 64, 60000, 40)],
                         ids=lambda s: "-".join(map(str, s)))
def test_a_sink_and_a_crowd(shape, log2_weight):
    """A slot with nearly all the weight, and 60,000 others of 2^-n each that agree on a
    value: small weights add up."""
    B, Hq, Hkv, d, M, T = shape
    x = inputs(*shape, "bf16", seed=log2_weight)
    s = np.zeros(M)
    s[1234] = log2_weight
    _weights(x, s)
    x["v_cache"][:] = 0.0
    x["v_cache"][..., 0] = 1.0
    x["v_cache"][:, :, 1234] = np.eye(d, dtype=np.float32)[1]
    _coded(x)
    _attend(x, f"{shape} crowd 2^-{log2_weight}")


@pytest.mark.parametrize("d,T", [(64, 1), (128, 1), (64, 40), (128, 9), (128, 300)])
def test_values_against_their_weights(d, T):
    """Value rows from 2^-40 to 2^40 whose weights fall as they grow."""
    shape = (1, 8, 2, d, 900, T)
    x = inputs(*shape, "bf16", seed=d + T)
    e = np.round(80 * np.arange(900) / 900 - 40)
    _weights(x, -1.25 * e)
    x["v_cache"] *= np.exp2(e).astype(np.float32)[:, None]
    _coded(x)
    _attend(x, f"against {shape}")


@pytest.mark.parametrize("size", [2.0 ** -117, 2.0 ** -60, 2.0 ** 60, 2.0 ** 90])
@pytest.mark.parametrize("chunk_too", [False, True])
@pytest.mark.parametrize("shape", SHAPES[:1] + SHAPES[2:5], ids=lambda s: "-".join(map(str, s)))
def test_values_of_one_far_size(shape, chunk_too, size):
    """All value rows of the cache, or all there are, far from 1; the chunk's scores are
    12 (log2) above the cache's."""
    x = inputs(*shape, "bf16", seed=3)
    _weights(x, np.full(shape[4], -12.0))
    x["v_cache"] *= np.float32(size)
    if chunk_too:
        x["v_new"] *= np.float32(size)
    _coded(x)
    _attend(x, f"{shape} size {size} {chunk_too}")


@pytest.mark.parametrize("T", [1, 5, 200])
@pytest.mark.parametrize("slots", [slice(37, 38), slice(0, 64), slice(250, 300)])
def test_a_nan_value_row_reaches_the_output_alone(T, slots):
    """The output of its KV head is NaN; lse, weights and the other head are as without."""
    x = inputs(1, 4, 2, 64, 300, T, "bf16", seed=T)
    new = [dev(x[n], BF) for n in ("q", "k_new", "v_new")]
    runs = []
    for nan in (False, True):
        if nan:
            x["v_scales"][0, 1, slots] = np.nan
        b = H.alloc_step(1, 4, 2, T, 300, 64, BF, q8=True)
        H.h2o_sdpa_chunk_q8(new[0], *dev_cache(x), *new[1:], b["out"], b["lse"], b["wsum"],
                            b["workspace"], float(x["scale"]))
        runs.append(b)
    a, b = runs
    assert torch.equal(a["out"][:, :2], b["out"][:, :2]) and torch.isnan(b["out"][:, 2:]).all()
    close("bf16", "nan value", lse=(b["lse"], U.to_np(a["lse"])), wsum=(b["wsum"], U.to_np(a["wsum"])))

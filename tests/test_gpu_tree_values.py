"""Trees over values far from 1 with scores that rise along the keys: the weights of the
keys before a maximum are small, and finite values give finite results.

Weights are two bf16 terms (2^-16), the output is rounded by at most 2^-8 of its size, the
scores are off by 2^-16 or so here: 2^-8 + 2^-11 normwise by query head leaves room for the
sums."""
import numpy as np
import pytest
import torch

import oracle
from paper_2608_19920_amd import h2o as H
import _gpu as U
from _q8tree import dev, inputs

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


@pytest.mark.parametrize("size", [2.0 ** -90, 1.0, 2.0 ** 70, 2.0 ** 90])
@pytest.mark.parametrize("rise", [12, 60])
@pytest.mark.parametrize("B,Hq,Hkv,d,M,T", [(1, 8, 2, 64, 300, 9), (1, 16, 2, 64, 1500, 150),
                                            (2, 7, 1, 128, 900, 30), (1, 4, 4, 128, 0, 200)])
def test_scores_that_rise(B, Hq, Hkv, d, M, T, rise, size):
    x = inputs(B, Hq, Hkv, d, M, T, "bf16", seed=rise)
    # every query has 8 in its first element, keys there what gives their score (log2)
    x["q"] *= np.float32(0.25)
    x["q"][..., 0] = 8.0
    # a ladder of 4 steps over cache and nodes
    ladder = np.repeat(np.arange(4) - 3, -(-(M + T) // 4))[:M + T] * (rise / 3)
    need = (ladder * np.log(2) / (float(x["scale"]) * 8)).astype(np.float32)
    for n, part in (("k_cache", need[:M]), ("k_new", need[M:])):
        x[n] = (0.5 * x[n]).astype(np.float32)
        x[n][..., 0] = part
    rnd = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(BF).float().numpy()
    for n in ("v_cache", "v_new"):
        x[n] = rnd(x[n] * np.float32(size))
    for n in ("q", "k_cache", "k_new"):
        x[n] = rnd(x[n])
    parents = np.tile(np.arange(-1, T - 1, dtype=np.int32), (B, 1))
    out = torch.empty(B, Hq, T, d, dtype=BF, device=U.DEV)
    lse = torch.empty(B, Hq, T, device=U.DEV)
    ws = torch.full((max(16, H.h2o_tree_workspace_bytes(B, Hq, Hkv, T, M, d, BF)),), 255,
                    dtype=torch.uint8, device=U.DEV)
    U.say("tree", B, Hq, Hkv, d, M, T, rise, size)
    H.h2o_sdpa_tree(dev(x["q"], BF), dev(x["k_cache"], BF), dev(x["v_cache"], BF), dev(x["k_new"], BF),
                    dev(x["v_new"], BF), dev(parents), out, lse, ws, float(x["scale"]))
    o, l, _ = oracle.sdpa_chunk(x["q"], x["k_cache"], x["v_cache"], x["k_new"], x["v_new"], x["scale"])
    assert torch.isfinite(out).all()
    e = oracle.rel_err(U.to_np(out), o, (-2, -1))
    assert e <= 2.0 ** -8 + 2.0 ** -11, e
    assert np.abs(U.to_np(lse) - l).max() <= 1e-4 * max(1.0, np.abs(l).max())

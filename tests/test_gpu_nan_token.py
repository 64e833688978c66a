"""A NaN in one key of a bf16 cache and the token step: the query that reads it gets
NaN, the scores of the head's other slots and the other heads are as without it."""
import numpy as np
import pytest
import torch

from paper_2608_19920_amd import h2o as H
from paper_2608_19920_amd import workloads as W
import _gpu as U

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fused", [True, False])
@pytest.mark.parametrize("M", [300, 5000])      # one finish kernel; combine and insert
@pytest.mark.parametrize("G,d", [(4, 64), (7, 128), (1, 128)])
def test_a_nan_key_costs_no_other_slot_its_score(G, d, M, fused):
    B, Hkv = 2, 2
    x = W.make_inputs(W.custom("t", B=B, Hq=G * Hkv, Hkv=Hkv, d=d, M=M, T=1, dtype="bf16",
                               heavy_frac=0.02), seed=M + G)
    dev = lambda a, t: torch.from_numpy(np.ascontiguousarray(a)).to(U.DEV).to(t)
    runs = []
    for nan in (False, True):
        st = dict(k_cache=dev(x["k_cache"], torch.bfloat16), v_cache=dev(x["v_cache"], torch.bfloat16),
                  scores=dev(x["scores"], torch.float32), token_pos=dev(x["token_pos"], torch.int32))
        if nan:
            st["k_cache"][1, 1, 7, 3] = float("nan")
        b = H.alloc_step(B, G * Hkv, Hkv, 1, M, d, torch.bfloat16)
        U.say("token step", G, d, M, nan)
        H.step(st, *(dev(x[n], torch.bfloat16) for n in ("q", "k_new", "v_new")), b, int(x["pos0"]),
               float(x["scale"]), fused=fused)
        torch.cuda.synchronize()
        runs.append((b, st))
    (b0, s0), (b1, s1) = runs
    bad = torch.zeros(B, Hkv, dtype=torch.bool)
    bad[1, 1] = True
    heads = bad.repeat_interleave(G, 1)
    for n in ("out", "lse"):
        assert torch.equal(b0[n].cpu()[~heads], b1[n].cpu()[~heads]), n
    for n, t0, t1 in (("wsum", b0["wsum"], b1["wsum"]), ("scores", s0["scores"], s1["scores"])):
        assert torch.equal(t0.cpu()[~bad], t1.cpu()[~bad]), n
    assert torch.isnan(b1["out"].cpu()[heads]).all()
    assert (b1["lse"].cpu()[heads] == -float("inf")).all()
    w = b1["wsum"].cpu()[1, 1]
    slots = [j for j in range(M + 1) if j != 7]
    assert not w[slots].any()
    kept = torch.ones(M, dtype=torch.bool)
    kept[7] = False
    kept[b1["evict_idx"].cpu()[1, 1, 0]] = False
    assert torch.equal(s1["scores"].cpu()[1, 1][kept], torch.from_numpy(x["scores"])[1, 1][kept])

"""Inputs and comparisons shared by the GPU tests of the 8-bit cache and the tree."""
import numpy as np
import torch

import oracle
from paper_2608_19920_amd import h2o as H
from paper_2608_19920_amd import workloads as W
import _gpu as U

# lse and the summed weights of a bf16 call are float32 sums over exact products of
# bf16 values and codes: a logit is off by d * 2^-24 * scale * sum_d |q k| at most,
# about 2e-4 with keys scaled x4 (the premise of _gpu.SEL_TOL), in the weights as a
# relative error. 1e-3 and, against lse of a few units, 1e-4 leave room for the sums.
WSUM_TOL, LSE_TOL = {"f32": 1e-5, "bf16": 1e-3}, {"f32": 1e-6, "bf16": 1e-4}


def inputs(B, Hq, Hkv, d, M, T, dtype, seed, heavy=0.05):
    """numpy arrays of the chunk's call; the cache also as codes and scales."""
    x = W.make_inputs(W.custom("t", B=B, Hq=Hq, Hkv=Hkv, d=d, M=M, T=T, dtype=dtype,
                               heavy_frac=heavy), seed=seed)
    for n in "kv":
        x[n + "_codes"], x[n + "_scales"] = oracle.quantize(x[n + "_cache"])
        x[n + "_values"] = oracle.dequantize(x[n + "_codes"], x[n + "_scales"])
    return x


def dev(a, dt=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).to(U.DEV)
    return (t if dt is None else t.to(dt)).contiguous()


def dev_cache(x):
    return [dev(x[n]) for n in ("k_codes", "k_scales", "v_codes", "v_scales")]


def guarded(n, *shape, dtype=torch.float32, fill=7.0):
    """A tensor with `n` elements of `fill` behind it: (tensor, its tail)."""
    size = int(np.prod(shape))
    buf = torch.full((size + n,), fill, dtype=dtype, device=U.DEV)
    return buf[:size].view(*shape), buf[size:]


def close(dtype, what, **pairs):
    """out normwise per (b, head) slice as everywhere, lse and wsum as above."""
    for name, (g, r) in pairs.items():
        g = U.to_np(g)
        assert np.isfinite(g).all(), f"{what}: {name} not finite"
        if g.size == 0:
            continue
        if name == "wsum":
            e, tol = oracle.elem_err(g, r, (-1,)), WSUM_TOL[dtype]
        elif name == "lse":
            # a row that sees itself alone has an lse anywhere near 0: against 1 there
            e, tol = float((np.abs(g - r) / np.maximum(1.0, np.abs(r))).max()), LSE_TOL[dtype]
        else:
            e, tol = oracle.rel_err(g, r, (-2, -1)), U.TOL[dtype]
        U.say(f"  {what} {name} {e:.2e} (tol {tol})")
        assert e <= tol, f"{what}: {name} error {e:.3e} above {tol}"

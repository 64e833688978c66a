"""8-bit cache and tree at sizes that take the large blocks, several key ranges and
several row ranges, offsets past 32 bits, and a stream of their own."""
import numpy as np
import pytest
import torch

import oracle
from paper_2608_19920_amd import h2o as H
import _gpu as U
import test_gpu_q8 as steps
from _q8tree import close, dev, dev_cache, inputs

pytestmark = pytest.mark.gpu

CASES = [  # B, Hq, Hkv, d, M, T, dtype
    (1, 8, 2, 128, 2100, 260, "bf16"),      # 1,040 rows a head
    (2, 16, 2, 64, 1500, 150, "bf16"),      # 1,200 rows a head, blocks of every shape
    (1, 32, 2, 64, 4000, 70, "bf16"),       # 16 query heads a KV head
    (2, 28, 4, 128, 6000, 19, "bf16"),      # many key ranges
    (1, 16, 16, 128, 700, 640, "bf16"),     # as many chunk keys as slots
    (1, 8, 2, 128, 900, 120, "f32"),
    (3, 4, 4, 64, 3000, 33, "f32"),
]


@pytest.mark.slow
@pytest.mark.parametrize("case", CASES, ids=["-".join(map(str, c)) for c in CASES])
def test_attention(case):
    *shape, dtype = case
    B, Hq, Hkv, d, M, T = shape
    x, tdt = inputs(*shape, dtype, seed=M), U.TDT[dtype]
    b = H.alloc_step(B, Hq, Hkv, T, M, d, tdt, q8=True)
    b["workspace"].fill_(255)
    U.say("attend", case)
    H.h2o_sdpa_chunk_q8(dev(x["q"], tdt), *dev_cache(x), dev(x["k_new"], tdt),
                        dev(x["v_new"], tdt), b["out"], b["lse"], b["wsum"], b["workspace"],
                        float(x["scale"]))
    torch.cuda.synchronize()
    o, l, w = oracle.sdpa_chunk(x["q"], x["k_values"], x["v_values"], x["k_new"], x["v_new"],
                                x["scale"])
    close(dtype, str(case), out=(b["out"], o), lse=(b["lse"], l), wsum=(b["wsum"], w))


@pytest.mark.parametrize("dtype,q8", [("bf16", False), ("bf16", True), ("f32", True)])
def test_chain_of_a_large_tree(dtype, q8):
    """A chain is the causal chunk: 200 nodes of it, then a path of 150 of them."""
    B, Hq, Hkv, d, M, T, A = 1, 16, 2, 64, 2500, 200, 150
    x, tdt = inputs(B, Hq, Hkv, d, M, T, dtype, seed=1), U.TDT[dtype]
    c = dev_cache(x) if q8 else [dev(x["k_cache"], tdt), None, dev(x["v_cache"], tdt), None]
    q, kn, vn = dev(x["q"], tdt), dev(x["k_new"], tdt), dev(x["v_new"], tdt)
    new = lambda *s, dt=torch.float32: torch.empty(*s, dtype=dt, device=U.DEV)
    out, lse = new(B, Hq, T, d, dt=tdt), new(B, Hq, T)
    ws = torch.full((H.h2o_tree_workspace_bytes(B, Hq, Hkv, T, M, d, tdt),), 255,
                    dtype=torch.uint8, device=U.DEV)
    H.h2o_sdpa_tree(q, c[0], c[2], kn, vn, dev(np.arange(-1, T - 1, dtype=np.int32)[None]), out, lse,
                    ws, float(x["scale"]), k_scales=c[1], v_scales=c[3])
    kv = [x[n + ("_values" if q8 else "_cache")] for n in "kv"]
    o, l, _ = oracle.sdpa_chunk(x["q"], *kv, x["k_new"], x["v_new"], x["scale"])
    close(dtype, "chain", out=(out, o), lse=(lse, l))
    ka, va, wsum = new(B, Hkv, A, d, dt=tdt), new(B, Hkv, A, d, dt=tdt), new(B, Hkv, M + A)
    ws.fill_(255)
    H.h2o_tree_accept(q, c[0], kn, vn, lse, dev(np.arange(A, dtype=np.int32)[None]), ka, va, wsum,
                      ws, float(x["scale"]), k_scales=c[1])
    cut = lambda a: a[:, :, :A]
    _, _, w = oracle.sdpa_chunk(cut(x["q"]), *kv, cut(x["k_new"]), cut(x["v_new"]), x["scale"])
    close(dtype, "path", wsum=(wsum, w))


@pytest.mark.slow
@pytest.mark.parametrize("T", [1, 21])
def test_offsets_past_32_bits(T):
    """Codes of more than 2^31 bytes, the last head alone with data: written, attended,
    read back and evicted there."""
    B, Hq, Hkv, d, M = 2, 72, 36, 128, 1 << 18
    kc, vc = (torch.zeros(B, Hkv, M, d, dtype=torch.int8, device=U.DEV) for _ in range(2))
    ks, vs = (torch.zeros(B, Hkv, M, device=U.DEV) for _ in range(2))
    assert kc.numel() > 1 << 31
    rng = np.random.default_rng(T)
    # the last 64 slots of the last head, the other rows of that head zeros: their score is
    # 0, their weight one each
    rows = [torch.zeros(B, Hkv, 64, d, dtype=torch.bfloat16, device=U.DEV) for _ in range(2)]
    for r in rows:
        r[-1, -1] = dev(rng.standard_normal((64, d)).astype(np.float32), torch.bfloat16)
    idx = torch.full((B, Hkv, 64), -1, dtype=torch.int32, device=U.DEV)
    idx[-1, -1] = torch.arange(M - 64, M, device=U.DEV)
    H.h2o_kv_quantize(*rows, kc, ks, vc, vs, idx=idx)
    back = [torch.zeros_like(r) for r in rows]
    H.h2o_kv_dequantize(kc, ks, vc, vs, *back, idx=idx)
    for r, g in zip(rows, back):
        c, s = oracle.quantize(r[-1, -1].float().cpu().numpy())
        want = torch.from_numpy((c.astype(np.float32) * s[:, None])).to(torch.bfloat16)
        assert torch.equal(g[-1, -1].cpu(), want)
    q = dev(rng.standard_normal((B, Hq, T, d)).astype(np.float32), torch.bfloat16)
    kn, vn = (dev(rng.standard_normal((B, Hkv, T, d)).astype(np.float32), torch.bfloat16)
              for _ in range(2))
    b = H.alloc_step(B, Hq, Hkv, T, M, d, torch.bfloat16, q8=True)
    scores = torch.ones(B, Hkv, M, device=U.DEV)
    scores[..., M - T:] = -100.0
    U.say("step past 32 bits", T)
    H.step_q8(dict(k_codes=kc, k_scales=ks, v_codes=vc, v_scales=vs, scores=scores), q, kn, vn, b, M)
    torch.cuda.synchronize()
    # one KV head in float64: 2^18 - 64 zero rows, then the 64 rows
    kv = [np.concatenate([np.zeros((1, 1, 64, d)), oracle.dequantize(
        *oracle.quantize(r[-1:, -1:].float().cpu().numpy()))], 2) for r in rows]
    n0 = M - 64
    Q, KN, VN = (U.to_np(t) for t in (q[-1:, -2:], kn[-1:, -1:], vn[-1:, -1:]))
    s = np.einsum("gtd,jd->gtj", Q[0], np.concatenate([kv[0][0, 0, 64:], KN[0, 0]])) / np.sqrt(d)
    s[:, :, 64:] = np.where(np.tril(np.ones((T, T), bool)), s[:, :, 64:], -np.inf)
    m = np.maximum(s.max(-1, keepdims=True), 0)
    e = np.exp(s - m)
    tot = e.sum(-1, keepdims=True) + n0 * np.exp(-m)
    p = e / tot
    o = p @ np.concatenate([kv[1][0, 0, 64:], VN[0, 0]])
    close("bf16", "last head", out=(b["out"][-1:, -2:], o[None]),
          lse=(b["lse"][-1:, -2:], (m + np.log(tot))[None, :, :, 0]),
          wsum=(b["wsum"][-1:, -1:, M - 64:], p.sum((0, 1))[None, None]))
    assert torch.equal(b["evict_idx"][-1, -1].cpu(), torch.arange(M - T, M, dtype=torch.int32))
    c, sc = oracle.quantize(kn[-1, -1].float().cpu().numpy())
    assert np.array_equal(kc[-1, -1, M - T:].cpu().numpy(), c)
    assert np.array_equal(ks[-1, -1, M - T:].cpu().numpy(), sc)


def test_two_streams_at_once():
    """The same calls on two streams, each with its own buffers, give one stream's bits."""
    B, Hq, Hkv, d, M, T, A = 1, 8, 2, 64, 1200, 30, 6
    sets = []
    for seed in (1, 2):
        x = inputs(B, Hq, Hkv, d, M, T, "bf16", seed=seed)
        c = dev_cache(x)
        q, kn, vn = (dev(x[n], torch.bfloat16) for n in ("q", "k_new", "v_new"))
        par = dev(np.arange(-1, T - 1, dtype=np.int32)[None])
        path = dev(np.arange(A, dtype=np.int32)[None])

        def run(c=c, q=q, kn=kn, vn=vn, par=par, path=path):
            new = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt, device=U.DEV)
            b = H.alloc_step(B, Hq, Hkv, T, M, d, torch.bfloat16, q8=True)
            ws = new(H.h2o_tree_workspace_bytes(B, Hq, Hkv, T, M, d, torch.bfloat16), dt=torch.uint8)
            out, lse, wsum = new(B, Hq, T, d, dt=torch.bfloat16), new(B, Hq, T), new(B, Hkv, M + A)
            ka, va = (new(B, Hkv, A, d, dt=torch.bfloat16) for _ in range(2))
            for _ in range(3):
                H.h2o_sdpa_chunk_q8(q, *c, kn, vn, b["out"], b["lse"], b["wsum"], b["workspace"])
                H.h2o_sdpa_tree(q, c[0], c[2], kn, vn, par, out, lse, ws, k_scales=c[1], v_scales=c[3])
                H.h2o_tree_accept(q, c[0], kn, vn, lse, path, ka, va, wsum, ws, k_scales=c[1])
            return [b["out"], b["lse"], b["wsum"], out, lse, ka, va, wsum]

        sets.append(run)
    want = [r() for r in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = []
    for r, st in zip(sets, streams):
        with torch.cuda.stream(st):
            got.append(r())
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        for a, b in zip(g, w):
            assert torch.equal(a, b)


@pytest.mark.slow
@pytest.mark.parametrize("case", [
    (1, 2, 1, 64, 4500, 4100, "bf16", "h2o", True),      # more rows than one launch selects
    (1, 2, 2, 64, 4300, 4200, "f32", "h2o_norm", True),
    (2, 4, 2, 64, 40000, 3, "bf16", "h2o", True),        # a head's scores beyond LDS
    (1, 8, 2, 128, 33000, 300, "bf16", "h2o_norm", True),
    (2, 6, 3, 128, 9000, 1, "bf16", "h2o_orig", True),
], ids=lambda c: "-".join(map(str, c)))
def test_steps_of_many_rows_and_slots(case):
    steps.test_step_is_its_three_parts(case)


@pytest.mark.parametrize("d,T", [(64, 1), (128, 1), (64, 40), (128, 9), (128, 300)])
@pytest.mark.parametrize("rising", [True, False])
def test_values_and_scores_of_every_size(d, T, rising):
    """Value rows from 2^-40 to 2^40 and none at all, scores that rise or fall along the
    cache. The weights are off by 2^-12 of their size, or 2^-20 of the largest one; the
    output is rounded by at most 2^-8: 2^-8 + 2^-11 normwise leaves room for the sums."""
    B, Hq, Hkv, M = 1, 8, 2, 900
    x = inputs(B, Hq, Hkv, d, M, T, "bf16", seed=d + T)
    ramp = np.arange(M) / M
    if not rising:
        ramp = ramp[::-1]
    x["v_cache"] *= np.exp2(np.round(80 * ramp - 40)).astype(np.float32)[:, None]
    x["v_cache"][:, :, 100:140] = 0.0
    x["v_cache"][:, 0, :64] = 0.0
    x["k_cache"] = (0.3 * x["k_cache"] + np.float32(6 / d ** 0.5) * (ramp[:, None] - 0.5) *
                    x["q"][:, ::4, -1:, :]).astype(np.float32)
    for n in "kv":
        x[n + "_codes"], x[n + "_scales"] = oracle.quantize(x[n + "_cache"])
        x[n + "_values"] = oracle.dequantize(x[n + "_codes"], x[n + "_scales"])
    b = H.alloc_step(B, Hq, Hkv, T, M, d, torch.bfloat16, q8=True)
    bf = torch.bfloat16
    H.h2o_sdpa_chunk_q8(dev(x["q"], bf), *dev_cache(x), dev(x["k_new"], bf), dev(x["v_new"], bf),
                        b["out"], b["lse"], b["wsum"], b["workspace"], float(x["scale"]))
    o, l, w = oracle.sdpa_chunk(x["q"], x["k_values"], x["v_values"], x["k_new"], x["v_new"],
                                x["scale"])
    close("bf16", "sizes", lse=(b["lse"], l), wsum=(b["wsum"], w))
    e = oracle.rel_err(U.to_np(b["out"]), o, (-2, -1))
    assert e <= 2.0 ** -8 + 2.0 ** -11, e


@pytest.mark.parametrize("B,Hq,Hkv,d,M,T", [(1, 16, 16, 128, 700, 1), (1, 8, 2, 64, 3000, 3),
                                            (2, 4, 2, 128, 500, 20), (1, 8, 1, 64, 400, 100)])
@pytest.mark.parametrize("q8", [True, False])
def test_a_tree_is_off_by_its_rounding_alone(B, Hq, Hkv, d, M, T, q8):
    """As above, of a tree over either cache, by query head."""
    x, bf = inputs(B, Hq, Hkv, d, M, T, "bf16", seed=M), torch.bfloat16
    parents = np.tile(np.arange(-1, T - 1) // 2, (B, 1)).astype(np.int32)
    c = dev_cache(x) if q8 else [dev(x["k_cache"], bf), None, dev(x["v_cache"], bf), None]
    out = torch.empty(B, Hq, T, d, dtype=bf, device=U.DEV)
    lse = torch.empty(B, Hq, T, device=U.DEV)
    ws = torch.empty(max(16, H.h2o_tree_workspace_bytes(B, Hq, Hkv, T, M, d, bf)),
                     dtype=torch.uint8, device=U.DEV)
    H.h2o_sdpa_tree(dev(x["q"], bf), c[0], c[2], dev(x["k_new"], bf), dev(x["v_new"], bf),
                    dev(parents), out, lse, ws, float(x["scale"]), k_scales=c[1], v_scales=c[3])
    kv = [x[n + ("_values" if q8 else "_cache")] for n in "kv"]
    o, l = oracle.sdpa_tree(x["q"], *kv, x["k_new"], x["v_new"], parents, x["scale"])
    e = oracle.rel_err(U.to_np(out), o, (-2, -1))
    assert e <= 2.0 ** -8 + 2.0 ** -11, e

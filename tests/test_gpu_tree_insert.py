"""The insert after an accepted path on the GPU: batch entries that accepted different
numbers of tokens, bit for bit against the oracle, and a draft loop of such a batch."""
import numpy as np
import pytest
import torch

import oracle
from paper_2608_19920_amd import h2o as H
import _gpu as U
from _q8tree import close, dev, dev_cache, guarded, inputs

pytestmark = pytest.mark.gpu


def _paths(kind, B, T, A, rng):
    p = np.tile(np.arange(A, dtype=np.int32), (B, 1))
    if kind == "ragged":              # the first n of a path, n from 0 to A
        for b in range(B):
            p[b, (b * A) // max(1, B - 1) if B > 1 else A // 2:] = -1
    elif kind == "gaps":
        p[rng.random((B, A)) < 0.4] = -1
        p[rng.random((B, A)) < 0.1] = T
        p[0, 0], p[-1, -1] = 2 ** 31 - 1, -2 ** 31
    elif kind == "none":
        p[:] = -1
    return p


CASES = [  # B, Hkv, M, T, A, d, paths
    (1, 1, 1, 1, 1, 64, "full"), (1, 1, 1, 3, 1, 128, "none"), (3, 2, 50, 16, 5, 64, "ragged"),
    (4, 3, 333, 61, 9, 128, "gaps"), (2, 2, 100, 100, 100, 64, "gaps"), (3, 2, 700, 60, 33, 128, "ragged"),
    (2, 1, 3000, 2100, 2050, 64, "gaps"), (3, 1, 40000, 70, 65, 64, "ragged"),
    (2, 1, 36000, 5000, 4500, 64, "gaps"), (2, 2, 64, 8, 4, 64, "none"),
]


@pytest.mark.parametrize("dtype,q8", [("bf16", False), ("bf16", True), ("f32", False), ("f32", True)])
@pytest.mark.parametrize("policy", ["h2o", "h2o_norm", "h2o_orig"])
@pytest.mark.parametrize("case", CASES, ids=["-".join(map(str, c)) for c in CASES])
def test_insert(case, policy, dtype, q8):
    B, Hkv, M, T, A, d, kind = case
    rng = np.random.default_rng(M + A)
    tdt = U.TDT[dtype]
    f = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(tdt).float().numpy()
    kv, acc = [f(B, Hkv, M, d) for _ in range(2)], [f(B, Hkv, A, d) for _ in range(2)]
    # ties among the scores; ages of at least 1 for every entry
    scores = rng.integers(0, max(2, M // 3), (B, Hkv, M)).astype(np.float32)
    pos0 = rng.integers(M + 10, M + 50, B).astype(np.int32)
    tp = rng.integers(0, M + 10, (B, Hkv, M)).astype(np.int32)
    wsum = rng.random((B, Hkv, M + A)).astype(np.float32)
    path = _paths(kind, B, T, A, rng)
    rows = [oracle.quantize(x) for x in kv] if q8 else None
    cache = [dev(rows[0][0]), dev(rows[0][1]), dev(rows[1][0]), dev(rows[1][1])] if q8 else \
        [dev(kv[0], tdt), None, dev(kv[1], tdt), None]
    idx, ig = guarded(16, B, Hkv, A, dtype=torch.int32, fill=77)
    sc, sg = guarded(16, B, Hkv, M)
    pos, pg = guarded(16, B, Hkv, M, dtype=torch.int32)
    sc.copy_(dev(scores))
    pos.copy_(dev(tp))
    n = H.h2o_evict_workspace_bytes(B, Hkv, M, A, policy)
    ws, wg = guarded(64, max(n, 16), dtype=torch.uint8, fill=255)
    U.say("insert", case, policy, dtype, q8)
    H.h2o_tree_insert(cache[0], cache[2], sc, pos, dev(acc[0], tdt), dev(acc[1], tdt), dev(wsum),
                      dev(path), dev(pos0), idx, T, policy, ws, k_scales=cache[1], v_scales=cache[3])
    torch.cuda.synchronize()
    for g, v in ((ig, 77), (sg, 7), (pg, 7), (wg, 255)):
        assert (g == v).all()
    want = oracle.tree_insert(kv[0], kv[1], scores, tp, acc[0], acc[1], wsum, path, pos0, T, policy)
    np.testing.assert_array_equal(idx.cpu().numpy(), want[4])
    np.testing.assert_array_equal(sc.cpu().numpy(), want[2])
    np.testing.assert_array_equal(pos.cpu().numpy(), want[3])
    for i in range(2):
        if q8:
            c, s = oracle.quantize(want[i])
            np.testing.assert_array_equal(cache[2 * i].cpu().numpy(), c)
            np.testing.assert_array_equal(cache[2 * i + 1].cpu().numpy(), s)
        else:
            np.testing.assert_array_equal(cache[2 * i].float().cpu().numpy(), want[i])


@pytest.mark.parametrize("policy", ["h2o", "h2o_orig"])
def test_without_positions(policy):
    B, Hkv, M, A, d = 2, 2, 40, 3, 64
    rng = np.random.default_rng(0)
    f = lambda *s: rng.standard_normal(s).astype(np.float32)
    x = dict(k_cache=f(B, Hkv, M, d), v_cache=f(B, Hkv, M, d), scores=f(B, Hkv, M), token_pos=None,
             k_acc=f(B, Hkv, A, d), v_acc=f(B, Hkv, A, d), wsum=f(B, Hkv, M + A),
             path=np.array([[0, 1, -1], [2, -1, -1]], np.int32))
    g = {n: None if v is None else dev(v) for n, v in x.items()}
    idx = torch.empty(B, Hkv, A, dtype=torch.int32, device=U.DEV)
    ws = torch.empty(max(16, H.h2o_evict_workspace_bytes(B, Hkv, M, A, policy)), dtype=torch.uint8,
                     device=U.DEV)
    H.h2o_tree_insert(**g, pos0=None, evict_idx=idx, T=3, policy=policy, workspace=ws)
    want = oracle.tree_insert(**x, pos0=np.zeros(B, int), T=3, policy=policy)
    for got, w in ((g["k_cache"], want[0]), (g["v_cache"], want[1]), (g["scores"], want[2]), (idx, want[4])):
        np.testing.assert_array_equal(got.cpu().numpy(), w)


@pytest.mark.parametrize("dtype,q8,policy", [("bf16", True, "h2o"), ("f32", False, "h2o_norm"),
                                             ("bf16", False, "h2o_orig")])
def test_a_batch_that_accepts_different_numbers(dtype, q8, policy):
    """Draft, attend, accept, accumulate and insert, four times: an entry that accepted
    nothing is left as it was, and every entry's cache is that of its own tokens alone."""
    B, Hq, Hkv, d, M, T, A = 4, 8, 2, 64, 120, 12, 5
    x, tdt = inputs(B, Hq, Hkv, d, M, T, dtype, seed=9), U.TDT[dtype]
    cache = dev_cache(x) if q8 else [dev(x["k_cache"], tdt), None, dev(x["v_cache"], tdt), None]
    scores, tp = dev(x["scores"]), dev(x["token_pos"])
    pos = np.full(B, int(x["pos0"]), np.int32)
    new = lambda *s, dt=torch.float32: torch.empty(*s, dtype=dt, device=U.DEV)
    out, lse, wsum = new(B, Hq, T, d, dt=tdt), new(B, Hq, T), new(B, Hkv, M + A)
    ka, va, idx = new(B, Hkv, A, d, dt=tdt), new(B, Hkv, A, d, dt=tdt), new(B, Hkv, A, dt=torch.int32)
    ws = new(H.h2o_tree_workspace_bytes(B, Hq, Hkv, T, M, d, tdt), dt=torch.uint8)
    ews = new(max(16, H.h2o_evict_workspace_bytes(B, Hkv, M, A, policy)), dt=torch.uint8)
    values = lambda i: oracle.dequantize(cache[i].cpu().numpy(), cache[i + 1].cpu().numpy()) if q8 \
        else U.to_np(cache[i])
    rng = np.random.default_rng(1)
    for n in range(4):
        counts = [(n + 2 * b) % (A + 1) for b in range(B)]
        counts[n] = 0
        q, kn, vn = (dev(rng.standard_normal(s).astype(np.float32), tdt)
                     for s in ((B, Hq, T, d), (B, Hkv, T, d), (B, Hkv, T, d)))
        parents = np.stack([[int(rng.integers(-1, i)) if i else -1 for i in range(T)] for _ in range(B)])
        path = np.full((B, A), -1, np.int32)
        for b, k in enumerate(counts):
            path[b, :k] = np.sort(rng.permutation(T)[:k])
            parents[b, path[b, :k]] = np.concatenate([[-1], path[b, :k]])[:k]
        before = [t.clone() if t is not None else None for t in (*cache, scores, tp)]
        old = [values(0), values(2)]
        U.say("draft", n, counts)
        H.h2o_sdpa_tree(q, cache[0], cache[2], kn, vn, dev(parents.astype(np.int32)), out, lse, ws,
                        k_scales=cache[1], v_scales=cache[3])
        H.h2o_tree_accept(q, cache[0], kn, vn, lse, dev(path), ka, va, wsum, ws, k_scales=cache[1])
        H.h2o_accumulate_scores(scores, wsum)
        acc = scores.clone()
        H.h2o_tree_insert(cache[0], cache[2], scores, tp, ka, va, wsum, dev(path), dev(pos), idx, T,
                          policy, ews, k_scales=cache[1], v_scales=cache[3])
        torch.cuda.synchronize()
        now = [values(0), values(2)]
        want = oracle.tree_insert(old[0], old[1], acc.cpu().numpy(), before[5].cpu().numpy(),
                                  U.to_np(ka), U.to_np(va), wsum.cpu().numpy(), path, pos, T, policy)
        np.testing.assert_array_equal(idx.cpu().numpy(), want[4])
        np.testing.assert_array_equal(scores.cpu().numpy(), want[2])
        np.testing.assert_array_equal(tp.cpu().numpy(), want[3])
        for b, k in enumerate(counts):
            if k == 0:                # nothing accepted: nothing changes, the scores included
                for t, t0 in zip((*cache, scores, tp), before):
                    assert t is None or torch.equal(t[b], t0[b])
                continue
            # the entry alone: its chunk of k tokens on its cache before
            at = path[b, :k]
            one = lambda t: U.to_np(t[b:b + 1])[:, :, at]
            o, l, w = oracle.sdpa_chunk(one(q), old[0][b:b + 1], old[1][b:b + 1], one(kn), one(vn))
            got = torch.cat([wsum[b:b + 1, :, :M], wsum[b:b + 1, :, M:M + k]], -1)
            close(dtype, f"draft {n} entry {b}", out=(torch.from_numpy(one(out)), o), wsum=(got, w))
            for h in range(Hkv):
                kept = np.setdiff1d(np.arange(M), idx[b, h, :k].cpu().numpy())
                for i in range(2):
                    np.testing.assert_array_equal(now[i][b, h, kept], old[i][b, h, kept])
                    put = U.to_np((kn, vn)[i])[b, h, at]
                    if q8:
                        put = oracle.dequantize(*oracle.quantize(put.astype(np.float32)))
                    np.testing.assert_array_equal(now[i][b, h, idx[b, h, :k].cpu().numpy()], put)
        pos += np.asarray(counts, np.int32)


def test_captured_with_new_paths():
    """A graph of accept, accumulate and insert, replayed with other paths and positions
    between eager calls of the same."""
    B, Hq, Hkv, d, M, T, A = 3, 8, 2, 64, 200, 16, 4
    x, bf = inputs(B, Hq, Hkv, d, M, T, "bf16", seed=2), torch.bfloat16
    q, kn, vn = dev(x["q"], bf), dev(x["k_new"], bf), dev(x["v_new"], bf)
    lse = torch.full((B, Hq, T), 6.0, device=U.DEV)
    rng = np.random.default_rng(3)
    path, pos = dev(_paths("gaps", B, T, A, rng)), dev(np.full(B, M, np.int32))

    def state():
        new = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt, device=U.DEV)
        return dict(c=dev_cache(x), scores=dev(x["scores"]), tp=dev(x["token_pos"]),
                    ka=new(B, Hkv, A, d, dt=bf), va=new(B, Hkv, A, d, dt=bf), wsum=new(B, Hkv, M + A),
                    idx=new(B, Hkv, A, dt=torch.int32),
                    ws=new(max(16, H.h2o_tree_workspace_bytes(B, Hq, Hkv, T, M, d, bf)), dt=torch.uint8))

    def call(s):
        c = s["c"]
        H.h2o_tree_accept(q, c[0], kn, vn, lse, path, s["ka"], s["va"], s["wsum"], s["ws"], k_scales=c[1])
        H.h2o_accumulate_scores(s["scores"], s["wsum"])
        H.h2o_tree_insert(c[0], c[2], s["scores"], s["tp"], s["ka"], s["va"], s["wsum"], path, pos,
                          s["idx"], T, k_scales=c[1], v_scales=c[3])

    one, two = state(), state()
    call(state())
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        call(one)
    for n in range(4):
        path.copy_(dev(_paths("gaps", B, T, A, rng)))
        pos.add_(A)
        g.replay()
        call(two)
        torch.cuda.synchronize()
        for k in ("scores", "tp", "ka", "va", "wsum", "idx"):
            assert torch.equal(one[k], two[k]), (n, k)
        for a, b in zip(one["c"], two["c"]):
            assert torch.equal(a, b)

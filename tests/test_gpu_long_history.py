"""The long-history operators as a serving loop uses them: step after step, attention behind a shared prefix, acceptance, the keys'
weights, the history update and, when the history has outgrown its budget, eviction - every step against the oracle."""
import numpy as np
import pytest

import oracle
import paper_2412_00061_amd as pkg
from workloads.device import dev_f32, dev_i32, dev_i64, to_device
from workloads.generate import round_to_storage

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,H,Hkv,dh", [("bf16", 6, 2, 64), ("bf16", 3, 3, 128), ("f32", 4, 1, 32)])
def test_steps_of_a_batch_that_outgrows_its_budget(dtype, H, Hkv, dh):
    import torch
    rng = np.random.default_rng(H * dh)
    B, N, T, P, budget, slack, sink, recent = 3, 12, 4, 25, 48, 24, 2, 16
    cap, scale = budget + slack, dh ** -0.5
    f = lambda *s: round_to_storage(rng.standard_normal(s, dtype=np.float32), dtype)  # noqa: E731
    ctx = pkg.Context(max_batch=B, max_slots=T, max_topk=1, max_vocab_rows=16, max_nodes=N, max_heads=H, max_head_dim=dh)
    kp, vp = f(Hkv, P, dh), f(Hkv, P, dh)
    dkp, dvp, plen = to_device(kp, dtype), to_device(vp, dtype), dev_i32([P])
    zeros = np.zeros((B, Hkv, cap, dh), dtype=np.float32)
    dk, dv = to_device(zeros, dtype), to_device(zeros, dtype)
    off = dev_i64(np.arange(B) * (Hkv * cap * dh))
    length = dev_i32([0] * B)
    state = {"weight": [dev_f32(np.zeros((B, Hkv, cap))) for _ in range(2)], "pos": [dev_i32(np.zeros((B, Hkv, cap))) for _ in range(2)]}
    next_pos = np.full(B, P, dtype=np.int32)  # the sequences continue the prefix
    ws = torch.empty(pkg.prefix_verify_attn_workspace_bytes(B, H, Hkv, dh, N), dtype=torch.uint8, device="cuda")
    evictions = 0
    for step in range(60):
        q, kt, vt = f(B, H, N, dh), f(B, Hkv, N, dh), f(B, Hkv, N, dh)
        n = rng.integers(1, N + 1, B)
        parent, token, seen = np.full((B, N), -1), np.full((B, N), -1), np.zeros((B, N, N), dtype=bool)
        depth = np.full((B, N), -1)
        for b in range(B):
            depth[b, 0], token[b, 0], seen[b, 0, 0] = 0, 1, True
            for i in range(1, n[b]):
                j = int(rng.integers(max(0, i - 2), i))
                j = j if depth[b, j] < T else 0
                parent[b, i], depth[b, i], token[b, i] = j, depth[b, j] + 1, 100 + i
                seen[b, i] = seen[b, j]
                seen[b, i, i] = True
        target = np.full((B, N), 7)
        for b in range(B):  # the base model agrees with one path for a while
            node = int(n[b]) - 1 if rng.random() < 0.8 else 0
            while node > 0:
                target[b, parent[b, node]] = token[b, node]
                node = parent[b, node]
        words = np.zeros((B, N, 1), dtype=np.uint64)
        for j in range(N):
            words[:, :, 0] |= seen[:, :, j].astype(np.uint64) << np.uint64(j)
        dq, dkt, dvt, dn = to_device(q, dtype), to_device(kt, dtype), to_device(vt, dtype), dev_i32(n)
        w, pos = state["weight"][0], state["pos"][0]
        before = {"k": dk.float().cpu().numpy(), "v": dv.float().cpu().numpy(), "w": w.cpu().numpy(), "L": length.cpu().numpy()}

        att = pkg.prefix_verify_attn(ctx, dq, dkp, dvp, plen, dk, dv, off, length, cap, dkt, dvt, dn, dev_i64(words.view(np.int64)), scale,
                                     want_lse=True, workspace=ws)
        acc = pkg.accept_longest(ctx, dn, dev_i32(token), dev_i32(parent), dev_i32(depth), dev_i32(target), T)
        pkg.kv_weight_update(ctx, dq, att["lse"], dk, off, length, cap, dkt, acc["accept_len"], acc["accept_nodes"], scale, w, pos=pos,
                             next_pos=dev_i32(next_pos))
        grown = torch.empty_like(length)
        pkg.kv_commit(ctx, dkt, dvt, acc["accept_len"], acc["accept_nodes"], off, length, cap, dk, dv, ctx_len_out=grown)

        alen, path = acc["accept_len"].cpu().numpy(), acc["accept_nodes"].cpu().numpy()
        out, lse, got_w = att["out"].cpu().numpy(), att["lse"].cpu().numpy(), w.cpu().numpy()
        for b in range(B):
            L, nb = int(before["L"][b]), int(n[b])
            want, want_lse = oracle.prefix_attention(q[b, :, :nb], kp, vp, before["k"][b, :, :L], before["v"][b, :, :L], kt[b], vt[b], nb,
                                                     seen[b, :nb, :nb], scale)
            # (weights within 2^-15, values of a few units: the attention's own test has the bound row by row)
            assert np.abs(out[b, :, :nb] - want).max() <= 2.0 ** -15 * 6 and np.abs(lse[b, :, :nb] - want_lse).max() <= 2.0 ** -17
            nodes = [int(v) for v in path[b, :alen[b] + 1]]
            assert nodes[0] == 0 and all(parent[b, y] == x for x, y in zip(nodes, nodes[1:]))
            added, fresh = oracle.weight_update(q[b], lse[b].astype(np.float64), before["k"][b, :, :L], kt[b], nodes, scale)
            total = np.concatenate([before["w"][b, :, :L] + added, fresh], 1)
            assert np.allclose(got_w[b, :, :L + len(nodes)], total, rtol=2.0 ** -15, atol=1e-7)
            assert np.array_equal(pos.cpu().numpy()[b, :, L:L + len(nodes)], np.tile(next_pos[b] + np.arange(len(nodes)), (Hkv, 1)))
            assert int(grown[b]) == L + len(nodes)
        next_pos = next_pos + alen + 1
        length = grown
        if int(length.max()) + T + 1 > cap:
            evictions += 1
            full = {"k": dk.float().cpu().numpy(), "v": dv.float().cpu().numpy(), "w": w.cpu().numpy(), "pos": pos.cpu().numpy(), "L": length.cpu().numpy()}
            res = pkg.kv_evict(ctx, dk, dv, off, length, cap, dh, w, budget, pos=pos, next_pos=dev_i32(next_pos), sink=P + sink,
                               recent=recent)
            gk = dk.float().cpu().numpy()
            for b in range(B):
                L = int(full["L"][b])
                for h in range(Hkv):
                    kept = oracle.evict(full["w"][b, h, :L], full["pos"][b, h, :L], int(next_pos[b]), budget, P + sink, recent)
                    assert np.array_equal(res["kept"][b, h, :len(kept)].cpu().numpy(), kept)
                    assert np.array_equal(gk[b, h, :len(kept)], full["k"][b, h, kept])
                    newest = [p for p in full["pos"][b, h, :L] if p >= next_pos[b] - recent]
                    assert set(newest) <= set(res["pos"][b, h, :len(kept)].cpu().numpy().tolist())
                assert int(res["ctx_len"][b]) == min(L, budget)
            state["weight"][:] = [res["weight"], w]
            state["pos"][:] = [res["pos"], pos]
            length = res["ctx_len"]
    assert evictions >= 3
    ctx.close()

"""kv_weight_update against the float64 oracle, and its refusals."""
import ctypes
import math

import numpy as np
import pytest

import oracle
import paper_2412_00061_amd as pkg
from workloads.device import dev_f32, dev_i32, dev_i64, to_device
from workloads.generate import round_to_storage

pytestmark = pytest.mark.gpu


def make(seed, B, H, Hkv, N, dh, T, ctx, cap, dtype):
    rng = np.random.default_rng(seed)
    f = lambda *s: round_to_storage(rng.standard_normal(s, dtype=np.float32), dtype)  # noqa: E731
    c = dict(B=B, H=H, Hkv=Hkv, N=N, dh=dh, T=T, ctx=list(ctx), cap=cap, dtype=dtype, scale=dh ** -0.5)
    c["q"], c["kt"], c["kc"] = f(B, H, N, dh), f(B, Hkv, N, dh), f(B, Hkv, cap, dh)
    c["lse"] = (np.log(np.maximum(1, np.array(ctx)))[:, None, None] + 1 + rng.random((B, H, N))).astype(np.float32)
    c["weight"] = rng.random((B, Hkv, cap), dtype=np.float32)
    c["pos"] = rng.integers(0, 1000, (B, Hkv, cap)).astype(np.int32)
    c["next"] = rng.integers(1000, 2000, B).astype(np.int32)
    c["alen"] = np.array([rng.integers(0, min(T, N - 1) + 1) for _ in range(B)], dtype=np.int32)
    c["path"] = np.full((B, T + 1), -1, dtype=np.int32)
    for b in range(B):
        c["kc"][b, :, ctx[b]:] = np.nan
        c["path"][b, :c["alen"][b] + 1] = np.concatenate([[0], 1 + np.sort(rng.permutation(N - 1)[:c["alen"][b]])])
    return c


def run(ctx, c, with_pos=True):
    d = {n: to_device(c[n], c["dtype"]) for n in ("q", "kt", "kc")}
    weight, pos = dev_f32(c["weight"]), dev_i32(c["pos"]) if with_pos else None
    pkg.kv_weight_update(ctx, d["q"], dev_f32(c["lse"]), d["kc"], dev_i64(np.arange(c["B"]) * (c["Hkv"] * c["cap"] * c["dh"])),
                         dev_i32(c["ctx"]), c["cap"], d["kt"], dev_i32(c["alen"]), dev_i32(c["path"]), c["scale"], weight, pos=pos,
                         next_pos=dev_i32(c["next"]) if with_pos else None)
    return weight.cpu().numpy(), pos.cpu().numpy() if with_pos else None


def check(c, weight, pos):
    for b in range(c["B"]):
        L, path = c["ctx"][b], [int(v) for v in c["path"][b, :c["alen"][b] + 1]]
        added, fresh = oracle.weight_update(c["q"][b], c["lse"][b].astype(np.float64), c["kc"][b, :, :L], c["kt"][b], path, c["scale"])
        new = max(0, min(len(path), c["cap"] - L))
        want = c["weight"][b].astype(np.float64)
        want[:, :L] += added
        want[:, L:L + new] = fresh[:, :new]
        # A score: (dh + 2) 2^-24 sum |q k| scale, twice for its scaling; lse and the exponent's argument: 2^-23 of what they
        # are; the exponential 2^-23; an addition for every row, and the old weight's.
        rows = len(path) * c["H"] // c["Hkv"]
        big = max(float(np.abs(c["q"][b]).astype(np.float64).max(-1).max()) * float(np.abs(k[~np.isnan(k)]).max(initial=0)) * c["dh"]
                  for k in (c["kc"][b, :, :L], c["kt"][b])) * c["scale"]
        rel = 2 * (c["dh"] + 2) * 2.0 ** -24 * big / 4 + 2.0 ** -22 * (big / 4 + np.abs(c["lse"][b]).max() + 1) + (rows + 2) * 2.0 ** -24
        off = np.abs(weight[b].astype(np.float64) - want)
        gathered = np.zeros_like(want)
        gathered[:, :L], gathered[:, L:L + new] = added, fresh[:, :new]
        assert np.all(off <= rel * gathered + 2.0 ** -23 * np.abs(want)), (b, float((off / (rel * gathered + 1e-9)).max()))
        if pos is not None:
            want_pos = c["pos"][b].copy()
            want_pos[:, L:L + new] = c["next"][b] + np.arange(new)
            assert np.array_equal(pos[b], want_pos)


SHAPES = [
    # B, H, Hkv, N, dh, T, ctx, cap
    (1, 1, 1, 1, 8, 1, [0], 1),
    (2, 2, 2, 9, 128, 8, [0, 700], 709),
    (3, 4, 2, 17, 64, 5, [1, 31, 33], 34),                 # new rows beyond the capacity are dropped
    (2, 8, 1, 64, 128, 8, [1500, 511], 1600),              # 72 rows: three blocks of them
    (1, 12, 1, 20, 80, 3, [2049], 2060),
    (4, 3, 3, 33, 16, 8, [512, 513, 5, 64], 530),
    (1, 40, 8, 128, 96, 8, [600], 601),
    (1, 20, 1, 9, 64, 8, [300], 320),                      # 180 rows: more blocks than stay in registers
    (1, 256, 1, 9, 32, 8, [130], 140),                     # as many rows as a key head may have
    (1, 8, 8, 9, 16, 8, [40001], 40010),                   # several tiles for a wavefront
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s[:6])))
def test_against_the_oracle(shape, dtype):
    c = make(sum(shape[:6]), *shape, dtype)
    ctx = pkg.Context(max_batch=c["B"], max_slots=1, max_topk=1, max_vocab_rows=16, max_nodes=c["N"], max_heads=c["H"], max_head_dim=c["dh"])
    for with_pos in (True, False):
        check(c, *run(ctx, c, with_pos))
    w1, _ = run(ctx, c)
    w2, _ = run(ctx, c)
    assert np.array_equal(w1, w2)
    ctx.close()


def test_paths_with_entries_that_are_no_nodes():
    c = make(3, 3, 4, 2, 20, 64, 6, [40, 100, 7], 128, "bf16")
    ctx = pkg.Context(max_batch=3, max_slots=1, max_topk=1, max_vocab_rows=16, max_nodes=20, max_heads=4, max_head_dim=64)
    c["alen"][:] = [2, 6, 0]
    c["path"][:] = -1
    c["path"][0, :3], c["path"][1], c["path"][2, 0] = [0, 3, 9], [0, 1, 2, 3, 4, 5, 6], 0
    want, pos = run(ctx, c)
    # the same rows, with lengths that have to be clamped
    d = dict(c, alen=np.array([2, 99, -5], dtype=np.int32))
    got, gpos = run(ctx, d)
    assert np.array_equal(want, got) and np.array_equal(pos, gpos)
    # an entry that is no node: no row of it, no place for it
    d = dict(c, path=c["path"].copy())
    d["path"][0, 1] = 20
    d["path"][0, 2] = -1
    got, gpos = run(ctx, d)
    only = dict(c, alen=np.array([0, 6, 0], dtype=np.int32))
    want, pos = run(ctx, only)
    assert np.array_equal(want, got) and np.array_equal(pos, gpos)
    # a row that saw nothing
    d = dict(c, lse=c["lse"].copy(), alen=np.array([0, 0, 0], dtype=np.int32))
    d["lse"][:, :, 0] = -math.inf
    got, _ = run(ctx, d)
    for b in range(3):
        L = c["ctx"][b]
        assert np.array_equal(got[b, :, :L], c["weight"][b, :, :L]) and np.all(got[b, :, L] == 0)
    ctx.close()


def test_refusals():
    import torch
    c = make(1, 2, 4, 2, 5, 64, 3, [4, 4], 16, "bf16")
    ctx = pkg.Context(max_batch=2, max_slots=1, max_topk=1, max_vocab_rows=16, max_nodes=5, max_heads=4, max_head_dim=64)
    t = {n: to_device(c[n], "bf16") for n in ("q", "kt", "kc")}
    t.update(lse=dev_f32(c["lse"]), off=dev_i64([0, 2 * 16 * 64]), ctx=dev_i32(c["ctx"]), alen=dev_i32(c["alen"]), path=dev_i32(c["path"]),
             weight=dev_f32(c["weight"]), pos=dev_i32(c["pos"]), next=dev_i32(c["next"]))
    p = {n: ctypes.c_void_p(x.data_ptr()) for n, x in t.items()}

    def go(want, text, handle=ctx.handle, **k):
        a = dict(dt=1, q=p["q"], lse=p["lse"], kc=p["kc"], off=p["off"], ctx=p["ctx"], cap=16, kt=p["kt"], alen=p["alen"], path=p["path"],
                 T=3, B=2, H=4, Hkv=2, dh=64, N=5, scale=0.1, weight=p["weight"], pos=p["pos"], next=p["next"])
        a.update(k)
        assert ctx.lib.kv_weight_update(handle, *a.values()) == want, k
        if handle:
            assert text in ctx.last_error(), (k, ctx.last_error())

    go(-1, "", handle=None)
    for name in ("q", "lse", "kc", "off", "ctx", "kt", "alen", "path", "weight"):
        go(-1, "null", **{name: None})
    go(-1, "next_pos", next=None)
    for name in ("T", "B", "H", "Hkv", "dh", "N", "cap"):
        go(-1, "positive", **{name: 0})
    go(-1, "multiple of H_kv", Hkv=3)
    go(-1, "element type", dt=2)
    for s in (0.0, -2.0, math.inf, math.nan):
        go(-1, "scale", scale=s)
    go(-2, "multiple of 8", dh=12)
    go(-2, "2^30", cap=(1 << 30) + 1)
    go(-2, "T <=", T=9)
    go(-2, "limits", B=3)
    go(-2, "limits", H=6)
    go(-2, "limits", N=6)
    for name in ("q", "kc", "kt"):
        go(-1, "aligned", **{name: ctypes.c_void_p(t[name].data_ptr() + 4)})
    torch.cuda.synchronize()
    assert np.array_equal(t["weight"].cpu().numpy(), c["weight"])
    with pytest.raises(pkg.CtcspecError, match="weight"):
        pkg.kv_weight_update(ctx, t["q"], t["lse"], t["kc"], t["off"], t["ctx"], 15, t["kt"], t["alen"], t["path"], 0.1, t["weight"])
    ctx.close()

"""kv_evict against the oracle - every output is exact -, and its refusals."""
import ctypes
import math

import numpy as np
import pytest

import oracle
import paper_2412_00061_amd as pkg
from workloads.device import dev_f32, dev_i32, dev_i64, to_device
from workloads.generate import round_to_storage

pytestmark = pytest.mark.gpu


def make(seed, B, Hkv, dh, cap, ctx, budget, sink, recent, dtype, weights="decades"):
    rng = np.random.default_rng(seed)
    c = dict(B=B, Hkv=Hkv, dh=dh, cap=cap, ctx=list(ctx), budget=budget, sink=sink, recent=recent, dtype=dtype)
    w = {"decades": lambda s: rng.random(s) ** -1.5 * 1e-3 * (rng.random(s) > 0.1), "equal": lambda s: np.full(s, 0.25),
         "few": lambda s: rng.integers(0, 3, s) * 1.0, "signed": lambda s: rng.standard_normal(s),
         "odd": lambda s: rng.choice([np.nan, np.inf, -np.inf, 0.0, -0.0, 1.0, 1e-42, -3.0], s)}[weights]
    c["weight"] = w((B, Hkv, cap)).astype(np.float32)
    c["pos"] = np.stack([[rng.permutation(cap) for _ in range(Hkv)] for _ in range(B)]).astype(np.int32)
    c["next"] = np.array([L + int(rng.integers(0, cap - L + 1)) for L in (min(max(x, 1), cap) for x in ctx)], dtype=np.int32)
    c["k"] = round_to_storage(rng.standard_normal((B, Hkv, cap, dh), dtype=np.float32), dtype)
    c["v"] = round_to_storage(rng.standard_normal((B, Hkv, cap, dh), dtype=np.float32), dtype)
    return c


def check(c, with_pos=True):
    import torch
    ctx = pkg.Context(max_batch=c["B"], max_slots=1, max_topk=1, max_vocab_rows=16, max_nodes=1, max_heads=c["Hkv"], max_head_dim=c["dh"])
    place = np.random.default_rng(1).permutation(c["B"])
    k, v = np.empty_like(c["k"]), np.empty_like(c["v"])
    k[place], v[place] = c["k"], c["v"]
    k, v = to_device(k, c["dtype"]), to_device(v, c["dtype"])
    B, Hkv, cap, budget = c["B"], c["Hkv"], c["cap"], c["budget"]
    out = {"kept": torch.full((B, Hkv, budget), -9, dtype=torch.int32, device="cuda"), "weight": torch.full((B, Hkv, cap), -9.0, device="cuda"),
           "ctx_len": torch.full((B,), -9, dtype=torch.int32, device="cuda"), "pos": torch.full((B, Hkv, cap), -9, dtype=torch.int32, device="cuda")}
    more = dict(pos=dev_i32(c["pos"]), next_pos=dev_i32(c["next"]), sink=c["sink"], recent=c["recent"]) if with_pos else {}
    args = (ctx, k, v, dev_i64(place * (Hkv * cap * c["dh"])), dev_i32(c["ctx"]), cap, c["dh"], dev_f32(c["weight"]), budget)
    for again in range(2):  # the inputs stay, so the second call finds and leaves the same
        pkg.kv_evict(*args, out=out, **more)
        got = {n: t.cpu().numpy() for n, t in out.items()}
        gk, gv = k.float().cpu().numpy()[place], v.float().cpu().numpy()[place]
        for b in range(B):
            L = min(max(c["ctx"][b], 0), cap)
            n = min(L, budget)
            assert got["ctx_len"][b] == n
            for h in range(Hkv):
                kept = oracle.evict(c["weight"][b, h, :L], c["pos"][b, h, :L] if with_pos else None, int(c["next"][b]), budget,
                                    c["sink"] if with_pos else 0, c["recent"] if with_pos else 0)
                assert np.array_equal(got["kept"][b, h, :n], kept) and np.all(got["kept"][b, h, n:] == -1), (b, h)
                assert np.array_equal(got["weight"][b, h, :n], c["weight"][b, h, kept], equal_nan=True)
                assert np.all(got["weight"][b, h, n:] == -9)
                if with_pos:
                    assert np.array_equal(got["pos"][b, h, :n], c["pos"][b, h, kept]) and np.all(got["pos"][b, h, n:] == -9)
                rows = np.concatenate([kept, np.arange(n, cap)])  # rows behind the new length stay as they were
                assert np.array_equal(gk[b, h], c["k"][b, h, rows]) and np.array_equal(gv[b, h], c["v"][b, h, rows])
    ctx.close()


SHAPES = [
    # B, Hkv, dh, cap, ctx, budget, sink, recent
    (1, 1, 8, 1, [1], 1, 0, 0),
    (1, 1, 8, 2, [2], 1, 0, 1),
    (2, 3, 64, 70, [64, 70], 5, 1, 2),
    (3, 2, 128, 1100, [1100, 1024, 1025], 1024, 4, 100),
    (4, 2, 80, 700, [0, 333, 334, 700], 333, 2, 50),
    (1, 2, 128, 5000, [5000], 129, 16, 64),
    (2, 1, 16, 40000, [40000, 33000], 20000, 4, 1000),       # 20000 rows may move: more than a round of them
    (1, 1, 8, 70000, [70000], 69000, 0, 0),
    (2, 2, 64, 300, [300, 1000000], 500, 3, 10),             # a budget beyond the capacity
    (1, 4, 64, 2320, [2304], 2048, 4, 256),
    (3, 1, 8, 40000, [3000, 17000, 200], 129, 4, 64),        # short histories in a long cache
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s[:4])) + f"-{s[5]}")
def test_against_the_oracle(shape, dtype):
    c = make(sum(shape[:4]), *shape, dtype)
    check(c)
    check(c, with_pos=False)


@pytest.mark.parametrize("weights", ["equal", "few", "signed", "odd"])
@pytest.mark.parametrize("L,budget", [(100, 37), (3000, 1500), (1025, 1024), (2048, 1)])
def test_ties_and_weights_of_every_kind(weights, L, budget):
    c = make(L, 2, 2, 32, L, [L, L - 7], budget, 0, 0, "bf16", weights)
    check(c)
    c.update(sink=min(3, budget // 2), recent=budget // 3)
    check(c)


@pytest.mark.parametrize("weights", ["equal", "few", "signed", "odd", "decades"])
@pytest.mark.parametrize("L,budget", [(9000, 5000), (16384, 300), (17000, 9000), (70001, 1001)])
def test_ties_in_long_histories(weights, L, budget):
    """Thousands of rows with one weight: the search goes on in their indexes."""
    c = make(L, 1, 2, 8, L, [L], budget, 0, 0, "bf16", weights)
    check(c)
    c.update(sink=min(30, budget // 2), recent=budget // 3)
    check(c)


@pytest.mark.parametrize("spread", [1e-7, 1e-4, 1e-2])
def test_weights_that_share_their_leading_digits(spread):
    """Thousands of different weights next to each other."""
    c = make(7, 1, 2, 8, 30000, [30000], 12345, 0, 0, "bf16")
    c["weight"] = (1.5 + spread * np.random.default_rng(3).random(c["weight"].shape)).astype(np.float32)
    check(c)


def test_positions_at_the_ends_of_their_range():
    """Without recent rows no position is too high, and a sequence shorter than `recent` keeps what it holds."""
    top = 2 ** 31 - 1
    c = make(6, 1, 1, 8, 200, [200], 20, 3, 0, "f32")
    c["pos"][0, 0, 100:] = top
    check(c)
    c.update(sink=0, recent=20, next=np.array([top], dtype=np.int32))
    check(c)
    c["next"] = np.array([-(2 ** 31) + 4], dtype=np.int32)
    c["pos"][0, 0, ::3] = -(2 ** 31) + 1
    check(c)


def test_positions_that_occur_more_than_once():
    """More rows are to stay than the budget holds: those of smallest index."""
    c = make(4, 1, 2, 16, 400, [400], 50, 5, 5, "f32")
    c["pos"][:] = 1
    check(c)


def test_refusals():
    import torch
    c = make(1, 2, 2, 64, 32, [32, 20], 8, 1, 2, "bf16")
    ctx = pkg.Context(max_batch=2, max_slots=1, max_topk=1, max_vocab_rows=16, max_nodes=1, max_heads=2, max_head_dim=64)
    i32 = dict(dtype=torch.int32, device="cuda")
    t = dict(k=to_device(c["k"], "bf16"), v=to_device(c["v"], "bf16"), off=dev_i64([0, 2 * 32 * 64]), ctx=dev_i32(c["ctx"]),
             weight=dev_f32(c["weight"]), pos=dev_i32(c["pos"]), next=dev_i32(c["next"]), kept=torch.zeros((2, 2, 8), **i32),
             weight_out=torch.zeros((2, 2, 32), device="cuda"), pos_out=torch.zeros((2, 2, 32), **i32), ctx_out=torch.zeros(2, **i32))
    p = {n: ctypes.c_void_p(x.data_ptr()) for n, x in t.items()}

    def go(want, text, handle=ctx.handle, **k):
        a = dict(dt=1, k=p["k"], v=p["v"], off=p["off"], ctx=p["ctx"], cap=32, weight=p["weight"], pos=p["pos"], next=p["next"], B=2, Hkv=2,
                 dh=64, budget=8, sink=1, recent=2, kept=p["kept"], weight_out=p["weight_out"], pos_out=p["pos_out"], ctx_out=p["ctx_out"])
        a.update(k)
        assert ctx.lib.kv_evict(handle, *a.values()) == want, k
        if handle:
            assert text in ctx.last_error(), (k, ctx.last_error())

    go(-1, "", handle=None)
    for name in ("k", "v", "off", "ctx", "weight", "kept", "weight_out", "ctx_out"):
        go(-1, "null", **{name: None})
    for name in ("B", "Hkv", "dh", "cap", "budget"):
        go(-1, "positive", **{name: 0})
    go(-1, "element type", dt=3)
    go(-1, "sink", sink=-1)
    go(-1, "sink", recent=-1)
    go(-1, "sink", sink=5, recent=4)
    go(-1, "pos", pos=None)
    go(-1, "pos", pos_out=None)
    go(-1, "pos", pos=None, pos_out=None)
    go(-1, "next_pos", next=None)
    go(-1, "inputs", weight_out=p["weight"])
    go(-1, "inputs", pos_out=p["pos"])
    go(-1, "inputs", ctx_out=p["ctx"])
    go(-2, "multiple of 8", dh=60)
    go(-2, "limits", B=3)
    go(-2, "limits", Hkv=3)
    go(-2, "limits", dh=72)
    go(-2, "limits", cap=524289)
    go(-2, "limits", budget=(1 << 30) + 1)
    go(-1, "aligned", k=ctypes.c_void_p(t["k"].data_ptr() + 8))
    torch.cuda.synchronize()
    assert not any(t[n].any() for n in ("kept", "weight_out", "pos_out", "ctx_out"))
    with pytest.raises(pkg.CtcspecError, match="weight"):
        pkg.kv_evict(ctx, t["k"], t["v"], t["off"], t["ctx"], 31, 64, t["weight"], 8)
    with pytest.raises(pkg.CtcspecError, match="one dtype"):
        pkg.kv_evict(ctx, t["k"], t["v"].float(), t["off"], t["ctx"], 32, 64, t["weight"], 8)
    ctx.close()


def test_nan_is_never_kept_before_a_number():
    c = make(2, 1, 1, 8, 64, [64], 3, 0, 0, "f32")
    c["weight"][:] = math.nan
    c["weight"][0, 0, [60, 5]] = [-math.inf, -1.0]
    check(c)

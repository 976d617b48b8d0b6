"""q4_verify_attn against the float64 oracle over what the codes stand for: head layouts, lengths from nothing to many iterations, windows
and sinks, empty rows, values that are no numbers in hidden places, calls as the documentation allows them."""
import numpy as np
import pytest

import oracle
import paper_2412_00061_amd as pkg
from test_gpu_prefix_attn import mask_words
from workloads.device import dev_i32, dev_i64, to_device
from workloads.generate import round_to_storage

pytestmark = pytest.mark.gpu


def make(seed, B, H, Hkv, N, dh, ctx, n_nodes, *, window=0, sink=0, spread=1.0, spikes=0, room=0):
    """Operands with room behind every length; the sequences' blocks lie in another order than they count, and what lies behind a
    sequence's length stands for NaN."""
    rng = np.random.default_rng(seed)
    f = lambda *s: round_to_storage(rng.standard_normal(s, dtype=np.float32), "bf16")  # noqa: E731
    cap = max(ctx) + int(rng.integers(0, 5)) + room  # (more room: the work is dealt, where it would not be otherwise)
    c = dict(B=B, H=H, Hkv=Hkv, N=N, dh=dh, cap=cap, ctx=list(ctx), n=list(n_nodes), scale=dh ** -0.5, window=window, sink=sink)
    c["q"] = round_to_storage(f(B, H, N, dh) * np.float32(spread), "bf16")
    c["kt"], c["vt"] = f(B, Hkv, N, dh), f(B, Hkv, N, dh)
    kc, vc = f(B, Hkv, cap, dh), f(B, Hkv, cap, dh)
    for _ in range(spikes):  # keys that rows cannot overlook, anywhere
        b = rng.integers(B)
        if ctx[b]:
            kc[b, rng.integers(Hkv), rng.integers(ctx[b])] *= 8
    c["parts"] = [*oracle.q4_encode(kc), *oracle.q4_encode(vc)]  # [B, Hkv, cap, ..]
    seen, depth = np.zeros((B, N, N), dtype=bool), np.full((B, N), -1)
    for b in range(B):
        for i in (1, 3):
            c["parts"][i][b, :, ctx[b]:] = 255
        c["kt"][b, :, n_nodes[b]:] = c["vt"][b, :, n_nodes[b]:] = c["q"][b, :, n_nodes[b]:] = np.nan
        for i in range(n_nodes[b]):
            if i:
                parent = rng.integers(i)
                seen[b, i], depth[b, i] = seen[b, parent], depth[b, parent] + 1
            else:
                depth[b, i] = 0
            seen[b, i, i] = True
    c["seen"], c["depth"], c["place"] = seen, depth, rng.permutation(B)
    return c


def upload(c):
    import torch
    flat = []
    for part in c["parts"]:
        x = np.empty_like(part)
        x[c["place"]] = part
        flat.append(torch.from_numpy(x if x.size else np.zeros(16, dtype=np.uint8)).cuda())
    d = {n: to_device(c[n], "bf16") for n in ("q", "kt", "vt")}
    d.update(parts=flat, off=dev_i64(c["place"].astype(np.int64) * (c["Hkv"] * c["cap"])), ctx=dev_i32(c["ctx"]), n=dev_i32(c["n"]),
             mask=dev_i64(mask_words(c["seen"], c["N"]).view(np.int64)), depth=dev_i32(c["depth"]))
    return d


def context(c, **more):
    lim = dict(max_batch=c["B"], max_slots=1, max_topk=1, max_vocab_rows=16, max_nodes=c["N"], max_heads=c["H"], max_head_dim=c["dh"])
    lim.update(more)
    return pkg.Context(**lim)


def call(ctx, c, d, out_dtype, **more):
    cache = pkg.binding._Q4Cache() if c["cap"] == 0 else pkg.q4_cache(*d["parts"])
    return pkg.q4_verify_attn(ctx, d["q"], cache, d["off"], d["ctx"], c["cap"], d["kt"], d["vt"], d["n"], d["mask"], c["scale"],
                              node_depth=d["depth"] if c["window"] else None, window=c["window"], sink=c["sink"], out_dtype=out_dtype, want_lse=True,
                              **more)


def cached(c, b):
    L = c["ctx"][b]
    k, ks, v, vs = (p[b, :, :L] for p in c["parts"])
    return oracle.q4_decode(k, ks, c["dh"]), oracle.q4_decode(v, vs, c["dh"])


def reference(c, b, magnitudes=False):
    n = c["n"][b]
    k, v = cached(c, b)
    vt = c["vt"][b].astype(np.float64)
    return oracle.window_attention(c["q"][b, :, :n], k, np.abs(v) if magnitudes else v, c["kt"][b], np.abs(vt) if magnitudes else vt, n,
                                   c["seen"][b, :n, :n], c["depth"][b, :n], c["scale"], c["window"], c["sink"])


def allowed(c, b):
    """Relative error of a row's weights and of their sum, in float32 arithmetic.  A score is a sum of dh exact products: off by at most
    (dh + 2) 2^-24 sum |q k| scale, and half as much again where it is scaled; a weight by that, and the sum it is divided by, too; 2^-22 for
    the exponential and its argument's rounding, twice; an addition of 2^-24 for each of the 16 keys of a step of a product, for each
    tile's sum and its 16 weights, and for the joins of up to 64 parts, in numerator and sum; weights in three bf16 parts are within 2^-24."""
    n = c["n"][b]
    k, _ = cached(c, b)
    score = np.zeros((c["H"], n))
    for h in range(c["H"]):
        g = h // (c["H"] // c["Hkv"])
        keys = np.abs(np.concatenate([k[g], c["kt"][b, g, :n].astype(np.float64)]))
        score[h] = (np.nan_to_num(keys) @ np.abs(c["q"][b, h, :n].astype(np.float64)).T).max(0) * c["scale"]
    return 3 * (c["dh"] + 2) * 2.0 ** -24 * score + 2.0 ** -20 + ((c["ctx"][b] + n) / 8 + 160) * 2.0 ** -24


def check(c, res, sentinel=None):
    import torch
    out, lse = res["out"].float().cpu().numpy().astype(np.float64), res["lse"].cpu().numpy().astype(np.float64)
    bf16 = res["out"].dtype == torch.bfloat16
    for b in range(c["B"]):
        n = c["n"][b]
        if sentinel is not None:
            assert np.all(out[b, :, n:] == sentinel) and np.all(lse[b, :, n:] == sentinel)
        if not n:
            continue
        want, want_lse = reference(c, b)
        absolute, _ = reference(c, b, True)
        rel = allowed(c, b)
        off = np.abs(out[b, :, :n] - want)
        limit = (rel + (2.0 ** -8 if bf16 else 0))[..., None] * absolute + (2.0 ** -8 if bf16 else 2.0 ** -23) * np.abs(want) + 1e-30
        assert np.array_equal(np.isnan(out[b, :, :n]), np.isnan(want)), b
        real = ~np.isnan(want) & ~np.isinf(want)
        assert np.array_equal(out[b, :, :n][np.isinf(want)], want[np.isinf(want)])
        assert np.all((off <= limit)[real]), (b, float((off / limit)[real].max()))
        none = np.isneginf(want_lse)
        assert np.array_equal(np.isneginf(lse[b, :, :n]), none) and np.all(out[b, :, :n][none] == 0)
        assert np.array_equal(np.isnan(lse[b, :, :n]), np.isnan(want_lse))
        fine = np.isfinite(want_lse)
        assert np.all(np.abs(lse[b, :, :n] - want_lse)[fine] <= (rel + 2.0 ** -22 * np.abs(want_lse))[fine]), b


SHAPES = [
    # B, H, Hkv, N, dh, ctx, n_nodes
    (1, 1, 1, 1, 8, [0], [1]),                                       # one key: the row's own
    (1, 2, 2, 1, 128, [1], [1]),
    (2, 4, 4, 1, 128, [33, 0], [1, 1]),                              # single tokens
    (3, 4, 1, 1, 64, [700, 1, 129], [1, 0, 1]),                      # four heads on one key head
    (3, 4, 2, 7, 64, [1, 64, 30], [7, 1, 5]),
    (2, 2, 2, 33, 128, [31, 200], [33, 20]),                         # two blocks of 32 rows
    (8, 2, 2, 64, 128, [0, 5, 32, 33, 63, 64, 65, 500], [64, 1, 63, 33, 32, 31, 64, 2]),
    (5, 6, 1, 25, 96, [100, 1, 0, 7, 300], [25, 0, 13, 25, 1]),      # six heads on one key head, a place not in use
    (2, 3, 3, 128, 80, [1500, 3], [128, 97]),
    (3, 8, 2, 31, 40, [255, 256, 257], [31, 30, 8]),
    (2, 2, 1, 16, 32, [127, 129], [16, 16]),                         # 32 rows: a single block
    (1, 2, 2, 5, 112, [5000], [5]),                                  # many iterations
]


@pytest.mark.parametrize("room", [0, 1100])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_against_the_oracle(shape, bf16, room):
    import torch
    c = make(len(str(shape)), *shape, spikes=3, room=room)
    d, ctx = upload(c), context(c)
    dtype = torch.bfloat16 if bf16 else torch.float32
    out = {"out": torch.full((c["B"], c["H"], c["N"], c["dh"]), 55.0, dtype=dtype, device="cuda"),
           "lse": torch.full((c["B"], c["H"], c["N"]), 55.0, device="cuda")}
    check(c, call(ctx, c, d, dtype, out=out), sentinel=55.0)
    ctx.close()


WINDOWS = [(1, 0), (2, 1), (3, 40), (31, 0), (32, 32), (33, 5), (64, 31), (200, 100), (450, 4), (100000, 7), ((1 << 31) - 1, (1 << 31) - 1)]


@pytest.mark.parametrize("window,sink", WINDOWS)
@pytest.mark.parametrize("shape", [SHAPES[6], SHAPES[7], (2, 4, 2, 1, 128, [513, 77], [1, 1])])
def test_windows(shape, window, sink):
    import torch
    c = make(window % 1000 + sink % 1000, *shape, window=window, sink=sink, spikes=2)
    d, ctx = upload(c), context(c)
    for dtype in (torch.float32, torch.bfloat16):
        check(c, call(ctx, c, d, dtype))
    ctx.close()


@pytest.mark.parametrize("window,sink", [(1, 0), (7, 40), (33, 5), (150, 64)])
def test_windows_of_many_blocks(window, sink):
    """More blocks of rows than workgroups: shares with parts of several."""
    import torch
    rng = np.random.default_rng(window)
    c = make(window, 64, 13, 13, 2, 16, [int(x) for x in rng.integers(0, 300, 64)], [int(x) for x in rng.integers(0, 3, 64)], window=window, sink=sink)
    ctx = context(c)
    for dtype in (torch.float32, torch.bfloat16):
        check(c, call(ctx, c, upload(c), dtype))
    ctx.close()


@pytest.mark.parametrize("window,sink", [(1, 0), (2, 0), (3, 66), (5, 70), (9, 0)])
def test_windows_shorter_than_a_path(window, sink):
    """Trees of 128 nodes, paths up to dozens deep: nodes outside the window in every tile of the tree, sinks that end among them."""
    import torch
    c = make(window + sink, 3, 4, 2, 128, 64, [0, 65, 61], [128, 97, 66], window=window, sink=sink)
    for b in range(3):  # one long path, and what hangs on it
        for i in range(1, c["n"][b]):
            parent = i - 1 if i % 3 else max(0, i - 4)
            c["seen"][b, i], c["depth"][b, i] = c["seen"][b, parent], c["depth"][b, parent] + 1
            c["seen"][b, i, i] = True
    assert c["depth"].max() > 40
    ctx = context(c)
    for dtype in (torch.float32, torch.bfloat16):
        check(c, call(ctx, c, upload(c), dtype))
    c["vt"][0, 0, 3, 7], c["vt"][1, 1, 60, 9], c["vt"][2, 0, 65, 40] = np.inf, np.nan, -np.inf
    check(c, call(ctx, c, upload(c), torch.float32))
    ctx.close()


def test_a_window_that_holds_everything_is_none():
    import torch
    c = make(3, *SHAPES[8])
    d, ctx = upload(c), context(c)
    want = call(ctx, c, d, torch.float32)
    c.update(window=1500 + 128, sink=0)
    got = call(ctx, c, d, torch.float32)
    assert all(torch.equal(a[:, :, :97], b[:, :, :97]) for a, b in zip(want.values(), got.values()))
    ctx.close()


def test_peaked_and_far_scores():
    """Scores up to some hundreds, in either order along the keys: the reference moves, weights underflow."""
    import torch
    for order in (1, -1):
        c = make(11, 2, 2, 1, 20, 128, [900, 300], [20, 11], spread=4.0)
        grow = (2.0 ** np.linspace(-6, 3, c["cap"])[::order]).astype(np.float32)
        k = oracle.q4_decode(c["parts"][0], np.where(c["parts"][1] == 255, 127, c["parts"][1]), 128) * grow[None, None, :, None]
        codes, scales = oracle.q4_encode(k)
        for b, L in enumerate(c["ctx"]):
            c["parts"][0][b, :, :L], c["parts"][1][b, :, :L] = codes[b, :, :L], scales[b, :, :L]
        ctx = context(c)
        for dtype in (torch.float32, torch.bfloat16):
            check(c, call(ctx, c, upload(c), dtype))
        ctx.close()


@pytest.mark.parametrize("room", [0, 1100])
def test_rows_without_keys(room):
    import torch
    c = make(7, 3, 4, 2, 9, 64, [0, 0, 40], [9, 4, 9], room=room)
    c["seen"][0, 2] = c["seen"][0, 8] = c["seen"][1] = c["seen"][2, 5] = False
    ctx = context(c)
    for cap_zero in (False, True):
        if cap_zero:  # no cache at all
            c.update(ctx=[0, 0, 0], cap=0, parts=[p[:, :, :0] for p in c["parts"]])
        res = call(ctx, c, upload(c), torch.float32)
        check(c, res)
        assert torch.isneginf(res["lse"][0, :, 2]).all() and not res["out"][0, :, 8].any()
    ctx.close()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("N,n", [(20, 13), (70, 66)])
def test_no_numbers_in_hidden_and_seen_places(N, n, bf16):
    """Infinities and NaN in tree rows and blocks of cached rows that stand for NaN: they reach the rows that see them, and only these."""
    import torch
    c = make(N, 2, 2, 1, N, 96, [500, 61], [n, 5], window=60, sink=3)
    c["vt"][0, 0, 3, 7], c["vt"][0, 0, 4, 8], c["vt"][0, 0, 5, 40] = np.inf, -np.inf, np.nan
    c["vt"][0, 0, n - 1, 90], c["vt"][1, 0, 2, 95] = np.inf, np.nan
    c["kt"][0, 0, 6, 3] = np.nan
    L = 500
    c["parts"][3][0, 0, 1, 2] = c["parts"][3][0, 0, 100, 0] = c["parts"][3][0, 0, L - 59, 1] = 255  # seen by all; by none; by the root's row alone
    c["parts"][1][0, 0, 440:442] = 255  # keys before the window
    c["parts"][3][1, 0, 2, 0] = c["parts"][3][1, 0, 60, 2] = 255
    ctx = context(c)
    dtype = torch.bfloat16 if bf16 else torch.float32
    res = call(ctx, c, upload(c), dtype)
    check(c, res)
    assert torch.isnan(res["out"]).any() and torch.isinf(res["out"]).any() and torch.isfinite(res["out"][0, :, :2]).any()
    ctx.close()


@pytest.mark.parametrize("bf16", [False, True])
def test_no_numbers_in_dealt_shares(bf16):
    """The same where blocks are cut to pieces, and where a workgroup has one whole beside them."""
    import torch
    c = make(71, 3, 4, 2, 70, 80, [1500, 61, 1100], [66, 70, 5])
    c["vt"][0, 0, 3, 7], c["vt"][0, 1, 4, 8], c["vt"][0, 0, 65, 79] = np.inf, -np.inf, np.nan
    c["vt"][1, 1, 40, 0], c["vt"][2, 0, 1, 33] = np.nan, np.inf
    c["parts"][3][0, 0, 1499, 2] = c["parts"][3][1, 1, 60, 0] = 255  # blocks in the last, partial tile
    c["seen"][0, 10:20, 3] = False
    ctx = context(c)
    res = call(ctx, c, upload(c), torch.bfloat16 if bf16 else torch.float32)
    check(c, res)
    assert torch.isinf(res["out"]).any() and torch.isnan(res["out"]).any()
    ctx.close()


def test_scores_that_are_no_numbers():
    import torch
    c = make(5, 2, 2, 2, 6, 64, [40, 40], [6, 6])
    c["q"][0, 0, 1, 5], c["q"][0, 1, 2, 0] = np.nan, np.inf
    c["kt"][1, 0, 3, 2] = np.inf
    c["q"][1, 0, :, 2] = -np.abs(c["q"][1, 0, :, 2]) - 1  # a score of -infinity: no weight
    ctx = context(c)
    check(c, call(ctx, c, upload(c), torch.float32))
    ctx.close()


def test_lengths_outside_their_range_count_as_its_ends():
    import torch
    c = make(9, 3, 2, 2, 10, 64, [50, 50, 0], [10, 10, 10])
    c["parts"] = [p[:, :, :50] for p in c["parts"]]
    c["cap"] = 50
    d, ctx = upload(c), context(c)
    d["ctx"], d["n"] = dev_i32([50, 99999, -5]), dev_i32([99, 10, 10])
    check(c, call(ctx, c, d, torch.float32))
    d["n"] = dev_i32([10, -3, 10])
    c["n"] = [10, 0, 10]
    check(c, call(ctx, c, d, torch.float32))
    c.update(window=4, sink=0)  # depths beyond the nodes count as the last, negative ones as 0
    c["depth"][0, 9] = 9
    d["depth"] = dev_i32(np.where(np.arange(10) == 9, 12345, c["depth"]))
    c["depth"][:, 9] = 9
    d["depth"][:, 0] = -7
    check(c, call(ctx, c, d, torch.float32))
    ctx.close()


# ---- the calls ---------------------------------------------------------------------------------------------------
def big(seed=1, **more):
    return make(seed, 3, 8, 2, 40, 128, [700, 64, 350], [40, 17, 1], **{"room": 1100 * (seed % 2), **more})


def test_codes_beyond_32_bits():
    """A cache whose rows begin past 2^32 bytes of codes: the same bits as at its beginning."""
    import torch
    c = big()
    d, ctx = upload(c), context(c)
    want = call(ctx, c, d, torch.float32)
    far = (1 << 32) // 64 + 777
    for i, part in enumerate(d["parts"]):
        wide = torch.empty((far * part.shape[-1] + part.numel(),), dtype=torch.uint8, device="cuda")
        wide[far * part.shape[-1]:] = part.reshape(-1)
        d["parts"][i] = wide
    d["off"] = d["off"] + far
    got = call(ctx, c, d, torch.float32)
    for b, n in enumerate(c["n"]):
        assert all(torch.equal(want[x][b, :, :n], got[x][b, :, :n]) for x in want)
    ctx.close()


def outputs(c):
    import torch
    return {"out": torch.zeros((c["B"], c["H"], c["N"], c["dh"]), device="cuda"), "lse": torch.zeros((c["B"], c["H"], c["N"]), device="cuda")}


def test_two_streams_at_once_without_a_workspace():
    import torch
    cases = [big(1), big(2, window=90, sink=6)]
    alone, want = context(cases[0]), []
    data = [upload(c) for c in cases]
    for c, d in zip(cases, data):
        want.append(call(alone, c, d, torch.float32, out=outputs(c)))
    torch.cuda.synchronize()
    ctxs = [context(c, **{}) for c in cases]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = [[outputs(c) for c in cases] for _ in range(10)]
    torch.cuda.synchronize()
    for ctx, s in zip(ctxs, streams):
        ctx.set_stream(s)
    for o in outs:
        for i in range(2):
            call(ctxs[i], cases[i], data[i], torch.float32, out=o[i])
    torch.cuda.synchronize()
    for o in outs:
        assert all(torch.equal(o[i][x], want[i][x]) for i in range(2) for x in want[i])
    for ctx in (alone, *ctxs):
        ctx.close()


@pytest.mark.parametrize("more", [dict(window=90, sink=6, room=0), dict(room=1100)])
def test_captured_and_replayed(more):
    """Two calls that share a workspace in one graph; other lengths and inputs between the replays."""
    import torch
    stream = torch.cuda.Stream()
    cases = [big(s, **more) for s in (3, 4, 5)]
    for c in cases[1:]:  # (one shape of the buffers)
        assert c["B"] == cases[0]["B"]
        pad = cases[0]["cap"]
        c["parts"] = [np.concatenate([p, np.full((3, 2, 16, p.shape[-1]), 255, np.uint8)], 2)[:, :, :pad] if p.shape[2] < pad else p[:, :, :pad] for p in c["parts"]]
        c["cap"], c["ctx"] = pad, [min(x, pad) for x in c["ctx"]]
    cases[1]["n"], cases[2]["ctx"] = [3, 17, 0], [0, 64, 33]
    data = [upload(c) for c in cases]
    alone, want = context(cases[0]), []
    for c, d in zip(cases, data):
        want.append([{n: t.clone() for n, t in call(alone, c, d, dt, out=None if dt == torch.bfloat16 else outputs(c)).items()}
                     for dt in (torch.float32, torch.bfloat16)])
    live = {n: ([p.clone() for p in t] if n == "parts" else t.clone()) for n, t in data[0].items()}
    outs = [outputs(cases[0]), {**outputs(cases[0]), "out": torch.zeros((3, 8, 40, 128), dtype=torch.bfloat16, device="cuda")}]
    ws = torch.empty(pkg.q4_verify_attn_workspace_bytes(3, 8, 2, 128, 40), dtype=torch.uint8, device="cuda")
    ctx = context(cases[0], **{})
    torch.cuda.synchronize()
    ctx.set_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        for dt, o in zip((torch.float32, torch.bfloat16), outs):
            call(ctx, cases[0], live, dt, workspace=ws, out=o)
    for rep in range(6):
        i = rep % 3
        for n, t in live.items():
            for to, frm in zip(t, data[i][n]) if n == "parts" else ((t, data[i][n]),):
                to.copy_(frm)
        ws.fill_(0xff)
        for o in outs:
            for t in o.values():
                t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want[i]):
            for b, n in enumerate(cases[i]["n"]):
                assert all(torch.equal(o[x][b, :, :n], w[x][b, :, :n]) for x in w), (rep, b)
                assert all(not o[x][b, :, n:].any() for x in w)
    ctx.close()
    alone.close()


def test_bytes_for_a_large_call_serve_a_smaller_one():
    import torch
    c = make(2, 2, 8, 2, 3, 64, [70, 20], [3, 2])
    d, ctx = upload(c), context(c)
    ws = torch.full((pkg.q4_verify_attn_workspace_bytes(4, 8, 2, 64, 128),), 255, dtype=torch.uint8, device="cuda")
    for B in (1, 2, 3, 4):
        for N in (1, 3, 4, 8, 9, 64, 128):
            assert pkg.q4_verify_attn_workspace_bytes(B, 8, 2, 64, N) <= ws.numel()
    check(c, call(ctx, c, d, torch.float32, workspace=ws))
    ctx.close()

"""prefix_verify_attn's weights one by one: queries and keys are small whole numbers and the scale is a power of two, so every score is
exact, and key j's value is 1 in component j and 0 elsewhere, so component j of a result IS key j's weight.  What rounding does to a
weight then stands alone, and a float result has to carry it to the last bits."""
import numpy as np
import pytest

import oracle

U = 2.0 ** -24  # half a step of float
SCALE = 2.0 ** -6


def exact_case(seed, B, H, Hkv, N, dh, P, ctx, n_nodes, dtype):
    """As test_gpu_prefix_attn.make, with the keys numbered: the prefix's, then the cached ones, then the nodes."""
    rng = np.random.default_rng(seed)
    grid = lambda *s: rng.integers(-2, 3, s).astype(np.float32)  # noqa: E731
    c = dict(B=B, H=H, Hkv=Hkv, N=N, dh=dh, P=P, cap=max(ctx), pcap=P, ctx=list(ctx), n=list(n_nodes), dtype=dtype, scale=SCALE,
             place=rng.permutation(B))
    c["q"], c["kp"], c["kc"], c["kt"] = grid(B, H, N, dh), grid(Hkv, P, dh), grid(B, Hkv, max(ctx), dh), grid(B, Hkv, N, dh)
    for name, k in (("vp", c["kp"]), ("vc", c["kc"]), ("vt", c["kt"])):
        c[name] = np.zeros_like(k)
    c["vp"][:, range(P), range(P)] = 1
    seen = np.zeros((B, N, N), dtype=bool)
    for b in range(B):
        assert P + ctx[b] + n_nodes[b] <= dh
        c["vc"][b, :, range(ctx[b]), range(P, P + ctx[b])] = 1
        c["vt"][b, :, range(n_nodes[b]), range(P + ctx[b], P + ctx[b] + n_nodes[b])] = 1
        for i in range(n_nodes[b]):
            if i:
                seen[b, i] = seen[b, rng.integers(i)]
            seen[b, i, i] = True
    c["seen"] = seen
    return c


def tiles(c, b):
    """The components of keys that a kernel takes together: 32 of one kind."""
    start = 0
    for length in (c["P"], c["ctx"][b], c["n"][b]):
        for at in range(0, length, 32):
            yield slice(start + at, start + min(at + 32, length))
        start += length


def limits(spread, parts, bf16_out):
    """(how far a weight may be off, relative to it; how far its share of its tile's weights may be off).
    With A the width of a row's scores in the log2 domain: a weight's exponent is one rounding of a number up to A (half a step of A) of
    a product with a rounded log2(e) (A U), and an exponential costs a step (2 U); the reference is one number for all weights of
    a tile.  `parts`: what a weight's rounding to bf16 leaves of it.  Its parts are added one by one (3 U), and the result is scaled and
    added to in up to three joins (2 U each) and divided by the sum (2 U).  A join's factors (an exponential, 2 U, and their
    argument's rounding, A U) and the sum are common to a tile; the sum has 16 additions in a lane for a tile, of at most
    4 tiles, and one with the neighbour."""
    exponent = np.log2(spread) if spread > 0 else 0.0
    half = 2.0 ** np.floor(exponent) * U
    weight = np.log(2) * (half + spread * U) + 2 * U + parts
    alone = weight + 3 * U + 3 * 2 * U + 2 * U
    common = 3 * (2 * U + np.log(2) * spread * U) * 2 + weight + 24 * U + 3 * 2 * U
    out = 2.0 ** -8 if bf16_out else 0.0
    return alone + common + out, 2 * (alone + out)


def check_weights(c, b, out, parts, bf16_out):
    """out [H, n, dh] float64."""
    L, n, P = c["ctx"][b], c["n"][b], c["P"]
    want, _ = oracle.prefix_attention(c["q"][b, :, :n], c["kp"], c["vp"], c["kc"][b, :, :L], c["vc"][b, :, :L], c["kt"][b], c["vt"][b], n,
                                      c["seen"][b, :n, :n], SCALE)
    assert np.all(out[want == 0] == 0)
    low = np.where(want > 0, want, np.inf).min(-1)
    spread = float(np.log2(want.max(-1) / low).max())
    assert 0 <= spread < 8
    whole, share = limits(spread, parts, bf16_out)
    off = np.abs(out - want) / np.where(want > 0, want, 1)
    assert off.max() <= whole, (b, off.max() / whole)
    worst = 0.0
    for t in tiles(c, b):
        a, e = out[..., t], want[..., t]
        sa, se = a.sum(-1, keepdims=True), e.sum(-1, keepdims=True)
        some = se[..., 0] > 0
        off = np.abs(a / np.where(se > 0, sa, 1) - e / np.where(se > 0, se, 1))[some] / np.where(e > 0, e / np.where(se > 0, se, 1), 1)[some]
        worst = max(worst, float(off.max(initial=0.0)))
    assert worst <= share, (b, worst / share)


SHAPES = [
    # B, H, Hkv, N, dh, P, ctx, n_nodes
    (1, 2, 2, 1, 128, 60, [67], [1]),                    # 32 rows of a workgroup
    (2, 2, 2, 1, 64, 9, [40, 0], [1, 1]),
    (2, 4, 2, 16, 64, 30, [17, 3], [16, 15]),            # 64
    (2, 2, 1, 32, 128, 40, [56, 1], [32, 20]),           # 128
    (4, 4, 2, 64, 128, 8, [50, 0, 56, 1], [64, 64, 50, 7]),  # 256, behind a short prefix
    (3, 2, 2, 50, 128, 64, [14, 0, 3], [50, 1, 50]),     # 256: not all rows of a sequence in one block
    (1, 8, 2, 64, 128, 0, [64], [64]),                   # 256 rows of one sequence, no prefix
    (8, 5, 1, 20, 64, 33, [0, 1, 9, 11, 0, 4, 2, 3], [20, 20, 20, 20, 3, 20, 20, 0]),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", [("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s[:6])))
def test_weights(shape, dtype, out):
    import torch
    from test_gpu_prefix_attn import call, context, upload
    c = exact_case(3, *shape, dtype)
    ctx = context(c)
    res = call(ctx, c, upload(c), torch.bfloat16 if out == "bf16" else torch.float32)["out"].double().cpu().numpy()
    for b in range(c["B"]):
        if c["n"][b]:
            check_weights(c, b, res[b, :, :c["n"][b]], 2.0 ** -8 if out == "bf16" else U, out == "bf16")
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", [("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s[:6])))
def test_sums(shape, dtype, out):
    """lse: the sum takes the weights before they are rounded to bf16, so it has a float's bits whatever the result's type.  Off by the sum's
    relative error (what `limits` allows a weight without its parts), the reference's two roundings (a score in the log2 domain: of log2(e)
    and of the product), two steps of the logarithm, which is below 8 (half a step of that: 4 U), and the roundings of the sum of
    both, of ln 2 and of the last product."""
    import torch
    from test_gpu_prefix_attn import call, context, upload
    c = exact_case(7, *shape, dtype)
    ctx = context(c)
    res = call(ctx, c, upload(c), torch.bfloat16 if out == "bf16" else torch.float32)["lse"].double().cpu().numpy()
    for b in range(c["B"]):
        n = c["n"][b]
        if not n:
            continue
        L, P = c["ctx"][b], c["P"]
        weights, lse = oracle.prefix_attention(c["q"][b, :, :n], c["kp"], c["vp"], c["kc"][b, :, :L], c["vc"][b, :, :L], c["kt"][b], c["vt"][b], n,
                                               c["seen"][b, :n, :n], SCALE)
        low = np.where(weights > 0, weights, np.inf).min(-1)
        spread = float(np.log2(weights.max(-1) / low).max())
        top = np.abs(lse + np.log(weights.max(-1))) + spread  # the reference is a score within that
        lim = limits(spread, 0.0, False)[0] + 2 * top * U + 4 * 4 * U + 3 * (np.abs(lse) + top + 8) * U
        off = np.abs(res[b, :, :n] - lse)
        assert np.all(off <= lim), (b, float((off / lim).max()))
    ctx.close()


def bf16(x):
    import torch
    return torch.from_numpy(x).bfloat16().float().numpy()


@pytest.mark.parametrize("parts", [1, 2, 3])
def test_the_limits_tell_how_many_parts_a_weight_has(parts):
    """(On the CPU, in float: weights in three bf16 parts pass, in two or one they do not.)"""
    c = exact_case(3, *SHAPES[4], "bf16")
    L, n, P = c["ctx"][0], c["n"][0], c["P"]
    out = np.zeros((c["H"], n, c["dh"]))
    for h in range(c["H"]):
        g = h // 2
        keys = np.concatenate([c["kp"][g], c["kc"][0, g, :L], c["kt"][0, g, :n]])
        s = (c["q"][0, h, :n] @ keys.T) * np.float32(SCALE * np.log2(np.e))
        there = np.concatenate([np.ones((n, P + L), bool), c["seen"][0, :n, :n]], 1)
        p = np.exp2(s - np.where(there, s, -np.inf).max(1, keepdims=True)).astype(np.float32) * there
        whole, left = np.zeros_like(p), p
        for _ in range(parts):
            part = bf16(left)
            whole, left = whole + part, left - part
        out[h, :, :P + L + n] = whole / p.sum(1, keepdims=True, dtype=np.float32)
    if parts == 3:
        check_weights(c, 0, out, U, False)
    else:
        with pytest.raises(AssertionError):
            check_weights(c, 0, out, U, False)

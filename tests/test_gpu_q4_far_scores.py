"""q4_verify_attn where scores are far from 0: up to the ends of float's range, rows of all magnitudes side by side.  Queries and keys are
chosen so that every score is one product, exact in float."""
import numpy as np
import pytest

import oracle
from test_gpu_q4_attn import call, context, make, upload

pytestmark = pytest.mark.gpu


def far(seed, ctx_len, n, exponents, **more):
    """Queries with one component that is not 0, +-2^e, e from row to row another one; keys whose first components are multiples of 2^-6 below 8."""
    c = make(seed, len(ctx_len), 4, 2, max(n), 64, ctx_len, n, **more)
    rng = np.random.default_rng(seed)
    rows = np.arange(c["N"])
    c["kt"][..., 0] = np.round(c["kt"][..., 0] * 4) / 4
    for b in range(c["B"]):
        for h in range(4):
            e = np.asarray(exponents)[(rows + 3 * h + 5 * b) % len(exponents)]
            c["q"][b, h, :n[b]] = 0
            c["q"][b, h, rows[:n[b]], 0] = ((-1.0) ** rng.integers(0, 2, c["N"]) * 2.0 ** e)[:n[b]]
    return c


def check(c, res):
    """A score is exact, its scaling one rounding - its place in the softmax a difference of two of them, off by 2^-22 of itself (the factor,
    log2(e) times the scale, by 2^-23), where it counts: below 2^5, 2^-17, and a weight with it -; or, where the reference has no room for a fraction, a rounding of
    the score, which moves it by less than 2^-14 of what it is from the next one: weights there are 1 or 0.  2^-22 for the exponential, 2^-24 for each
    addition; twice, in numerator and sum.  A bf16 result has 2^-8 of the weights and 2^-8 of the result on top."""
    import torch
    bf16 = res["out"].dtype == torch.bfloat16
    out, lse = res["out"].double().cpu().numpy(), res["lse"].double().cpu().numpy()
    for b in range(c["B"]):
        n, L = c["n"][b], c["ctx"][b]
        k, ks, v, vs = (p[b, :, :L] for p in c["parts"])
        k, v = oracle.q4_decode(k, ks, 64), oracle.q4_decode(v, vs, 64)
        args = (n, c["seen"][b, :n, :n], c["depth"][b, :n], c["scale"], c["window"], c["sink"])
        want, want_lse = oracle.window_attention(c["q"][b, :, :n], k, v, c["kt"][b], c["vt"][b].astype(np.float64), *args)
        size, _ = oracle.window_attention(c["q"][b, :, :n], k, np.abs(v), c["kt"][b], np.abs(c["vt"][b]).astype(np.float64), *args)
        limit = (2.0 ** -15 + (2.0 ** -8 if bf16 else 0)) * size + (2.0 ** -8 if bf16 else 2.0 ** -23) * np.abs(want) + 1e-30
        assert np.all(np.isfinite(out[b, :, :n])), (b, np.argwhere(~np.isfinite(out[b, :, :n]))[:4])
        assert np.all(np.abs(out[b, :, :n] - want) <= limit), (b, float((np.abs(out[b, :, :n] - want) / limit).max()))
        assert np.all(np.abs(lse[b, :, :n] - want_lse) <= 2.0 ** -16 + 2.0 ** -21 * np.abs(want_lse)), b


# (with a scale of 2^-3 two scores differ by 2^(e - 9) at the least: from e = 18 on the largest one has all the weight)
EXPONENTS = [-2, 0, 2, 30, 12, 31, 33, 13, 36, 40, 18, 60, 90, 24, 120, 27, 28, 29]


@pytest.mark.parametrize("more", [dict(), dict(room=1100), dict(window=100, sink=5)])
@pytest.mark.parametrize("bf16", [False, True])
def test_all_magnitudes(more, bf16):
    import torch
    c = far(3, [300, 33, 0], [40, 17, 25], EXPONENTS, **more)
    ctx = context(c)
    check(c, call(ctx, c, upload(c), torch.bfloat16 if bf16 else torch.float32))
    ctx.close()


@pytest.mark.parametrize("bf16", [False, True])
def test_histories_of_many_pieces(bf16):
    import torch
    c = far(4, [5000, 1300], [9, 2], EXPONENTS)
    ctx = context(c)
    check(c, call(ctx, c, upload(c), torch.bfloat16 if bf16 else torch.float32))
    ctx.close()


@pytest.mark.parametrize("scale", [2e38, 1e-30])
def test_ends_of_the_scale(scale):
    """The largest scale, with queries so small that scores are as above; the smallest ones, with queries that are large."""
    import torch
    shift = -121 if scale > 1 else 95
    c = far(5, [200, 70], [20, 20], [e + shift for e in (0, 3, 10, 20, 26)])
    c["scale"] = float(np.float32(scale))
    ctx = context(c)
    for dtype in (torch.float32, torch.bfloat16):
        check(c, call(ctx, c, upload(c), dtype))
    ctx.close()


@pytest.mark.parametrize("room", [0, 1100])
def test_scores_below_the_range(room):
    """Scores that float cannot hold are infinite: rows that have only such, below the range, are rows without a key; their neighbours are as ever."""
    import torch
    c = make(6, 2, 2, 2, 12, 64, [100, 40], [12, 7], room=room)
    for i in (0, 2):  # every key has 1 to 7 in its first component
        c["parts"][i][..., 0] = (c["parts"][i][..., 0] & 0xf0) | 2 if i == 0 else c["parts"][i][..., 0]
    c["parts"][1][...] = np.where(c["parts"][1] == 255, 255, 127)
    c["kt"][..., 0] = np.where(np.isnan(c["kt"][..., 0]), np.nan, 1.0)
    c["q"][:, :, ::2] = np.where(np.isnan(c["q"][:, :, ::2]), np.nan, 0.0)
    c["q"][:, :, ::2, 0] = np.where(np.isnan(c["q"][:, :, ::2, 0]), np.nan, -2.0 ** 10)
    c["q"][:, :, 1::2] *= np.float32(2.0 ** -115)
    c["scale"] = 2e38
    ctx = context(c)
    d = upload(c)
    res = call(ctx, c, d, torch.float32)
    for b in range(2):
        n = c["n"][b]
        assert not res["out"][b, :, 0:n:2].any() and torch.isneginf(res["lse"][b, :, 0:n:2]).all()
        assert torch.isfinite(res["out"][b, :, 1:n:2]).all() and res["out"][b, :, 1:n:2].any()
    ctx.close()


@pytest.mark.parametrize("bf16", [False, True])
def test_no_numbers_beside_far_scores(bf16):
    """Keys that are no numbers or infinite reach the rows that see them, of whatever magnitude, and no others."""
    import torch
    c = far(7, [90, 40], [30, 30], EXPONENTS)
    c["kt"][0, :, 4, 0], c["kt"][0, :, 9, 0], c["kt"][1, :, 2, 0] = np.nan, np.inf, -np.inf
    ctx = context(c)
    out = call(ctx, c, upload(c), torch.bfloat16 if bf16 else torch.float32)["out"].float().cpu().numpy()
    for b, strange in ((0, (4, 9)), (1, (2,))):
        for h in range(4):
            for i in range(30):
                scores = [c["kt"][b, h // 2, j, 0] * c["q"][b, h, i, 0] for j in strange if c["seen"][b, i, j]]
                none = any(np.isnan(s) or s == np.inf for s in scores)
                assert np.all(np.isnan(out[b, h, i])) if none else np.all(np.isfinite(out[b, h, i])), (b, h, i)
    ctx.close()


@pytest.mark.parametrize("ctx_len,room", [([900, 70], 0), ([900, 70], 1100), ([6000, 3000], 0)])
@pytest.mark.parametrize("bf16", [False, True])
def test_references_that_move_between_large_scores(ctx_len, room, bf16):
    """Scores near 2^20, those of the last four tiles' last keys higher by 64 (8 when scaled): what the keys before them have gathered is scaled down
    by exactly what their weights would have been, whatever the references' roundings - half a unit of 2^-6 here."""
    import torch
    c = make(8, 2, 4, 2, 20, 64, ctx_len, [20, 20], room=room)
    codes, scales = c["parts"][0], c["parts"][1]
    codes[..., 0] = 0x02  # a first component of 1, a second one of 0
    scales[scales != 255] = 127
    for b, L in enumerate(ctx_len):
        codes[b, :, [L - 1, L - 33, L - 65], 0] = 0x22  # a second one of 1
        if L > 97:
            codes[b, :, L - 97, 0] = 0x22
    c["kt"][..., 0], c["kt"][..., 1] = 1.0, 0.0
    rows = np.arange(20)
    for b in range(2):
        for h in range(4):
            c["q"][b, h] = 0
            c["q"][b, h, :, 0] = 2.0 ** 20 * (1 + (7 * rows + 29 * h + 3 * b) % 128 / 128)
            c["q"][b, h, :, 1] = 64
    ctx = context(c)
    check(c, call(ctx, c, upload(c), torch.bfloat16 if bf16 else torch.float32))
    ctx.close()

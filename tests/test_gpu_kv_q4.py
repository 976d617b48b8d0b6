"""kv_append_q4, kv_commit_q4 and kv_read_q4 against the float64 oracle: codes, scales and what they stand for have to be equal."""
import numpy as np
import pytest

import oracle
import paper_2412_00061_amd as pkg
from workloads.device import dev_i32, dev_i64, to_device
from workloads.generate import round_to_storage

pytestmark = pytest.mark.gpu


def values(rng, shape, dtype):
    """Numbers of many magnitudes, blocks that are all zero, ties of the grid, the ends of the type's range."""
    x = (rng.standard_normal(shape) * 2.0 ** rng.integers(-12, 12, shape[:-1] + (1,))).astype(np.float32)
    flat = x.reshape(-1, shape[-1])
    for r in range(0, len(flat), 5):
        flat[r] = rng.choice(np.array([0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6, 7, 0.5], dtype=np.float32), shape[-1]) * rng.choice([-1, 1], shape[-1])
    flat[0] = 0
    if len(flat) > 6:
        flat[1, :3], flat[2, :3] = [3.3e38, -3.0e38, 1e-3], [1e-45, -2e-38, 1.2e-38]
        flat[3] = 7 * 2.0 ** 125
        flat[4, -1], flat[6, 0] = np.nan, -np.inf
    return round_to_storage(x, dtype)


def empty(rng, rows, dh):
    blocks = -(-dh // 32)
    return [rng.integers(0, 256, (rows, n), dtype=np.uint8) for n in (16 * blocks, blocks, 16 * blocks, blocks)]


def inside(parts, off, rows):
    """The sequences' blocks lie within the buffers: asked before anything is launched."""
    assert off.min() >= 0 and off.max() + rows <= min(len(p) for p in parts)


def upload(parts):
    import torch
    return [torch.from_numpy(p).cuda() for p in parts]


def context(B, H, dh, N=128):
    return pkg.Context(max_batch=B, max_slots=8, max_topk=1, max_vocab_rows=16, max_nodes=N, max_heads=H, max_head_dim=dh)


def expect(parts, k, v, at):
    """parts with row at[r] holding k[r], v[r]."""
    for i, x in ((0, k), (2, v)):
        codes, scales = oracle.q4_encode(x)
        parts[i][at], parts[i + 1][at] = codes, scales


CASES = [
    # B, Hkv, dh, max_rows, ctx, rows, kv_cap
    (1, 1, 8, 1, [0], [1], 1),
    (1, 2, 32, 3, [5], [0], 9),
    (2, 3, 128, 40, [0, 17], [40, 33], 60),
    (3, 2, 80, 50, [1, 60, 7], [50, 50, -2], 70),   # the second has room for ten
    (2, 1, 96, 7, [70, -1], [7, 999], 70),          # no room; more rows than there are
    (4, 5, 64, 9, [3, 0, 9, 2], [1, 2, 3, 9], 33),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,dh,rows,ctx,count,cap", CASES)
def test_append_and_read(B, H, dh, rows, ctx, count, cap, dtype):
    import torch
    rng = np.random.default_rng(dh + rows)
    k, v = values(rng, (B, H, rows, dh), dtype), values(rng, (B, H, rows, dh), dtype)
    parts = empty(rng, (B + 1) * H * cap, dh)
    off = rng.permutation(B).astype(np.int64) * (H * cap) + H * cap // 2
    inside(parts, off, H * cap)
    dev = upload(parts)
    cache, c = pkg.q4_cache(*dev), context(B, H, dh)
    out = torch.full((B,), -5, dtype=torch.int32, device="cuda")
    pkg.kv_append_q4(c, to_device(k, dtype), to_device(v, dtype), dev_i32(count), cache, dev_i64(off), dev_i32(ctx), cap, ctx_len_out=out)
    want_len = []
    for b in range(B):
        L, n = min(max(ctx[b], 0), cap), min(max(count[b], 0), rows)
        n = min(n, cap - L)
        want_len.append(L + n)
        for h in range(H):
            expect(parts, k[b, h, :n], v[b, h, :n], off[b] + h * cap + L + np.arange(n))
    assert out.tolist() == want_len
    for got, want in zip(dev, parts):
        assert np.array_equal(got.cpu().numpy(), want)
    # read back from two rows before, in either type; the rows behind the count keep what they held
    first = np.array(ctx) - 2
    for out_dtype in (torch.float32, torch.bfloat16):
        back = {n: torch.full((B, H, rows + 3, dh), 77.0, dtype=out_dtype, device="cuda") for n in ("k", "v")}
        pkg.kv_read_q4(c, cache, dev_i64(off), dev_i32(first), dev_i32(np.array(count) + 2), rows + 3, cap, H, dh, out_dtype=out_dtype, out=back)
        for name, i in (("k", 0), ("v", 2)):
            got = back[name].float().cpu().numpy()
            want = np.full_like(got, 77.0)
            for b in range(B):
                j = np.arange(max(0, min(count[b] + 2, rows + 3)))
                j = j[(first[b] + j >= 0) & (first[b] + j < cap)]
                for h in range(H):
                    at = off[b] + h * cap + first[b] + j
                    sane = parts[i + 1][at]
                    want[b, h, j] = oracle.q4_decode(parts[i][at], np.where((sane < 2) | ((sane > 252) & (sane < 255)), 255, sane), dh)
                    # (bytes that no call writes stand for nothing)
                    odd = np.repeat((sane < 2) | ((sane > 252) & (sane < 255)), 32, -1)[:, :dh]
                    row = got[b, h, j]
                    row[odd] = np.nan
                    got[b, h, j] = row
            assert np.array_equal(got, want, equal_nan=True)
    c.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,dh,N,T,ctx,cap", [(1, 1, 16, 1, 1, [0], 2), (3, 2, 128, 64, 8, [0, 31, 95], 100), (2, 4, 80, 128, 5, [7, 20], 22),
                                                (4, 1, 64, 9, 3, [5, 5, 5, 5], 5)])
def test_commit(B, H, dh, N, T, ctx, cap, dtype):
    import torch
    rng = np.random.default_rng(N + T)
    k, v = values(rng, (B, H, N, dh), dtype), values(rng, (B, H, N, dh), dtype)
    parts = empty(rng, B * H * cap, dh)
    off = rng.permutation(B).astype(np.int64) * (H * cap)
    inside(parts, off, H * cap)
    alen = rng.integers(0, min(T, N - 1) + 1, B)
    path = np.full((B, T + 1), -1)
    for b in range(B):
        path[b, :alen[b] + 1] = np.concatenate([[0], 1 + np.sort(rng.permutation(N - 1)[:alen[b]])]) if N > 1 else 0
    if N == 64:
        alen[0], path[0, :4] = 99, [3, -1, 64, 5]  # a path longer than T, entries that are no node, the same node twice
        path[0, 4:] = 5
    dev = upload(parts)
    c = context(B, H, dh, N)
    out = torch.zeros((B,), dtype=torch.int32, device="cuda")
    pkg.kv_commit_q4(c, to_device(k, dtype), to_device(v, dtype), dev_i32(alen), dev_i32(path), pkg.q4_cache(*dev), dev_i64(off), dev_i32(ctx), cap,
                     ctx_len_out=out)
    for b in range(B):
        n = min(max(alen[b], 0), T) + 1
        assert out[b].item() == min(ctx[b] + n, cap)
        for j in range(min(n, cap - ctx[b])):
            if 0 <= path[b, j] < N:
                for h in range(H):
                    expect(parts, k[b, h, path[b, j]], v[b, h, path[b, j]], off[b] + h * cap + ctx[b] + j)
    for got, want in zip(dev, parts):
        assert np.array_equal(got.cpu().numpy(), want)
    c.close()


def test_rows_beyond_32_bits():
    """A cache whose codes lie past 2^32 bytes and whose rows past 2^26: the same bytes as at its beginning."""
    import torch
    H, dh, cap, far = 2, 128, 50, (1 << 32) // 64 + 12345
    rng = np.random.default_rng(5)
    k, v = values(rng, (1, H, 20, dh), "bf16"), values(rng, (1, H, 20, dh), "bf16")
    dev = [torch.zeros((far + H * cap, n), dtype=torch.uint8, device="cuda") for n in (64, 4, 64, 4)]
    c, cache = context(1, H, dh), pkg.q4_cache(*dev)
    for off in (0, far):
        pkg.kv_append_q4(c, to_device(k, "bf16"), to_device(v, "bf16"), dev_i32([20]), cache, dev_i64([off]), dev_i32([3]), cap)
    back = [pkg.kv_read_q4(c, cache, dev_i64([off]), dev_i32([3]), dev_i32([20]), 20, cap, H, dh) for off in (0, far)]
    for d in dev:
        assert torch.equal(d[:H * cap], d[far:]) and not d[H * cap:far].any()
    for n in ("k", "v"):
        assert torch.equal(back[0][n].view(torch.int16), back[1][n].view(torch.int16)) and back[0][n].any()
    c.close()

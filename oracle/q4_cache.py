"""Oracle: a cache held in 4 bits and the attention over it, with and without a sliding window.

Test infrastructure only (see the package docstring).  float64 throughout, written from the definitions: the number format is the
microscaling one with 4-bit elements (sign, two bits of exponent, one of fraction) and a power of two for every 32 of them; the
attention is the verification attention of Sec. 2.1 over what the codes stand for."""
import numpy as np

BLOCK = 32
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def q4_encode(x):
    """x [.., dh] -> codes [.., 16 * blocks] uint8, scales [.., blocks] uint8."""
    x = np.asarray(x, dtype=np.float64)
    dh = x.shape[-1]
    blocks = -(-dh // BLOCK)
    padded = np.zeros(x.shape[:-1] + (blocks * BLOCK,))
    padded[..., :dh] = x
    padded = padded.reshape(x.shape[:-1] + (blocks, BLOCK))
    amax = np.abs(padded).max(-1)
    real = np.isfinite(amax)
    e = np.full(amax.shape, -125)
    for step in range(-125, 125):  # the smallest exponent whose 7-fold power holds the block
        e = np.where(real & (amax > 7 * 2.0 ** step), step + 1, e)
    y = np.where(real[..., None], padded, 0.0) / 2.0 ** e[..., None]
    off = np.abs(np.abs(y)[..., None] - GRID)
    near = off == off.min(-1, keepdims=True)
    code = np.where(near[..., 0::2].any(-1), near[..., 0::2].argmax(-1) * 2, near[..., 1::2].argmax(-1) * 2 + 1)  # of two the even one
    code = code + np.where((y < 0) & (code > 0), 8, 0)
    code = code.reshape(x.shape[:-1] + (blocks * BLOCK,)).astype(np.uint8)
    return code[..., 0::2] | code[..., 1::2] << 4, np.where(real, e + 127, 255).astype(np.uint8)


def q4_decode(codes, scales, dh):
    """What the codes stand for, [.., dh] float64."""
    codes, scales = np.asarray(codes), np.asarray(scales)
    c = np.stack([codes & 15, codes >> 4], -1).reshape(scales.shape + (BLOCK,))
    scale = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return (GRID[c & 7] * np.where(c & 8, -1.0, 1.0) * scale[..., None]).reshape(codes.shape[:-1] + (BLOCK * scales.shape[-1],))[..., :dh]


def window_attention(q, k_cache, v_cache, k_tree, v_tree, n_nodes, seen, depth, scale, window=0, sink=0):
    """One sequence.  q [H, >=n, dh]; k_cache [Hkv, L, dh]: exactly the cached rows, row j at position j; k_tree [Hkv, >=n, dh], node i
    at position L + depth[i]; seen bool [n, n]: which tree nodes a row sees.  With a window a row at position p sees of all these the keys
    at positions above p - window and below sink.  Head h reads key head h // (H // Hkv).  Returns (out [H, n, dh], lse [H, n]); a row
    without any key, or with no score above -infinity, has out 0 and lse -inf."""
    H, n, dh = q.shape[0], int(n_nodes), q.shape[-1]
    group, L = H // k_cache.shape[0], k_cache.shape[1]
    out, lse = np.zeros((H, n, dh)), np.full((H, n), -np.inf)
    for h in range(H):
        g = h // group
        keys = np.concatenate([k_cache[g], k_tree[g, :n]]).astype(np.float64)
        values = np.concatenate([v_cache[g], v_tree[g, :n]]).astype(np.float64)
        for i in range(n):
            sees = np.concatenate([np.ones(L, dtype=bool), np.asarray(seen[i, :n], dtype=bool)])
            if window:
                place = np.concatenate([np.arange(L), L + np.asarray(depth[:n])])
                sees &= (place > L + depth[i] - window) | (place < sink)
            if not sees.any():
                continue
            with np.errstate(invalid="ignore", over="ignore"):
                s = scale * (keys[sees] @ q[h, i].astype(np.float64))
                m = s.max()
                if m == -np.inf:
                    continue
                p = np.exp(s - m)
                lse[h, i] = m + np.log(p.sum())
                out[h, i] = (p / p.sum()) @ values[sees]
    return out, lse

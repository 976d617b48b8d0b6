"""Oracle: attention behind a prefix that a batch shares, the weight that cached keys gather, and eviction by it.

Test infrastructure only (see the package docstring).  float64 throughout, written from the definitions; the paper has no
formula for any of the three: the attention is the verification attention of Sec. 2.1 over one more block of keys, the weight
is the sum of the softmax weights that the accepted rows gave a key, and eviction keeps the rows with the largest sums."""
import numpy as np


def prefix_attention(q, k_prefix, v_prefix, k_cache, v_cache, k_tree, v_tree, n_nodes, seen, scale):
    """One sequence.  q [H, >=n, dh]; k_prefix [Hkv, P, dh], k_cache [Hkv, L, dh]: exactly the visible rows; k_tree
    [Hkv, >=n, dh]; seen bool [n, n]: which tree nodes a row sees.  Head h reads key head h // (H // Hkv).  Returns
    (out [H, n, dh], lse [H, n]); a row without any key has out 0 and lse -inf."""
    H, n, dh = q.shape[0], int(n_nodes), q.shape[-1]
    group = H // k_prefix.shape[0]
    out, lse = np.zeros((H, n, dh)), np.full((H, n), -np.inf)
    for h in range(H):
        g = h // group
        common = np.concatenate([k_prefix[g], k_cache[g]]).astype(np.float64)
        values = np.concatenate([v_prefix[g], v_cache[g]]).astype(np.float64)
        for i in range(n):
            own = np.nonzero(seen[i])[0]
            keys = np.concatenate([common, k_tree[g, own].astype(np.float64)])
            if not len(keys):
                continue
            s = scale * (keys @ q[h, i].astype(np.float64))
            m = s.max()
            p = np.exp(s - m)
            lse[h, i] = m + np.log(p.sum())
            out[h, i] = (p / p.sum()) @ np.concatenate([values, v_tree[g, own].astype(np.float64)])
    return out, lse


def weight_update(q, lse, k_cache, k_tree, path, scale):
    """One sequence.  q [H, N, dh], lse [H, N], k_cache [Hkv, L, dh] (the cached rows), k_tree [Hkv, N, dh], path: the
    accepted nodes from the root on.  Returns (added [Hkv, L]: what the cached keys gather, fresh [Hkv, len(path)]: what the
    path's own keys start with - a path node is seen by itself and by those after it)."""
    H, Hkv = q.shape[0], k_cache.shape[0]
    added, fresh = np.zeros((Hkv, k_cache.shape[1])), np.zeros((Hkv, len(path)))
    for h in range(H):
        g = h // (H // Hkv)
        for r, node in enumerate(path):
            if np.isneginf(lse[h, node]):
                continue
            row = q[h, node].astype(np.float64)
            added[g] += np.exp(scale * (k_cache[g].astype(np.float64) @ row) - lse[h, node])
            for m in range(r + 1):
                fresh[g, m] += np.exp(scale * (k_tree[g, path[m]].astype(np.float64) @ row) - lse[h, node])
    return added, fresh


def evict(weight, pos, next_pos, budget, sink, recent):
    """One sequence and key head.  weight [L], pos [L] or None.  Returns the old index of every row of the new cache."""
    L = len(weight)
    n = min(L, budget)

    def rank(j):
        guarded = pos is not None and (pos[j] < sink or (recent > 0 and pos[j] >= next_pos - recent))
        w = float(weight[j])
        return (0, 0.0, j) if guarded else ((2, 0.0, j) if np.isnan(w) else (1, -w, j))

    stays = sorted(sorted(range(L), key=rank)[:n])
    kept = list(range(n))
    arriving = iter([j for j in stays if j >= n])
    inside = set(stays)
    for j in range(n):
        if j not in inside:
            kept[j] = next(arriving)
    return np.array(kept, dtype=np.int64)

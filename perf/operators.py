"""The long-history operators' workloads: verification attention over a prefix that a batch shares, the attention weight
that cached keys gather, and eviction of the cache by it.

  attention   one layer of the tree-masked verification attention of a batch whose sequences continue one common prefix
              (prefix_verify_attn)
  weights     one layer's update of the weight that every cached key has gathered, after a step was accepted
              (kv_weight_update)
  evict       one layer's cache brought down to a number of rows per sequence and head (kv_evict)

`run` computes them in elementary float32 operations, or through the package's calls where `own` is set.  Sizes are those
of the workloads in `workloads/configs.py` (7B shapes, the ragged batch of eight, its float32 shapes), generic grouped
heads, and prefixes and histories up to the lengths for which such operators exist.
"""
import functools
import math

import torch

own = False

LLAMA_7B = dict(H=32, Hkv=32, dh=128, dtype="bf16")


def listed():
    return [
        # plain decoding, one token per sequence, of eight chats behind one system prompt: latency and one read of the prefix
        dict(name="attn_token_b8", kind="attention", B=8, nodes=1, prefix=2048, ctx_lo=16, ctx_hi=256, out="f32", **LLAMA_7B),
        # the ragged batch of eight with 64-node trees, behind a prompt of 2048
        dict(name="attn_tree_b8", kind="attention", B=8, nodes=64, prefix=2048, ctx_lo=256, ctx_hi=2048, out="f32", **LLAMA_7B),
        # the same batch over a document of 32768 tokens that all eight ask about, rows handed on in bf16: bound by the products
        dict(name="attn_document_b8", kind="attention", B=8, nodes=64, prefix=32768, ctx_lo=256, ctx_hi=2048, out="bf16",
             **LLAMA_7B),
        # grouped heads, odd sizes, sequences that have hardly begun
        dict(name="attn_grouped_odd", kind="attention", B=13, nodes=25, prefix=5003, ctx_lo=0, ctx_hi=777, H=40, Hkv=8,
             dh=128, dtype="bf16", out="bf16"),
        # a small float32 model
        dict(name="attn_f32_dh64", kind="attention", B=4, nodes=100, prefix=1500, ctx_lo=300, ctx_hi=900, H=12, Hkv=12,
             dh=64, dtype="f32", out="f32"),
        # the ragged batch of eight: up to nine accepted rows against 256 to 2048 cached keys
        dict(name="weights_b8", kind="weights", B=8, nodes=64, T=8, ctx_lo=256, ctx_hi=2048, **LLAMA_7B),
        # long histories with grouped heads
        dict(name="weights_long_grouped", kind="weights", B=4, nodes=64, T=8, ctx_lo=16384, ctx_hi=65536, H=32, Hkv=8,
             dh=128, dtype="bf16"),
        # a small float32 model, a head dimension that fills no power of two
        dict(name="weights_f32_dh80", kind="weights", B=3, nodes=17, T=5, ctx_lo=1, ctx_hi=777, H=6, Hkv=3, dh=80,
             dtype="f32"),
        # serving in equilibrium: every 256 tokens the cache of eight sequences goes back to 2048 rows
        dict(name="evict_step_b8", kind="evict", B=8, ctx_lo=2304, ctx_hi=2304, budget=2048, sink=4, recent=256, **LLAMA_7B),
        # a prompt of 65536 tokens brought down to 4096 rows
        dict(name="evict_prompt", kind="evict", B=1, ctx_lo=65536, ctx_hi=65536, budget=4096, sink=16, recent=512, **LLAMA_7B),
        # a small float32 model; one of the sequences may have nothing to evict yet
        dict(name="evict_small_f32", kind="evict", B=3, ctx_lo=100, ctx_hi=700, budget=333, sink=1, recent=33, H=4, Hkv=4,
             dh=64, dtype="f32"),
    ]


# ---- drawn cases -------------------------------------------------------------------------------------------------
def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _heads(rng, dtype):
    """(H, Hkv, dh): every head with keys of its own, or groups of up to eight that share them."""
    dh = rng.choice([128, 128, 128, 64, 96, 80] if dtype == "bf16" else [64, 64, 128, 16, 32, 80])
    Hkv = _log_int(rng, 2, 32 if dtype == "bf16" else 12)
    group = rng.choice([1, 1, 2, 4, 5, 8])
    while Hkv * group > 40:
        group = max(1, group // 2)
        Hkv = min(Hkv, 40 // group)
    return Hkv * group, Hkv, dh


def draw(rng):
    kind = rng.choice(["attention", "attention", "weights", "evict"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    H, Hkv, dh = _heads(rng, dtype)
    if kind == "attention":
        B = _log_int(rng, 1, 16)
        nodes = rng.choice([1, 16, 64, 128, rng.randint(1, 128)])
        most = (4 if dtype == "bf16" else 0.25) * 1e8 / (B * H * nodes)  # (row, key) pairs: below the largest listed case's
        hi = _log_int(rng, 8, int(max(16, min(2048, most / 4))))
        return dict(kind=kind, B=B, nodes=nodes, prefix=_log_int(rng, 8, int(max(16, min(32768, most / 2)))),
                    ctx_lo=max(0, hi // rng.randint(1, 8) - rng.randint(0, 3)), ctx_hi=hi, H=H, Hkv=Hkv, dh=dh, dtype=dtype,
                    out=rng.choice(["f32", "bf16"]) if dtype == "bf16" else "f32")
    B = _log_int(rng, 1, 16)
    most = (1 << 21) // (B * Hkv)  # cached rows of a layer: at most 2 M
    hi = _log_int(rng, 64, min(65536, most if dtype == "bf16" else most // 4))
    lo = max(1, hi // rng.randint(1, 4))
    if kind == "weights":
        return dict(kind=kind, B=B, nodes=rng.choice([16, 64, 128, rng.randint(9, 128)]), T=rng.randint(1, 8), ctx_lo=lo,
                    ctx_hi=hi, H=H, Hkv=Hkv, dh=dh, dtype=dtype)
    budget = max(8, int(hi * rng.uniform(0.05, 0.95)))
    return dict(kind=kind, B=B, ctx_lo=lo, ctx_hi=hi, budget=budget, sink=rng.randint(0, min(16, budget // 4)),
                recent=rng.randint(0, budget // 3), H=H, Hkv=Hkv, dh=dh, dtype=dtype)


# ---- inputs ------------------------------------------------------------------------------------------------------
def _randn(g, shape, dtype):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)


def _keys(g, shape, dtype):
    """Unit-scale keys, a few of them (one in 64, and the first) larger: those that rows keep looking at."""
    k = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    heavy = torch.rand(shape[:-1], generator=g, device="cuda") < 1.0 / 64
    heavy[..., 0] = True
    return (k * torch.where(heavy, 3.0, 1.0)[..., None]).to(dtype)


def _i32(g, lo, hi, shape):
    """Uniform in [lo, hi]."""
    return torch.randint(lo, hi + 1, shape, generator=g, device="cuda", dtype=torch.int32)


def _trees(B, N, seed):
    """Trees as the CTC transform builds them: at most 8 deep, node ids in creation order; their ancestor masks."""
    rng = torch.Generator().manual_seed(int(seed))
    words = (N + 63) // 64
    mask, counts = torch.zeros((B, N, words), dtype=torch.int64), []
    for b in range(B):
        n = N if N < 8 else int(torch.randint(3 * N // 4, N + 1, (1,), generator=rng))
        u = torch.rand(N, generator=rng).tolist()
        parent, depth, rows = [-1], [0], [1]
        for i in range(1, n):
            j = int(u[i] * i)
            while depth[j] >= 8:
                j = parent[j]
            parent.append(j)
            depth.append(depth[j] + 1)
            rows.append(rows[j] | 1 << i)
        for i, bits in enumerate(rows):
            for w in range(words):
                v = (bits >> (64 * w)) & 0xFFFFFFFFFFFFFFFF
                mask[b, i, w] = v - (1 << 64) if v >= 1 << 63 else v
        counts.append(n)
    return mask.cuda(), torch.tensor(counts, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    B, H, Hkv, dh = (case[n] for n in ("B", "H", "Hkv", "dh"))
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    cap = case["ctx_hi"] + 16
    s = dict(case=case, kv_cap=cap, scale=1.0 / math.sqrt(dh), ctx_len=_i32(g, case["ctx_lo"], case["ctx_hi"], (B,)),
             kv_off=torch.arange(B, device="cuda", dtype=torch.int64) * (Hkv * cap * dh),
             k_cache=_keys(g, (B, Hkv, cap, dh), dt))
    if case["kind"] != "evict":
        N = case["nodes"]
        s.update(q=_randn(g, (B, H, N, dh), dt), k_tree=_keys(g, (B, Hkv, N, dh), dt))
    if case["kind"] == "attention":
        s["mask"], s["n_nodes"] = _trees(B, N, seed)
        s.update(v_cache=_randn(g, (B, Hkv, cap, dh), dt), v_tree=_randn(g, (B, Hkv, N, dh), dt),
                 k_prefix=_keys(g, (Hkv, case["prefix"], dh), dt), v_prefix=_randn(g, (Hkv, case["prefix"], dh), dt),
                 prefix_len=torch.tensor([case["prefix"]], dtype=torch.int32, device="cuda"),
                 out=torch.zeros((B, H, N, dh), dtype=torch.bfloat16 if case["out"] == "bf16" else torch.float32, device="cuda"),
                 lse=torch.zeros((B, H, N), device="cuda"))
        return s
    # rows in the order in which earlier evictions left them: every position once, the last ones where they were appended
    s["next_pos"] = s["ctx_len"] + 2 * cap
    s["pos"] = torch.argsort(torch.rand((B, Hkv, cap), generator=g, device="cuda"), -1).to(torch.int32)
    tail = s["ctx_len"][:, None, None] - torch.arange(cap, device="cuda")
    s["pos"] = torch.where((tail > 0) & (tail <= cap // 16), s["next_pos"][:, None, None] - tail, s["pos"]).to(torch.int32)
    # weights over several decades; rows that nobody looked at have gathered nothing
    u = torch.rand((B, Hkv, cap), generator=g, device="cuda")
    s["weight"] = torch.where(u < 0.05, 0.0, 1e-3 * (u + 1e-4) ** -1.5 * 0.1)
    if case["kind"] == "weights":
        T = case["T"]
        longest = min(T, N - 1)
        nodes = torch.rand((B, N), generator=g, device="cuda")
        nodes[:, 0] = -1.0  # the path begins at the root
        path = torch.sort(torch.argsort(nodes, -1)[:, :longest + 1], -1).values.to(torch.int32)
        s["accept_len"] = _i32(g, 0, longest, (B,))
        s["accept_nodes"] = torch.full((B, T + 1), -1, dtype=torch.int32, device="cuda")
        s["accept_nodes"][:, :longest + 1] = path
        s["accept_nodes"][torch.arange(T + 1, device="cuda") > s["accept_len"][:, None]] = -1
        # what the attention gave the rows
        s["lse"] = torch.empty((B, H, N), device="cuda")
        for b, L in enumerate(s["ctx_len"].tolist()):
            keys = torch.cat([s["k_cache"][b, :, :L], s["k_tree"][b]], 1).float().transpose(1, 2)
            z = (s["q"][b].float().view(Hkv, -1, dh) * s["scale"]) @ keys
            s["lse"][b] = torch.logsumexp(z, -1).view(H, N)
        return s
    n = case["budget"]
    s.update(v_cache=_randn(g, (B, Hkv, cap, dh), dt), kept=torch.zeros((B, Hkv, n), dtype=torch.int32, device="cuda"),
             weight_out=torch.zeros((B, Hkv, cap), device="cuda"),
             pos_out=torch.zeros((B, Hkv, cap), dtype=torch.int32, device="cuda"), ctx_len_out=torch.zeros_like(s["ctx_len"]))
    return s


# ---- the framework's calls ---------------------------------------------------------------------------------------
@functools.lru_cache(maxsize=None)
def _serving():
    """The context that a serving program keeps for its life."""
    import paper_2412_00061_amd as pkg
    return pkg, pkg.Context(max_batch=16, max_slots=4, max_topk=1, max_vocab_rows=256, max_nodes=128, max_heads=40,
                            max_head_dim=128)


@functools.lru_cache(maxsize=None)
def _workspace(B, H, Hkv, dh, N):
    """The attention's scratch, one for all calls of a shape."""
    pkg, _ = _serving()
    return torch.empty(pkg.prefix_verify_attn_workspace_bytes(B, H, Hkv, dh, N), dtype=torch.uint8, device="cuda")


def _bind(s):
    """The call with its arguments marshalled, as launch loops keep it."""
    pkg, ctx = _serving()
    case = s["case"]
    B, H, Hkv, dh = (case[n] for n in ("B", "H", "Hkv", "dh"))
    code = {"bf16": pkg.binding.CTCSPEC_BF16, "f32": pkg.binding.CTCSPEC_F32}
    dt, cap = code[case["dtype"]], s["kv_cap"]
    if case["kind"] == "attention":
        N = case["nodes"]
        ws = _workspace(B, H, Hkv, dh, N)
        return pkg.prepared(ctx, "prefix_verify_attn", dt, s["q"], s["k_prefix"], s["v_prefix"], s["prefix_len"], case["prefix"],
                            s["k_cache"], s["v_cache"], s["kv_off"], s["ctx_len"], cap, s["k_tree"], s["v_tree"], s["n_nodes"],
                            s["mask"], B, H, Hkv, dh, N, s["scale"], ws, ws.numel(), code[case["out"]], s["out"], s["lse"])
    if case["kind"] == "weights":
        return pkg.prepared(ctx, "kv_weight_update", dt, s["q"], s["lse"], s["k_cache"], s["kv_off"], s["ctx_len"], cap,
                            s["k_tree"], s["accept_len"], s["accept_nodes"], case["T"], B, H, Hkv, dh, case["nodes"], s["scale"],
                            s["weight"], s["pos"], s["next_pos"])
    return pkg.prepared(ctx, "kv_evict", dt, s["k_cache"], s["v_cache"], s["kv_off"], s["ctx_len"], cap, s["weight"], s["pos"],
                        s["next_pos"], B, Hkv, dh, case["budget"], case["sink"], case["recent"], s["kept"], s["weight_out"],
                        s["pos_out"], s["ctx_len_out"])


# ---- the plain forms ---------------------------------------------------------------------------------------------
def _attention(s):
    case = s["case"]
    B, H, Hkv, dh, N = (case[n] for n in ("B", "H", "Hkv", "dh", "nodes"))
    G, cap, P = H // Hkv, s["kv_cap"], case["prefix"]
    q = s["q"].float().view(B, Hkv, G * N, dh) * s["scale"]
    by_head = q.transpose(0, 1).reshape(Hkv, B * G * N, dh)
    kp, vp = s["k_prefix"].float(), s["v_prefix"].float()
    sp = (by_head @ kp.transpose(1, 2)).view(Hkv, B, G, N, P)
    sp.masked_fill_(torch.arange(P, device="cuda") >= s["prefix_len"], -math.inf)
    so = (q @ s["k_cache"].float().transpose(2, 3)).view(B, Hkv, G, N, cap)
    so.masked_fill_((torch.arange(cap, device="cuda") >= s["ctx_len"][:, None])[:, None, None, None], -math.inf)
    st = (q @ s["k_tree"].float().transpose(2, 3)).view(B, Hkv, G, N, N)
    seen = ((s["mask"][..., None] >> torch.arange(64, device="cuda")) & 1).bool().view(B, N, -1)[..., :N]
    node = torch.arange(N, device="cuda") < s["n_nodes"][:, None]
    seen = seen & node[:, None]
    st.masked_fill_(~seen[:, None, None], -math.inf)
    m = torch.maximum(torch.maximum(sp.amax(-1).transpose(0, 1), so.amax(-1)), st.amax(-1))
    pp = sp.sub_(m.transpose(0, 1)[..., None]).exp_()
    po, pt = so.sub_(m[..., None]).exp_(), st.sub_(m[..., None]).exp_()
    total = pp.sum(-1).transpose(0, 1) + po.sum(-1) + pt.sum(-1)
    o = (pp.view(Hkv, B * G * N, P) @ vp).view(Hkv, B, G, N, dh).transpose(0, 1)
    o = o + (po.view(B, Hkv, G * N, cap) @ s["v_cache"].float()).view(B, Hkv, G, N, dh)
    o = o + (pt.view(B, Hkv, G * N, N) @ s["v_tree"].float()).view(B, Hkv, G, N, dh)
    rows = node[:, None, None, :]
    o = torch.where(rows[..., None], o / total[..., None], 0.0).reshape(B, H, N, dh)
    lse = torch.where(rows, m + total.log(), 0.0).reshape(B, H, N)
    return {"out": o.to(s["out"].dtype), "lse": lse}


def _weights(s):
    case = s["case"]
    B, H, Hkv, dh, N, T = (case[n] for n in ("B", "H", "Hkv", "dh", "nodes", "T"))
    G, cap = H // Hkv, s["kv_cap"]
    path = s["accept_nodes"].clamp(0, N - 1).long()
    row = (torch.arange(T + 1, device="cuda") <= s["accept_len"][:, None]) & (s["accept_nodes"] >= 0)
    at = path[:, None, :, None].expand(B, H, T + 1, dh)
    q = s["q"].gather(2, at).float().view(B, Hkv, G * (T + 1), dh) * s["scale"]
    lse = s["lse"].gather(2, at[..., 0]).view(B, Hkv, G * (T + 1), 1)
    live = row[:, None, None, :].expand(B, Hkv, G, T + 1).reshape(B, Hkv, G * (T + 1), 1)
    p = torch.where(live, torch.exp(q @ s["k_cache"].float().transpose(2, 3) - lse), 0.0).sum(2)
    cached = torch.arange(cap, device="cuda") < s["ctx_len"][:, None]
    s["weight"] += torch.where(cached[:, None], p, 0.0)
    kt = s["k_tree"].gather(2, path[:, None, :, None].expand(B, Hkv, T + 1, dh)).float()
    above = torch.arange(T + 1, device="cuda")[:, None] >= torch.arange(T + 1, device="cuda")
    pt = torch.where(live, torch.exp(q @ kt.transpose(2, 3) - lse), 0.0).view(B, Hkv, G, T + 1, T + 1)
    pt = torch.where(above, pt, 0.0).sum((2, 3))
    # new rows behind the cached ones; what falls behind the capacity goes to a column that is cut off again
    to = s["ctx_len"][:, None] + torch.arange(T + 1, device="cuda")
    to = torch.where(row & (to < cap), to, cap).long()[:, None].expand(B, Hkv, T + 1)
    for name, new in (("weight", pt), ("pos", (s["next_pos"][:, None] + torch.arange(T + 1, device="cuda", dtype=torch.int32))[:, None].expand(B, Hkv, T + 1))):
        wide = torch.cat([s[name], s[name][..., :1]], -1)
        s[name].copy_(wide.scatter_(2, to, new)[..., :cap])
    return {"weight": s["weight"], "pos": s["pos"]}


def _evict(s):
    case = s["case"]
    B, Hkv, dh, budget = (case[n] for n in ("B", "Hkv", "dh", "budget"))
    cap = s["kv_cap"]
    at = torch.arange(cap, device="cuda")
    L = s["ctx_len"][:, None, None]
    n = L.clamp(max=budget)
    row = at < L
    guarded = row & ((s["pos"] < case["sink"]) | (s["pos"] >= s["next_pos"][:, None, None] - case["recent"]))
    order = torch.sort(torch.where(row, s["weight"], -math.inf), dim=-1, descending=True, stable=True).indices
    rank = torch.where(guarded, 2, torch.where(row, 1, 0)).gather(-1, order)
    order = order.gather(-1, torch.sort(rank, dim=-1, descending=True, stable=True).indices)
    keep = torch.zeros_like(row.expand(B, Hkv, cap)).scatter(-1, order, (at < n).expand(B, Hkv, cap))
    hole = ~keep & (at < n)
    last = torch.sort(torch.where(keep & (at >= n), at, cap), -1).values
    kept = torch.where(hole, last.gather(-1, (hole.cumsum(-1) - 1).clamp(min=0)), at)
    live, kept = (at < n)[..., :min(budget, cap)], kept[..., :min(budget, cap)]
    kept = torch.where(live, kept, 0)
    width = kept.shape[-1]
    s["kept"].fill_(-1)
    s["kept"][..., :width] = torch.where(live, kept, -1)
    for name in ("weight", "pos"):
        to = s[name + "_out"][..., :width]
        to.copy_(torch.where(live, s[name].gather(-1, kept), to))
    wide = kept[..., None].expand(B, Hkv, width, dh)
    for cache in (s["k_cache"], s["v_cache"]):
        to = cache[:, :, :width]
        to.copy_(torch.where(live[..., None], cache.gather(2, wide), to))
    s["ctx_len_out"].copy_(n[:, 0, 0])
    return {name: s[name] for name in ("kept", "weight_out", "pos_out", "ctx_len_out", "k_cache", "v_cache")}


def run(state):
    kind = state["case"]["kind"]
    if own:
        if "call" not in state:
            state["call"] = _bind(state)
        state["call"]()
        names = {"attention": ("out", "lse"), "weights": ("weight", "pos"),
                 "evict": ("kept", "weight_out", "pos_out", "ctx_len_out", "k_cache", "v_cache")}[kind]
        return {n: state[n] for n in names}
    return {"attention": _attention, "weights": _weights, "evict": _evict}[kind](state)


# ---- what a pass cannot do without -------------------------------------------------------------------------------
def work(case):
    B, H, Hkv, dh = (case[n] for n in ("B", "H", "Hkv", "dh"))
    e = 4 if case["dtype"] == "f32" else 2
    L = 0.5 * (case["ctx_lo"] + case["ctx_hi"])
    if case["kind"] == "attention":
        N, P = case["nodes"], case["prefix"]
        n = N if N < 8 else 0.875 * N  # nodes that the trees have
        return {"bytes": 2.0 * e * dh * Hkv * (P + B * (L + n)) + B * H * n * (dh * (e + (2 if case["out"] == "bf16" else 4)) + 4),
                "flops": 4.0 * B * H * n * dh * (P + L + n)}
    if case["kind"] == "weights":
        r = 1 + 0.5 * min(case["T"], case["nodes"] - 1)
        return {"bytes": B * Hkv * (L * (e * dh + 8.0) + 2 * r * (e * dh + 4.0)) + e * B * H * r * dh,
                "flops": 2.0 * r * B * H * L * dh}
    # weight and position of every row, the table of the kept ones with theirs; of K and V the rows from behind the budget that
    # stay, read and written: the recent ones and the budget's share of the others
    n = min(L, case["budget"])
    tail = L - n
    fresh = min(tail, case["recent"], L / 16)
    moved = fresh + (tail - fresh) * max(0.0, n - fresh) / max(1.0, L - fresh)
    return {"bytes": B * Hkv * (8.0 * L + 12.0 * n + 4.0 * e * dh * moved), "flops": 10.0 * B * Hkv * L}


# ---- the same outputs in 64 bits ---------------------------------------------------------------------------------
def _exact_attention(s):
    case = s["case"]
    B, H, N, dh = s["q"].shape
    out, lse = torch.zeros((B, H, N, dh), dtype=torch.float64, device="cuda"), torch.zeros((B, H, N), dtype=torch.float64, device="cuda")
    bit = torch.arange(64, device="cuda")
    counts, lengths = s["n_nodes"].tolist(), s["ctx_len"].tolist()
    for b in range(B):
        n, L = counts[b], lengths[b]
        see = torch.ones((n, case["prefix"] + L + n), dtype=torch.bool, device="cuda")
        see[:, case["prefix"] + L:] = ((s["mask"][b, :n, :, None] >> bit) & 1).reshape(n, -1)[:, :n].bool()
        for h in range(H):
            hk = h * case["Hkv"] // H
            keys = torch.cat([s["k_prefix"][hk], s["k_cache"][b, hk, :L], s["k_tree"][b, hk, :n]]).double()
            vals = torch.cat([s["v_prefix"][hk], s["v_cache"][b, hk, :L], s["v_tree"][b, hk, :n]]).double()
            z = torch.where(see, s["scale"] * (s["q"][b, h, :n].double() @ keys.t()), -math.inf)
            lse[b, h, :n] = torch.logsumexp(z, -1)
            out[b, h, :n] = torch.softmax(z, -1) @ vals
    return {"out": out, "lse": lse}


def _exact_weights(s):
    case = s["case"]
    G = case["H"] // case["Hkv"]
    weight, pos = s["weight"].double(), s["pos"].clone()
    for b, (L, a) in enumerate(zip(s["ctx_len"].tolist(), s["accept_len"].tolist())):
        nodes = s["accept_nodes"][b, :a + 1].long()
        new = max(0, min(a + 1, s["kv_cap"] - L))
        for hk in range(case["Hkv"]):
            keys = torch.cat([s["k_cache"][b, hk, :L], s["k_tree"][b, hk, nodes]]).double()
            total = torch.zeros(L + a + 1, dtype=torch.float64, device="cuda")
            for h in range(hk * G, hk * G + G):
                w = torch.exp(s["scale"] * (s["q"][b, h, nodes].double() @ keys.t()) - s["lse"][b, h, nodes].double()[:, None])
                w[:, L:] = torch.tril(w[:, L:])
                total += w.sum(0)
            weight[b, hk, :L] += total[:L]
            weight[b, hk, L:L + new] = total[L:L + new]
        pos[b, :, L:L + new] = s["next_pos"][b] + torch.arange(new, device="cuda", dtype=torch.int32)
    return {"weight": weight, "pos": pos}


def _exact_evict(s):
    import numpy as np
    case, budget = s["case"], s["case"]["budget"]
    weight, pos = s["weight"].cpu().numpy().astype(np.float64), s["pos"].cpu().numpy()
    out = {"kept": np.full((case["B"], case["Hkv"], budget), -1, dtype=np.int32), "weight_out": np.zeros_like(weight),
           "pos_out": np.zeros_like(pos), "ctx_len_out": np.minimum(s["ctx_len"].cpu().numpy(), budget)}
    rows = np.tile(np.arange(s["kv_cap"]), (case["B"], case["Hkv"], 1))  # which old row every row of the caches is
    for b, (L, end) in enumerate(zip(s["ctx_len"].tolist(), s["next_pos"].tolist())):
        n = min(L, budget)
        for h in range(case["Hkv"]):
            w, p = weight[b, h, :L], pos[b, h, :L]
            free = ~((p < case["sink"]) | (p >= end - case["recent"]))
            chosen = np.sort(np.lexsort((np.arange(L), -w, free))[:n])
            rows[b, h, np.setdiff1d(np.arange(n), chosen)] = chosen[chosen >= n]
            k = rows[b, h, :n]
            out["kept"][b, h, :n], out["weight_out"][b, h, :n], out["pos_out"][b, h, :n] = k, w[k], p[k]
    at = torch.from_numpy(rows).cuda()[..., None]
    out.update({name: torch.take_along_dim(s[name], at, 2).double() for name in ("k_cache", "v_cache")})
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"attention": _exact_attention, "weights": _exact_weights, "evict": _exact_evict}[case["kind"]](s)

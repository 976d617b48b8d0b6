"""The workloads of the 4-bit cache and of the filtered draw: keys and values that join a cache held in 4 bits and are read back
from it, the verification attention over such a cache with and without a sliding window, and the target's token drawn under
per-sequence sampling filters.

  store       the rows of a prompt appended to a layer's 4-bit cache, and read back as what they stand for
              (kv_append_q4, kv_read_q4)
  commit      the accepted path appended to it, and read back (kv_commit_q4, kv_read_q4)
  attention   one layer of the tree-masked verification attention over a 4-bit cache; with a window, rows see the last positions
              and the first few (q4_verify_attn)
  sample      the target's token after every node under temperature, top-k, top-p and min-p (verify_sample_filtered)

`run` computes them in elementary operations - float32, and 64 bits where cut-offs are compared -, or through the package's calls
where `own` is set.  Sizes are those of the workloads in `workloads/configs.py` (7B shapes, the ragged batch of eight), generic grouped
heads, and histories up to the lengths for which a cache is held in 4 bits.
"""
import functools
import math

import torch

own = False

LLAMA_7B = dict(H=32, Hkv=32, dh=128, dtype="bf16")


def listed():
    return [
        # a prompt of 4096 tokens goes into the cache of one layer: bound by its bytes
        dict(name="store_prompt", kind="store", B=1, rows_lo=4096, rows_hi=4096, ctx_lo=0, ctx_hi=0, **LLAMA_7B),
        # continued prompts of several lengths of a small float32 model, a head dimension that fills no whole block of 32
        dict(name="store_odd_f32", kind="store", B=3, rows_lo=100, rows_hi=777, ctx_lo=1, ctx_hi=333, H=6, Hkv=3, dh=80,
             dtype="f32"),
        # the ragged batch of eight: up to nine accepted rows behind 256 to 2048 cached ones: latency
        dict(name="commit_step_b8", kind="commit", B=8, nodes=64, T=8, ctx_lo=256, ctx_hi=2048, **LLAMA_7B),
        # grouped heads, one sequence
        dict(name="commit_grouped_b1", kind="commit", B=1, nodes=128, T=5, ctx_lo=5000, ctx_hi=5000, H=40, Hkv=8, dh=128,
             dtype="bf16"),
        # plain decoding of the ragged batch, one token per sequence: latency
        dict(name="attn_token_b8", kind="attention", B=8, nodes=1, ctx_lo=256, ctx_hi=2048, window=0, sink=0, out="f32", **LLAMA_7B),
        # single tokens behind long histories, grouped heads: bound by the cache's bytes
        dict(name="attn_token_long", kind="attention", B=4, nodes=1, ctx_lo=16384, ctx_hi=65536, window=0, sink=0, out="bf16", H=32,
             Hkv=8, dh=128, dtype="bf16"),
        # the ragged batch of eight with 64-node trees
        dict(name="attn_tree_b8", kind="attention", B=8, nodes=64, ctx_lo=256, ctx_hi=2048, window=0, sink=0, out="f32", **LLAMA_7B),
        # 64-node trees behind documents of 32768 tokens: bound by the products
        dict(name="attn_document", kind="attention", B=4, nodes=64, ctx_lo=32768, ctx_hi=32768, window=0, sink=0, out="bf16",
             **LLAMA_7B),
        # the same trees where rows see the last 4096 positions and the first 16
        dict(name="attn_window_b8", kind="attention", B=8, nodes=64, ctx_lo=16384, ctx_hi=32768, window=4096, sink=16, out="bf16",
             **LLAMA_7B),
        # grouped heads, odd sizes, a short window, sequences that have hardly begun
        dict(name="attn_window_odd", kind="attention", B=13, nodes=25, ctx_lo=0, ctx_hi=5003, window=777, sink=5, out="f32", H=40,
             Hkv=8, dh=80, dtype="bf16"),
        # plain decoding of a batch of eight, filters of each request's own: latency
        dict(name="sample_token_b8", kind="sample", B=8, nodes=1, V=32000),
        # the ragged batch of eight with 64-node trees: a draw at every node
        dict(name="sample_tree_b8", kind="sample", B=8, nodes=64, V=32000),
    ]


# ---- drawn cases -------------------------------------------------------------------------------------------------
def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _heads(rng):
    """(H, Hkv, dh): every head with keys of its own, or groups of up to eight that share them."""
    dh = rng.choice([128, 128, 128, 64, 96, 80, 32])
    Hkv = _log_int(rng, 2, 32)
    group = rng.choice([1, 1, 2, 4, 5, 8])
    while Hkv * group > 40:
        group = max(1, group // 2)
        Hkv = min(Hkv, 40 // group)
    return Hkv * group, Hkv, dh


def draw(rng):
    kind = rng.choice(["store", "commit", "attention", "attention", "attention", "sample", "sample"])
    if kind == "sample":
        V = _log_int(rng, 100, 65533)
        B = _log_int(rng, 1, 16)
        most = 8 * 64 * 32000 // (V * B)  # nodes: no more logits than the largest listed case
        return dict(kind=kind, B=B, nodes=max(1, min(most, rng.choice([1, 16, 64, rng.randint(1, 128)]))), V=V)
    H, Hkv, dh = _heads(rng)
    B = _log_int(rng, 1, 16)
    if kind == "store":
        rows = _log_int(rng, 1, max(2, min(8192, 4096 * 32 // (B * Hkv))))
        ctx = rng.randint(0, 1000)
        return dict(kind=kind, B=B, rows_lo=max(1, rows // rng.randint(1, 4)), rows_hi=rows, ctx_lo=ctx // 2, ctx_hi=ctx, H=H, Hkv=Hkv,
                    dh=dh, dtype=rng.choice(["bf16", "bf16", "f32"]))
    if kind == "commit":
        hi = _log_int(rng, 1, 8192)
        return dict(kind=kind, B=B, nodes=rng.choice([16, 64, 128, rng.randint(9, 128)]), T=rng.randint(1, 8), ctx_lo=hi // 2, ctx_hi=hi,
                    H=H, Hkv=Hkv, dh=dh, dtype=rng.choice(["bf16", "bf16", "f32"]))
    nodes = rng.choice([1, 1, 16, 64, 128, rng.randint(1, 128)])
    most = min(2.5e8 / (B * H * nodes), 1.5e6 / (B * Hkv))  # (row, key) pairs and cached rows: below the largest listed cases'
    hi = _log_int(rng, 8, int(max(16, min(65536, most))))
    window, sink = 0, 0
    if rng.random() < 0.5:
        window, sink = _log_int(rng, 1, hi + 16), rng.choice([0, 1, 4, rng.randint(0, 64)])
    return dict(kind=kind, B=B, nodes=nodes, ctx_lo=max(0, hi // rng.randint(1, 8) - rng.randint(0, 3)), ctx_hi=hi, window=window,
                sink=sink, out=rng.choice(["f32", "bf16"]), H=H, Hkv=Hkv, dh=dh, dtype="bf16")


# ---- the format --------------------------------------------------------------------------------------------------
# Rows of dh elements in blocks of 32, the last one filled up with zeros: 4-bit codes (sign, then 0 0.5 1 1.5 2 3 4 6), two in a byte,
# the even element in the low half, and for each block the exponent e of its scale 2^e as the byte e + 127.
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _blocks(dh):
    return (dh + 31) // 32


def _encode(x):
    """x [.., dh] -> codes [.., 16 blocks], scales [.., blocks].  The exponent is the smallest with |x| <= 7 2^e in the block, the code
    the nearest value, ties to the even code."""
    x = x.float()
    x = torch.nn.functional.pad(x, (0, -x.shape[-1] % 32)).unflatten(-1, (-1, 32))
    amax = x.abs().amax(-1)
    part, e = torch.frexp(amax)
    e = torch.where(amax > 0, e - torch.where(part <= 0.875, 3, 2), -125).clamp(-125, 125)
    a = torch.ldexp(x, -e[..., None])
    sign, a = (a < 0), a.abs()
    code = ((a > 0.25).byte() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)).byte()
    code = (code + 8 * (sign & (code > 0))).byte().flatten(-2)
    return code[..., 0::2] + 16 * code[..., 1::2], (e + 127).byte()


def _decode(codes, scales, dh):
    """float32 [.., dh]."""
    table = torch.tensor(GRID + tuple(-v for v in GRID), device="cuda")
    x = table[torch.stack([codes & 15, codes >> 4], -1).flatten(-2).int()].unflatten(-1, (-1, 32))
    return torch.ldexp(x, scales.int()[..., None] - 127).flatten(-2)[..., :dh]


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
    """Trees as the CTC transform builds them: at most 8 deep, node ids in creation order; masks, depths and node counts."""
    rng = torch.Generator().manual_seed(int(seed))
    words = (N + 63) // 64
    mask, depths, counts = torch.zeros((B, N, words), dtype=torch.int64), torch.full((B, N), -1, dtype=torch.int32), []
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
        depths[b, :n] = torch.tensor(depth)
        counts.append(n)
    return mask.cuda(), depths.cuda(), torch.tensor(counts, dtype=torch.int32, device="cuda")


def _pick(g, values, B):
    return torch.tensor(values, device="cuda")[_i32(g, 0, len(values) - 1, (B,)).long()]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    B = case["B"]
    if case["kind"] == "sample":
        N, V = case["nodes"], case["V"]
        z = 2.5 * torch.randn((B, N, V), generator=g, device="cuda")
        # about two dozen tokens that the model means
        favoured = torch.rand((B, N, V), generator=g, device="cuda") < 24.0 / V
        z = torch.where(favoured, 9 + z, z)
        n = N if N < 8 else _i32(g, 3 * N // 4, N, (B,))
        return dict(case=case, logits=z, n_nodes=n if torch.is_tensor(n) else torch.full((B,), N, dtype=torch.int32, device="cuda"),
                    uniforms=torch.rand((B, N), generator=g, device="cuda"),
                    temperature=_pick(g, [1.0, 1.0, 0.7, 1.3, 0.0], B), top_k=_pick(g, [0, 20, 50, 1000], B).int(),
                    top_p=_pick(g, [1.0, 0.95, 0.9, 0.5], B), min_p=_pick(g, [0.0, 0.0, 0.02, 0.1], B),
                    target=torch.zeros((B, N), dtype=torch.int32, device="cuda"),
                    n_kept=torch.zeros((B, N), dtype=torch.int32, device="cuda"), logp=torch.zeros((B, N), device="cuda"))
    H, Hkv, dh = (case[n] for n in ("H", "Hkv", "dh"))
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    rows = {"store": case.get("rows_hi"), "commit": case.get("T", 0) + 1, "attention": 0}[case["kind"]]
    cap, blocks = case["ctx_hi"] + rows + 16, _blocks(dh)
    s = dict(case=case, kv_cap=cap, scale=1.0 / math.sqrt(dh), ctx_len=_i32(g, case["ctx_lo"], case["ctx_hi"], (B,)),
             kv_off=torch.arange(B, device="cuda", dtype=torch.int64) * (Hkv * cap))
    for name, make in (("k", _keys), ("v", _randn)):
        s[name + "_codes"] = torch.empty((B, Hkv, cap, 16 * blocks), dtype=torch.uint8, device="cuda")
        s[name + "_scales"] = torch.empty((B, Hkv, cap, blocks), dtype=torch.uint8, device="cuda")
        for b in range(B):  # (a sequence at a time: the values themselves are eight times as large)
            s[name + "_codes"][b], s[name + "_scales"][b] = _encode(make(g, (Hkv, cap, dh), dt))
    if case["kind"] == "store":
        s.update(k_rows=_keys(g, (B, Hkv, rows, dh), dt), v_rows=_randn(g, (B, Hkv, rows, dh), dt),
                 n_rows=_i32(g, case["rows_lo"], rows, (B,)))
    if case["kind"] != "store":
        N = case["nodes"]
        s.update(k_tree=_keys(g, (B, Hkv, N, dh), dt), v_tree=_randn(g, (B, Hkv, N, dh), dt))
    if case["kind"] == "commit":
        T = case["T"]
        longest = min(T, N - 1)
        nodes = torch.rand((B, N), generator=g, device="cuda")
        nodes[:, 0] = -1.0  # the path begins at the root
        path = torch.sort(torch.argsort(nodes, -1)[:, :longest + 1], -1).values.to(torch.int32)
        s["accept_len"] = _i32(g, 0, longest, (B,))
        s["accept_nodes"] = torch.full((B, T + 1), -1, dtype=torch.int32, device="cuda")
        s["accept_nodes"][:, :longest + 1] = path
        s["accept_nodes"][torch.arange(T + 1, device="cuda") > s["accept_len"][:, None]] = -1
        s["n_rows"] = s["accept_len"] + 1
    if case["kind"] == "attention":
        s["mask"], s["depth"], s["n_nodes"] = _trees(B, N, seed)
        s.update(q=_randn(g, (B, H, N, dh), dt),
                 out=torch.zeros((B, H, N, dh), dtype=torch.bfloat16 if case["out"] == "bf16" else torch.float32, device="cuda"),
                 lse=torch.zeros((B, H, N), device="cuda"))
    else:
        s.update(ctx_len_out=torch.zeros_like(s["ctx_len"]),
                 k_back=torch.zeros((B, Hkv, rows, dh), dtype=dt, device="cuda"), v_back=torch.zeros((B, Hkv, rows, dh), dtype=dt, device="cuda"))
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
    return torch.empty(pkg.q4_verify_attn_workspace_bytes(B, H, Hkv, dh, N), dtype=torch.uint8, device="cuda")


def _bind(s):
    """The calls with their arguments marshalled, as launch loops keep them."""
    pkg, ctx = _serving()
    case = s["case"]
    if case["kind"] == "sample":
        return [pkg.prepared(ctx, "verify_sample_filtered", s["logits"], s["n_nodes"], s["uniforms"], s["temperature"], s["top_k"],
                             s["top_p"], s["min_p"], case["B"], case["nodes"], case["V"], s["target"], s["n_kept"], s["logp"])]
    B, H, Hkv, dh = (case[n] for n in ("B", "H", "Hkv", "dh"))
    code = {"bf16": pkg.binding.CTCSPEC_BF16, "f32": pkg.binding.CTCSPEC_F32}
    dt, cap = code[case["dtype"]], s["kv_cap"]
    cache = pkg.q4_cache(s["k_codes"], s["k_scales"], s["v_codes"], s["v_scales"])
    if case["kind"] == "attention":
        N = case["nodes"]
        ws = _workspace(B, H, Hkv, dh, N)
        return [pkg.prepared(ctx, "q4_verify_attn", dt, s["q"], cache, s["kv_off"], s["ctx_len"], cap, s["k_tree"], s["v_tree"],
                             s["n_nodes"], s["depth"], s["mask"], B, H, Hkv, dh, N, s["scale"], case["window"], case["sink"], ws, ws.numel(),
                             code[case["out"]], s["out"], s["lse"])]
    if case["kind"] == "store":
        rows = case["rows_hi"]
        put = pkg.prepared(ctx, "kv_append_q4", dt, s["k_rows"], s["v_rows"], s["n_rows"], rows, cache, s["kv_off"], s["ctx_len"], cap, B,
                           Hkv, dh, s["ctx_len_out"])
    else:
        rows = case["T"] + 1
        put = pkg.prepared(ctx, "kv_commit_q4", dt, s["k_tree"], s["v_tree"], s["accept_len"], s["accept_nodes"], case["T"], cache,
                           s["kv_off"], s["ctx_len"], cap, B, Hkv, dh, case["nodes"], s["ctx_len_out"])
    return [put, pkg.prepared(ctx, "kv_read_q4", cache, s["kv_off"], s["ctx_len"], s["n_rows"], rows, cap, B, Hkv, dh, dt, s["k_back"],
                              s["v_back"])]


# ---- the plain forms ---------------------------------------------------------------------------------------------
def _stored(s):
    """Rows quantised, put behind the cached ones, read back from there."""
    case = s["case"]
    B, Hkv, dh = (case[n] for n in ("B", "Hkv", "dh"))
    rows = s["k_back"].shape[2]
    j = torch.arange(rows, device="cuda")
    live = j < s["n_rows"][:, None]
    at = (s["ctx_len"][:, None] + j).long()[:, None, :, None]
    for name in ("k", "v"):
        if case["kind"] == "store":
            new = s[name + "_rows"]
        else:
            new = s[name + "_tree"].gather(2, s["accept_nodes"].clamp(min=0).long()[:, None, :, None].expand(B, Hkv, rows, dh))
        for to, fresh in zip((s[name + "_codes"], s[name + "_scales"]), _encode(new)):
            where = at.expand(B, Hkv, rows, to.shape[-1])
            to.scatter_(2, where, torch.where(live[:, None, :, None], fresh, to.gather(2, where)))
        back = _decode(s[name + "_codes"].gather(2, at.expand(B, Hkv, rows, s[name + "_codes"].shape[-1])),
                       s[name + "_scales"].gather(2, at.expand(B, Hkv, rows, s[name + "_scales"].shape[-1])), dh)
        s[name + "_back"].copy_(torch.where(live[:, None, :, None], back.to(s[name + "_back"].dtype), s[name + "_back"]))
    s["ctx_len_out"].copy_(s["ctx_len"] + s["n_rows"])


def _seen(s):
    """Which cached rows [B,N,cap] and which nodes [B,N,N] a node sees; which nodes there are [B,N]."""
    case = s["case"]
    B, N, W, sink = case["B"], case["nodes"], case["window"], case["sink"]
    at = torch.arange(s["kv_cap"], device="cuda")
    L, depth = s["ctx_len"][:, None, None], s["depth"]
    cached = (at < L).expand(B, N, -1)
    tree = ((s["mask"][..., None] >> torch.arange(64, device="cuda")) & 1).bool().view(B, N, -1)[..., :N]
    node = torch.arange(N, device="cuda") < s["n_nodes"][:, None]
    tree = tree & node[:, None]
    if W:
        cached = cached & ((at > L + depth[..., None] - W) | (at < sink))
        tree = tree & ((depth[:, None, :] > depth[..., None] - W) | (L + depth[:, None, :] < sink))
    return cached, tree, node


def _attention(s):
    case = s["case"]
    B, H, Hkv, dh, N = (case[n] for n in ("B", "H", "Hkv", "dh", "nodes"))
    G, cap = H // Hkv, s["kv_cap"]
    cached, tree, node = _seen(s)
    q = s["q"].float().view(B, Hkv, G * N, dh) * s["scale"]
    sc = (q @ _decode(s["k_codes"], s["k_scales"], dh).transpose(2, 3)).view(B, Hkv, G, N, cap)
    sc.masked_fill_(~cached[:, None, None], -math.inf)
    st = (q @ s["k_tree"].float().transpose(2, 3)).view(B, Hkv, G, N, N)
    st.masked_fill_(~tree[:, None, None], -math.inf)
    m = torch.maximum(sc.amax(-1), st.amax(-1))
    pc, pt = sc.sub_(m[..., None]).exp_(), st.sub_(m[..., None]).exp_()
    total = pc.sum(-1) + pt.sum(-1)
    o = (pc.view(B, Hkv, G * N, cap) @ _decode(s["v_codes"], s["v_scales"], dh)).view(B, Hkv, G, N, dh)
    o = o + (pt.view(B, Hkv, G * N, N) @ s["v_tree"].float()).view(B, Hkv, G, N, dh)
    rows = node[:, None, None, :]
    o = torch.where(rows[..., None], o / total[..., None], 0.0).reshape(B, H, N, dh)
    lse = torch.where(rows, m + total.log(), 0.0).reshape(B, H, N)
    return {"out": o.to(s["out"].dtype), "lse": lse}


def _sample(s):
    case = s["case"]
    V = case["V"]
    live = torch.arange(case["nodes"], device="cuda") < s["n_nodes"][:, None]
    t, p = s["temperature"].double()[:, None, None], s["top_p"].double()[:, None, None]
    greedy = t <= 0
    order = torch.sort(s["logits"], dim=-1, descending=True, stable=True)
    w = torch.exp((order.values.double() - order.values[..., :1].double()) / torch.where(greedy, 1.0, t))
    rank = torch.arange(V, device="cuda")
    k = torch.where(greedy, 1, torch.where(s["top_k"][:, None, None] > 0, s["top_k"][:, None, None], V))
    keep = rank < k
    before = torch.cumsum(torch.where(keep, w, 0.0), -1)
    mass = before[..., -1:]
    before = before - torch.where(keep, w, 0.0)
    keep = keep & ((before < p * mass) | (p >= 1) | (rank == 0)) & (w >= s["min_p"].double()[:, None, None])
    n_kept = keep.sum(-1).int()
    weights = torch.zeros_like(w).scatter_(-1, order.indices, torch.where(keep, w, 0.0))
    cum = weights.cumsum(-1)
    token = (cum > s["uniforms"].double()[..., None] * cum[..., -1:]).int().argmax(-1)
    logp = torch.log(weights.gather(-1, token[..., None]) / cum[..., -1:])[..., 0].float()
    return {"target": torch.where(live, token, -1).int(), "n_kept": torch.where(live, n_kept, 0).int(), "logp": torch.where(live, logp, 0.0)}


OUTPUTS = {"store": ("k_back", "v_back", "k_codes", "k_scales", "v_codes", "v_scales", "ctx_len_out"), "attention": ("out", "lse"),
           "sample": ("target", "n_kept", "logp")}
OUTPUTS["commit"] = OUTPUTS["store"]


def run(state):
    kind = state["case"]["kind"]
    if own:
        if "calls" not in state:
            state["calls"] = _bind(state)
        for call in state["calls"]:
            call()
    elif kind in ("attention", "sample"):
        return {"attention": _attention, "sample": _sample}[kind](state)
    else:
        _stored(state)
    return {n: state[n] for n in OUTPUTS[kind]}


# ---- what a pass cannot do without -------------------------------------------------------------------------------
def work(case):
    B = case["B"]
    if case["kind"] == "sample":
        n = case["nodes"] if case["nodes"] < 8 else 0.875 * case["nodes"]
        return {"bytes": 4.0 * B * n * (case["V"] + 4), "flops": 4.0 * B * n * case["V"]}  # maximum, difference, exponential, sum
    H, Hkv, dh = (case[n] for n in ("H", "Hkv", "dh"))
    e, row = 4 if case["dtype"] == "f32" else 2, 17.0 * _blocks(dh)  # bytes of an element, of a row in 4 bits
    if case["kind"] == "attention":
        N, W = case["nodes"], case["window"]
        n, L = N if N < 8 else 0.875 * N, 0.5 * (case["ctx_lo"] + case["ctx_hi"])
        if W:
            L = min(L, W + min(case["sink"], max(0.0, L - W)))
        return {"bytes": 2.0 * B * Hkv * (L * row + n * dh * e) + B * H * n * (dh * (e + (2 if case["out"] == "bf16" else 4)) + 4),
                "flops": 4.0 * B * H * n * dh * (L + n)}
    r = 0.5 * (case["rows_lo"] + case["rows_hi"]) if case["kind"] == "store" else 1 + 0.5 * min(case["T"], case["nodes"] - 1)
    # rows read, written in 4 bits, those read and written as values again; a maximum, a product, a rounding and a product
    return {"bytes": 2.0 * B * Hkv * r * (2.0 * e * dh + 2.0 * row), "flops": 8.0 * B * Hkv * r * dh}


# ---- the same outputs in 64 bits ---------------------------------------------------------------------------------
def _values(codes, scales, dh):
    """What codes stand for: sign, two bits of exponent and one of fraction, times the block's power of two."""
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    e, f = ((c >> 1) & 3).double(), (c & 1).double()
    x = torch.where(e > 0, (1 + f / 2) * torch.exp2(e - 1), f / 2) * (1 - 2 * (c >> 3).double())
    return (x.unflatten(-1, (-1, 32)) * torch.exp2(scales.double() - 127)[..., None]).flatten(-2)[..., :dh]


def _exact_store(s):
    case = s["case"]
    dh, blocks = case["dh"], _blocks(case["dh"])
    grid = torch.tensor(GRID, dtype=torch.float64, device="cuda")
    end = s["ctx_len"] + s["n_rows"]
    res = {n: s[n].clone() for n in ("k_codes", "k_scales", "v_codes", "v_scales")}
    res.update({n: s[n].double() for n in ("k_back", "v_back")}, ctx_len_out=end)
    for b, (L, r) in enumerate(zip(s["ctx_len"].tolist(), s["n_rows"].tolist())):
        for name in ("k", "v"):
            new = s[name + "_rows"][b, :, :r] if case["kind"] == "store" else s[name + "_tree"][b][:, s["accept_nodes"][b, :r].long()]
            x = torch.zeros((case["Hkv"], r, 32 * blocks), dtype=torch.float64, device="cuda")
            x[..., :dh] = new.double()
            x = x.view(case["Hkv"], r, blocks, 32)
            e = torch.ceil(torch.log2(x.abs().amax(-1) / 7).clamp(min=-125.0))
            # (a logarithm may miss an exact power of two)
            e = torch.where(x.abs().amax(-1) > 7 * torch.exp2(e), e + 1, e)
            e = torch.where(x.abs().amax(-1) <= 7 * torch.exp2(e - 1), e - 1, e).clamp(-125, 125)
            y = x / torch.exp2(e)[..., None]
            off = (y.abs()[..., None] - grid).abs()
            near = off.amin(-1, keepdim=True)
            pick = torch.where(off == near, torch.arange(8, device="cuda") % 2, 2).argmin(-1)  # the nearest; of two, the even one
            res[name + "_back"][b, :, :r] = (torch.sign(y) * grid[pick] * torch.exp2(e)[..., None]).flatten(-2)[..., :dh]
            code = (pick + torch.where((y < 0) & (pick > 0), 8, 0)).flatten(-2).byte()
            res[name + "_codes"][b, :, L:L + r] = code[..., 0::2] | code[..., 1::2] << 4
            res[name + "_scales"][b, :, L:L + r] = (e + 127).byte()
    return res


def _exact_attention(s):
    case = s["case"]
    B, H, N, dh = s["q"].shape
    W, sink, group = case["window"], case["sink"], H // case["Hkv"]
    out, lse = torch.zeros((B, H, N, dh), dtype=torch.float64, device="cuda"), torch.zeros((B, H, N), dtype=torch.float64, device="cuda")
    bit = torch.arange(64, device="cuda")
    counts, lengths = s["n_nodes"].tolist(), s["ctx_len"].tolist()
    for b in range(B):
        n, L = counts[b], lengths[b]
        keys = torch.cat([_values(s["k_codes"][b, :, :L], s["k_scales"][b, :, :L], dh), s["k_tree"][b, :, :n].double()], 1)
        vals = torch.cat([_values(s["v_codes"][b, :, :L], s["v_scales"][b, :, :L], dh), s["v_tree"][b, :, :n].double()], 1)
        place = torch.cat([torch.arange(L, device="cuda"), L + s["depth"][b, :n]])  # positions of the keys
        see = torch.ones((n, L + n), dtype=torch.bool, device="cuda")
        see[:, L:] = ((s["mask"][b, :n, :, None] >> bit) & 1).reshape(n, -1)[:, :n].bool()
        if W:
            back = (L + s["depth"][b, :n, None]) - place
            see &= (back < W) | (place < sink)
        for h in range(H):
            z = torch.where(see, s["scale"] * (s["q"][b, h, :n].double() @ keys[h // group].t()), -math.inf)
            lse[b, h, :n] = torch.logsumexp(z, -1)
            out[b, h, :n] = torch.softmax(z, -1) @ vals[h // group]
    return {"out": out, "lse": lse}


def _exact_sample(s):
    import numpy as np
    case = s["case"]
    z = s["logits"].cpu().numpy().astype(np.float64)
    par = {n: s[n].cpu().numpy().astype(np.float64) for n in ("temperature", "top_p", "min_p", "uniforms")}
    target = np.full((case["B"], case["nodes"]), -1, dtype=np.int32)
    kept, logp = np.zeros_like(target), np.zeros(target.shape)
    for b, (n, k) in enumerate(zip(s["n_nodes"].tolist(), s["top_k"].tolist())):
        for i in range(n):
            row = z[b, i]
            best = np.lexsort((np.arange(len(row)), -row))
            if par["temperature"][b] <= 0:
                best = best[:1]
            else:
                row = (row - row.max()) / par["temperature"][b]
                best = best[:k] if k > 0 else best
                mass = np.exp(row[best])
                if par["top_p"][b] < 1:
                    ahead = np.concatenate([[0.0], np.cumsum(mass)[:-1]])
                    best = best[:max(1, int((ahead < par["top_p"][b] * mass.sum()).sum()))]
                best = best[np.exp(row[best]) >= par["min_p"][b]]
            stays = np.sort(best)
            mass = np.exp(row[stays] - row[stays].max())
            cum = np.cumsum(mass)
            at = min(int(np.searchsorted(cum, par["uniforms"][b, i] * cum[-1], side="right")), len(stays) - 1)
            target[b, i], kept[b, i], logp[b, i] = stays[at], len(stays), np.log(mass[at] / cum[-1])
    return {"target": torch.from_numpy(target).cuda(), "n_kept": torch.from_numpy(kept).cuda(), "logp": torch.from_numpy(logp).cuda()}


def exact(case, seed):
    s = prepare(case, seed)
    return {"store": _exact_store, "commit": _exact_store, "attention": _exact_attention, "sample": _exact_sample}[case["kind"]](s)

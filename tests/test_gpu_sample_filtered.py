"""verify_sample_filtered against the float64 oracle: tokens and counts have to be equal, logarithms of probabilities near."""
import ctypes

import numpy as np
import pytest

import oracle
import paper_2412_00061_amd as pkg
from host_context import HostContext

INVALID, UNSUPPORTED = -1, -2
P = 4096


def context():
    return pkg.Context(max_batch=4, max_slots=1, max_topk=1, max_vocab_rows=8, max_nodes=8, max_heads=1, max_head_dim=8)


def run(logits, u, n_nodes=None, t=None, k=None, p=None, m=None, ctx=None, **more):
    import torch
    B, N, _ = logits.shape
    up = lambda x, kind: None if x is None else torch.tensor(np.asarray(x), dtype=kind, device="cuda")  # noqa: E731
    own = ctx is None
    ctx = ctx or context()
    res = pkg.verify_sample_filtered(ctx, torch.from_numpy(np.ascontiguousarray(logits, dtype=np.float32)).cuda(), up([N] * B if n_nodes is None else n_nodes, torch.int32),
                                     up(u, torch.float32), up([1.0] * B if t is None else t, torch.float32), top_k=up(k, torch.int32), top_p=up(p, torch.float32),
                                     min_p=up(m, torch.float32), want_kept=True, want_logp=True, **more)
    res = {n: x.cpu().numpy() for n, x in res.items()}
    if own:
        ctx.close()
    return res


def check(logits, u, n_nodes=None, t=None, k=None, p=None, m=None, **more):
    res = run(logits, u, n_nodes, t, k, p, m, **more)
    B, N, V = logits.shape
    f32 = lambda x, b, default: default if x is None else float(np.float32(x[b]))  # noqa: E731
    for b in range(B):
        for i in range(N):
            got = res["target_sampled"][b, i], res["n_kept"][b, i], res["logp"][b, i]
            if n_nodes is not None and i >= n_nodes[b]:
                assert got == (-1, 0, 0.0)
                continue
            want = oracle.sample_filtered(logits[b, i], float(np.float32(u[b, i])), f32(t, b, 1.0), 0 if k is None else int(k[b]), f32(p, b, 1.0), f32(m, b, 0.0))
            assert got[:2] == want[:2], (b, i, got, want)
            # each weight in the sum may be off by a unit of 2^-45 of the largest, the sum is at least that; one rounding to float
            assert got[2] == want[2] or abs(got[2] - want[2]) <= 2.0 ** -24 * abs(want[2]) + V * 2.0 ** -45, (b, i, got, want)
    return res


def rows(seed, B, N, V, scale=3.0):
    rng = np.random.default_rng(seed)
    return (rng.standard_normal((B, N, V)) * scale).astype(np.float32), rng.random((B, N)).astype(np.float32)


FILTERS = [dict(), dict(k=[1, 40, 1000]), dict(p=[0.9, 0.5, 0.999]), dict(m=[0.05, 0.5, 1e-4]), dict(k=[50, 7, 0], p=[0.8, 0.95, 0.3]),
           dict(k=[100, 300, 5], p=[0.99, 0.9, 0.999], m=[0.01, 0.0, 0.3], t=[0.7, 1.5, 0.3]), dict(t=[0.0, -1.0, 2.0], k=[3, 0, 0], p=[0.5, 1.0, 0.2]),
           dict(t=[1e-30, 1e30, 3.0], p=[0.9, 0.5, 1.0])]


@pytest.mark.gpu
@pytest.mark.parametrize("more", FILTERS)
@pytest.mark.parametrize("N,V", [(3, 1), (5, 7), (2, 1000), (3, 4097), (2, 32000), (2, 65533)])
def test_against_the_oracle(N, V, more):
    check(*rows(V, 3, N, V), **more)


@pytest.mark.gpu
def test_the_longest_rows():
    z, u = rows(5, 1, 2, 262144, 2.0)
    for more in (dict(), dict(k=[100000], p=[0.97]), dict(p=[0.9999], m=[1e-6])):
        check(z, u, **more)


@pytest.mark.gpu
@pytest.mark.parametrize("more", FILTERS + [dict(k=[1025, 2048, 3000], p=[0.31, 0.77, 0.5]), dict(k=[5000, 4999, 1])])
def test_equal_logits(more):
    """Thousands of them: bins that are divided by index."""
    rng = np.random.default_rng(1)
    z = np.stack([np.zeros((3, 5000)), rng.integers(0, 3, (3, 5000)), np.round(rng.standard_normal((3, 5000)))]).astype(np.float32)
    z[0, 1, 77] = 1.0
    z[0, 2] = -0.0
    z[0, 2, ::2] = 0.0
    check(z, rng.random((3, 3)), **more)


@pytest.mark.gpu
def test_shares_that_end_near_a_token():
    """Flat rows of 14000 tokens: a share known to 2^-18 covers a tenth of a token's weight, so of 120 rows about twelve need it exactly;
    temperatures for which it is not taken in float."""
    z, u = rows(17, 3, 40, 14000, 0.2)
    ctx = pkg.Context(max_batch=4, max_slots=1, max_topk=1, max_vocab_rows=8, max_nodes=40, max_heads=1, max_head_dim=8)
    check(z, u, p=[0.9, 0.97, 0.6], ctx=ctx)
    check(z[:, :4], u[:, :4], p=[0.9, 0.97, 0.6], m=[0.0, 0.5, 0.9], ctx=ctx)
    check(z[:, :3], u[:, :3], p=[0.9, 0.5, 0.9], t=[1e-33, 1e33, 2.0], ctx=ctx)
    ctx.close()


@pytest.mark.gpu
def test_no_numbers_and_infinities():
    rng = np.random.default_rng(2)
    z = rng.standard_normal((1, 8, 3001)).astype(np.float32)
    z[0, 0, ::2], z[0, 1, 1::2] = np.nan, -np.inf
    z[0, 2], z[0, 3] = -np.inf, np.nan
    z[0, 4, [5, 99, 2000]] = np.inf
    z[0, 5], z[0, 5, 1234] = -np.inf, -3.4e38
    z[0, 6, 3], z[0, 6, 4] = 3.4e38, -3.4e38
    z[0, 7, 100:] = -1e4  # weights that are 0 in 64 bits
    u = rng.random((1, 8))
    for more in (dict(), dict(k=[10]), dict(p=[0.9]), dict(k=[2000], p=[0.5], m=[0.2]), dict(t=[0.0]), dict(t=[float("nan")]), dict(t=[float("inf")], k=[7]),
                 dict(p=[float("nan")], m=[float("nan")]), dict(p=[0.0]), dict(p=[-2.0]), dict(m=[7.0]), dict(p=[3.0], m=[-1.0], k=[-5])):
        check(z, u, **more)


@pytest.mark.gpu
def test_ends_of_the_uniform_numbers():
    z, _ = rows(3, 1, 6, 500)
    u = np.array([[0.0, np.float32(1 - 2.0 ** -24), 1e-30, 0.5, 0.25, 0.75]])
    for more in (dict(), dict(k=[5]), dict(p=[0.9]), dict(t=[0.0])):
        check(z, u, **more)
    kept = oracle.filter_tokens(z[0, 0], 1.0, 5)[0]
    res = run(z, np.array([[1.0, 5.0, -1.0, np.nan, -0.0, np.inf]]), k=[5])  # outside [0, 1): the ends
    for i, end in enumerate((-1, -1, 0, 0, 0, -1)):
        assert res["target_sampled"][0, i] == oracle.filter_tokens(z[0, i], 1.0, 5)[0][end]
    assert len(kept) == 5


@pytest.mark.gpu
def test_rows_that_are_no_nodes_and_optional_outputs():
    import torch
    z, u = rows(4, 3, 5, 333)
    check(z, u, n_nodes=[5, 0, 3], k=[4, 4, 4])
    check(z, u, n_nodes=[99, -2, 5], p=[0.5, 0.5, 0.5])
    ctx = context()
    want = run(z, u, k=[4, 9, 0])
    got = pkg.verify_sample_filtered(ctx, torch.from_numpy(z).cuda(), torch.full((3,), 5, dtype=torch.int32, device="cuda"), torch.from_numpy(u).cuda(),
                                     torch.ones(3, device="cuda"), top_k=torch.tensor([4, 9, 0], dtype=torch.int32, device="cuda"))
    assert list(got) == ["target_sampled"] and np.array_equal(got["target_sampled"].cpu().numpy(), want["target_sampled"])
    ctx.close()


@pytest.mark.gpu
def test_captured_and_replayed_on_another_stream():
    import torch
    cases = [rows(s, 3, 8, 5003) for s in (7, 8, 9)]
    par = [dict(t=[1.0, 0.5, 0.0], k=[40, 0, 3], p=[0.9, 0.7, 1.0], m=[0.0, 0.01, 0.0]), dict(t=[2.0, 1.0, 1.0], k=[0, 0, 2000], p=[1.0, 1.0, 0.99], m=[0.0, 0.1, 0.0]),
           dict(t=[0.8, 0.8, 0.8], k=[1, 5, 0], p=[0.5, 0.5, 0.5], m=[0.5, 0.0, 0.0])]
    want = [check(z, u, **q) for (z, u), q in zip(cases, par)]
    kinds = dict(t=torch.float32, k=torch.int32, p=torch.float32, m=torch.float32)
    live = {n: torch.zeros(3, dtype=d, device="cuda") for n, d in kinds.items()}
    z, u, n = torch.zeros((3, 8, 5003), device="cuda"), torch.zeros((3, 8), device="cuda"), torch.full((3,), 8, dtype=torch.int32, device="cuda")
    out = {"target_sampled": torch.zeros((3, 8), dtype=torch.int32, device="cuda"), "n_kept": torch.zeros((3, 8), dtype=torch.int32, device="cuda"),
           "logp": torch.zeros((3, 8), device="cuda")}
    stream = torch.cuda.Stream()
    ctx = context()
    torch.cuda.synchronize()
    ctx.set_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        pkg.verify_sample_filtered(ctx, z, n, u, live["t"], top_k=live["k"], top_p=live["p"], min_p=live["m"], want_kept=True, want_logp=True, out=out)
    for rep in range(6):
        i = rep % 3
        z.copy_(torch.from_numpy(cases[i][0])), u.copy_(torch.from_numpy(cases[i][1]))
        for name, t in live.items():
            t.copy_(torch.tensor(par[i][name], dtype=kinds[name]))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(np.array_equal(out[x].cpu().numpy(), want[i][x]) for x in out)
    ctx.close()


# ---- refusals: on the host ---------------------------------------------------------------------------------------
ARGS = dict(logits=P, n=P, u=P, t=P, k=None, p=None, m=None, B=2, N=5, V=100, out=P, kept=None, logp=None)


@pytest.mark.parametrize("key,value,code,text", [(k, None, INVALID, "null pointer") for k in ("logits", "n", "u", "t", "out")] +
                         [(k, v, INVALID, "positive") for k in ("B", "N", "V") for v in (0, -1)] +
                         [("logits", P + 4, INVALID, "aligned"), ("V", 262145, UNSUPPORTED, "V <="), ("B", 65536, UNSUPPORTED, "B <="), ("N", 1 << 22, UNSUPPORTED, "max_nodes <")])
def test_refusals(key, value, code, text):
    HostContext().refuses("verify_sample_filtered", list(dict(ARGS, **{key: value}).values()), code, text)


def test_no_context():
    assert pkg.load_library().verify_sample_filtered(None, *ARGS.values()) == INVALID


def test_the_binding_looks_at_shapes(monkeypatch):
    import torch
    monkeypatch.setattr(pkg.binding, "_ptr", lambda t, dtype=None: None if t is None else ctypes.c_void_p(t.data_ptr()))
    z, u, n, t = torch.zeros((2, 3, 9)), torch.zeros((2, 3)), torch.zeros(2, dtype=torch.int32), torch.ones(2)
    for bad in (dict(uniforms=u[:1]), dict(n_nodes=n[:1]), dict(temperature=t[:1]), dict(top_k=n[:1]), dict(top_p=t[:1]), dict(min_p=t[:1])):
        with pytest.raises(pkg.CtcspecError, match=next(iter(bad))):
            pkg.verify_sample_filtered(None, **dict(dict(logits=z, n_nodes=n, uniforms=u, temperature=t), **bad))

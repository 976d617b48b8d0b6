"""Calls that bring no workspace: it comes from the pool of the context's stream, not of torch's current one, which would hand it on - to a
call on a third stream, say - while the kernels still write there."""
import contextlib

import pytest
import torch

import paper_2412_00061_amd as pkg
from paper_2412_00061_amd import binding


def attention(ctx, dev, **more):
    z = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device=dev)  # noqa: E731
    i = lambda *v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    return pkg.prefix_verify_attn(ctx, z(2, 4, 5, 64), z(2, 9, 64), z(2, 9, 64), i(9), z(2 * 2 * 8 * 64), z(2 * 2 * 8 * 64),
                                  torch.tensor([0, 2 * 8 * 64], device=dev), i(8, 3), 8, z(2, 2, 5, 64), z(2, 2, 5, 64), i(5, 5),
                                  torch.ones((2, 5, 1), dtype=torch.int64, device=dev), 0.125, **more)


def loss(ctx, dev):
    i = lambda *s: torch.ones(s, dtype=torch.int32, device=dev)  # noqa: E731
    return pkg.ctc_loss(ctx, torch.zeros((2, 4, 17), device=dev), i(2, 3), i(2), i(2) * 4, 16)


def layer(ctx, dev):
    z = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device=dev)  # noqa: E731
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device=dev)  # noqa: E731
    weights = pkg.layer_weights(z(256), z(768, 256), z(256, 256), z(256), z(1024, 256), z(256, 512))
    return pkg.draft_layer_forward(ctx, z(1, 2, 256), weights, i(1), z(8 * 256), z(8 * 256), i(1).long(), i(1), 8, 2, 512, 1e-5, 1e4)


@pytest.mark.parametrize("call", [attention, loss, layer])
def test_allocated_on_the_stream_of_the_context(call, monkeypatch):
    """(On the CPU: what is asked for, and on which stream.)"""
    class Context:
        stream, handle = "the context's", None

        class lib:
            prefix_verify_attn = ctc_loss = draft_layer_forward = staticmethod(lambda *a: 0)

        @staticmethod
        def _check(rc, what):
            assert rc == 0

    now, asked, empty = ["current"], [], torch.empty

    @contextlib.contextmanager
    def stream(s):
        now.append(s)
        yield
        now.pop()

    def allocate(*a, **k):
        if k.get("dtype") == torch.uint8:
            asked.append(now[-1])
        return empty(*a, **k)

    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch, "empty", allocate)
    monkeypatch.setattr(binding, "_ptr", lambda t, dtype=None: None)
    call(Context, "cpu")
    assert asked == ["the context's"] and now == ["current"]


@pytest.mark.gpu
def test_two_streams_in_turn():
    """Two contexts on two streams, called in turn without a workspace: the results of a call alone."""
    limits = dict(max_batch=8, max_slots=4, max_topk=1, max_vocab_rows=32, max_nodes=64, max_heads=8, max_head_dim=128)
    g = torch.Generator().manual_seed(3)
    f = lambda *s: torch.randn(s, generator=g).bfloat16().cuda()  # noqa: E731
    i = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    B, H, N, dh, P, cap = 8, 8, 64, 128, 500, 300
    mask = torch.tensor([[[(1 << r) - 1 | 1 << r] if r < 63 else [-1] for r in range(N)]] * B, device="cuda")
    mine = [(f(B, H, N, dh), f(H, P, dh), f(H, P, dh), i([P]), f(B * H * cap * dh), f(B * H * cap * dh),
             torch.arange(B, device="cuda") * (H * cap * dh), i([cap] * B), cap, f(B, H, N, dh), f(B, H, N, dh), i([N] * B), mask, 0.0884)
            for _ in range(2)]
    alone = pkg.Context(**limits)
    want = [pkg.prefix_verify_attn(alone, *m)["out"].clone() for m in mine]
    torch.cuda.synchronize()
    ctxs = [pkg.Context(**limits, stream=torch.cuda.Stream()) for _ in mine]
    out = [[torch.zeros_like(w) for w in want] for _ in range(20)]
    torch.cuda.synchronize()
    for row in out:
        for ctx, m, o in zip(ctxs, mine, row):
            pkg.prefix_verify_attn(ctx, *m, out={"out": o})
    torch.cuda.synchronize()
    for row in out:
        assert all(torch.equal(a, b) for a, b in zip(row, want))
    for ctx in (alone, *ctxs):
        ctx.close()


@pytest.mark.gpu
def test_captured_without_a_workspace():
    """Two calls in a graph, both with scratch of their own making; other tensors come and go between the replays."""
    g = torch.Generator().manual_seed(4)
    f = lambda *s: torch.randn(s, generator=g).bfloat16().cuda()  # noqa: E731
    i = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    B, H, N, dh, P, cap = 3, 4, 33, 64, 200, 100
    args = [(f(B, H, N, dh), f(2, P, dh), f(2, P, dh), i(P), f(B * 2 * cap * dh), f(B * 2 * cap * dh), torch.arange(B, device="cuda") * (2 * cap * dh),
             i(cap, 0, 7), cap, f(B, 2, N, dh), f(B, 2, N, dh), i(N, 1, 20), torch.full((B, N, 1), -1, dtype=torch.int64, device="cuda"), 0.125)
            for _ in range(2)]
    out = [{"out": torch.zeros((B, H, N, dh), device="cuda")} for _ in args]
    stream = torch.cuda.Stream()
    ctx = pkg.Context(max_batch=B, max_slots=1, max_topk=1, max_vocab_rows=16, max_nodes=N, max_heads=H, max_head_dim=dh, stream=stream)
    torch.cuda.synchronize()
    for a, o in zip(args, out):
        pkg.prefix_verify_attn(ctx, *a, out=o)
    torch.cuda.synchronize()
    want = [o["out"].clone() for o in out]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        for a, o in zip(args, out):
            pkg.prefix_verify_attn(ctx, *a, out=o)
    for _ in range(4):
        other = [torch.full((1 << 20,), 7.0, device="cuda") for _ in range(8)]
        for o in out:
            o["out"].zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o["out"], w) for o, w in zip(out, want)) and all((x == 7).all() for x in other)
        del other
    ctx.close()

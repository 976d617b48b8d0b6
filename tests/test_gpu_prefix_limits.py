"""prefix_verify_attn at the ends of what its limits allow: a prefix with room for millions of rows, and calls with more work than it counts."""
import pytest

import paper_2412_00061_amd as pkg

pytestmark = pytest.mark.gpu


def test_room_for_four_million_rows():
    """64 sequences x 128 nodes x 32 heads on one key head behind a prefix whose buffer holds 2^22 rows, 40 of them in use: the bits of a call
    whose buffer holds those."""
    import torch
    B, H, N, dh, P = 64, 32, 128, 16, 40
    g = torch.Generator().manual_seed(1)
    f = lambda *s: torch.randn(s, generator=g).bfloat16().cuda()  # noqa: E731
    i = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    ctx = pkg.Context(max_batch=B, max_slots=1, max_topk=1, max_vocab_rows=16, max_nodes=N, max_heads=H, max_head_dim=dh)
    q, k, v, kt, vt = f(B, H, N, dh), f(1, P, dh), f(1, P, dh), f(B, 1, N, dh), f(B, 1, N, dh)
    mask = torch.full((B, N, 2), -1, dtype=torch.int64, device="cuda")
    none = torch.zeros(8, dtype=torch.bfloat16, device="cuda")
    call = lambda k, v: pkg.prefix_verify_attn(ctx, q, k, v, i([P]), none, none, torch.zeros(B, dtype=torch.int64, device="cuda"), i([0] * B),  # noqa: E731
                                               0, kt, vt, i([N - b for b in range(B)]), mask, 0.25, want_lse=True,
                                               out={"out": torch.zeros((B, H, N, dh), device="cuda"), "lse": torch.zeros((B, H, N), device="cuda")})
    want = call(k, v)
    far = [torch.full((1, 1 << 22, dh), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    far[0][:, :P], far[1][:, :P] = k, v
    got = call(*far)
    assert all(torch.equal(want[n], got[n]) for n in want) and torch.isfinite(got["out"]).all() and got["out"].any()
    ctx.close()


def test_more_work_than_it_counts_is_refused():
    import torch
    ctx = pkg.Context(max_batch=64, max_slots=1, max_topk=1, max_vocab_rows=16, max_nodes=128, max_heads=32, max_head_dim=128)
    ws = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    at = ws.data_ptr()
    for pcap, cap in ((1 << 26, 64), (64, 1 << 26)):
        rc = ctx.lib.prefix_verify_attn(ctx.handle, 1, at, at, at, at, pcap, at, at, at, at, cap, at, at, at, at, 64, 32, 32, 128, 128, 0.1, at,
                                        1 << 20, 0, at, at)
        assert rc == -2 and "units" in ctx.last_error()
    torch.cuda.synchronize()
    assert not ws.any()  # nothing was launched
    ctx.close()

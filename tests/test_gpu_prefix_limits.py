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


@pytest.mark.parametrize("dtype,out", [("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32")])
def test_rows_whose_scores_are_all_minus_infinity(dtype, out):
    """They give no key a weight: as rows that see none."""
    import torch
    t, od = (torch.bfloat16 if x == "bf16" else torch.float32 for x in (dtype, out))
    B, H, N, dh, P, L = 2, 2, 5, 64, 37, 9
    ctx = pkg.Context(max_batch=B, max_slots=1, max_topk=1, max_vocab_rows=16, max_nodes=N, max_heads=H, max_head_dim=dh)
    z = lambda *s: torch.zeros(s, dtype=t, device="cuda")  # noqa: E731
    i = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    q, kp, kc, kt = z(B, H, N, dh), z(H, P, dh), z(B * H * L, dh), z(B, H, N, dh)
    for k in (kp, kc, kt):
        k[..., 0] = -1
    q[0, 1, 2, 0] = float("inf")
    v = [torch.ones_like(k) for k in (kp, kc, kt)]
    res = pkg.prefix_verify_attn(ctx, q, kp, v[0], i(P), kc.view(-1), v[1].view(-1), torch.arange(B, device="cuda") * (H * L * dh), i(L, L), L, kt,
                                 v[2], i(N, N), torch.full((B, N, 1), -1, dtype=torch.int64, device="cuda"), 0.125, out_dtype=od, want_lse=True)
    some = torch.ones((B, H, N), dtype=torch.bool, device="cuda")
    some[0, 1, 2] = False
    assert (res["out"][~some] == 0).all() and torch.isneginf(res["lse"][~some]).all()
    assert ((res["out"][some].float() - 1).abs() <= 2.0 ** -8).all() and torch.isfinite(res["lse"][some]).all()
    ctx.close()

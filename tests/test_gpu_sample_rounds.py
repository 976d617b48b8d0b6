"""verify_sample_filtered where top-p alone takes several rounds to list enough candidates: few parts of the row hold a logit, and their
largest ones do not weigh enough.  Every token is counted once, and every output is written."""
import numpy as np
import pytest

import paper_2412_00061_amd as pkg
from test_gpu_sample_filtered import check

pytestmark = pytest.mark.gpu
SENTINEL = -12345


def checked(logits, u, **more):
    import torch
    B, N, _ = logits.shape
    out = {"target_sampled": torch.full((B, N), SENTINEL, dtype=torch.int32, device="cuda"), "n_kept": torch.full((B, N), SENTINEL, dtype=torch.int32, device="cuda"),
           "logp": torch.full((B, N), float(SENTINEL), device="cuda")}
    check(logits, u, out=out, **more)


def context():
    return pkg.Context(max_batch=4, max_slots=1, max_topk=1, max_vocab_rows=8, max_nodes=8, max_heads=1, max_head_dim=8)


@pytest.mark.parametrize("lowest", range(200, 520, 40))
def test_short_broad_rows(lowest):
    """(Rows of an odd length begin at all four places between 16-byte boundaries.)"""
    ctx = context()
    for V in range(lowest, lowest + 40, 3):
        rng = np.random.default_rng(V)
        z, u = rng.standard_normal((3, 4, V)).astype(np.float32), rng.random((3, 4)).astype(np.float32)
        checked(z, u, p=[0.9, 0.95, 0.99], ctx=ctx)
        checked(z, u, p=[0.9, 0.95, 0.99], m=[0.02, 1e-3, 0.1], ctx=ctx)
    ctx.close()


@pytest.mark.parametrize("V", [3001, 32000, 65533, 128001])
def test_few_tokens_allowed(V):
    """40 to 200 tokens at random places, the others masked."""
    ctx = context()
    for few in range(40, 200, 7):
        rng = np.random.default_rng(few)
        z = np.full((3, 3, V), -np.inf, dtype=np.float32)
        for row in z.reshape(9, V):
            row[rng.choice(V, few, replace=False)] = rng.standard_normal(few)
        u = rng.random((3, 3)).astype(np.float32)
        checked(z, u, p=[0.9, 0.95, 0.99], ctx=ctx)
        checked(z, u, p=[0.8, 0.97, 0.99], m=[0.02, 1e-3, 0.0], ctx=ctx)
    ctx.close()


@pytest.mark.parametrize("V", [1, 2, 3, 5, 9, 13, 40, 160])
def test_hardly_any_parts(V):
    ctx = context()
    rng = np.random.default_rng(V)
    z, u = rng.standard_normal((4, 8, V)).astype(np.float32), rng.random((4, 8)).astype(np.float32)
    checked(z, u, p=[0.5, 0.9, 0.99, 0.9999], ctx=ctx)
    checked(z, u, p=[0.5, 0.9, 0.99, 0.9999], m=[0.3, 0.02, 1e-3, 0.0], ctx=ctx)
    ctx.close()


def test_borders_within_what_the_float_sum_is_off_by():
    """top_p such that the share ends within 2^-22 of it from a token's border, on either side: 2^-22 is less than the 2^-21 that the sum in float is
    trusted to, and more than the 2^-24 that a share rounded to float may move by.  All rows of a sequence have one share, so each has one row."""
    V, B = 14000, 64
    rng = np.random.default_rng(23)
    z = (rng.standard_normal((B, 1, V)) * 0.2).astype(np.float32)
    top_p, open_ends = [], 0
    for b in range(B):
        x = np.sort(z[b, 0].astype(np.float64))[::-1]
        w = np.exp(x - x[0])
        cum = np.cumsum(w) / w.sum()
        border = cum[rng.integers(V // 3, V - 100)]
        share = float(np.float32(border * (1 + (2.0 ** -22 if b % 2 else -2.0 ** -22))))
        top_p.append(share)
        open_ends += np.searchsorted(cum, share * (1 - 2.0 ** -21)) != np.searchsorted(cum, share * (1 + 2.0 ** -21))
        assert np.abs(cum - share).min() > 2.0 ** -26  # (no border within the roundings of 64 bits)
    assert open_ends == B
    ctx = pkg.Context(max_batch=B, max_slots=1, max_topk=1, max_vocab_rows=8, max_nodes=8, max_heads=1, max_head_dim=8)
    checked(z, rng.random((B, 1)).astype(np.float32), p=top_p, ctx=ctx)
    ctx.close()

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

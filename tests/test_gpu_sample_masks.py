"""verify_sample_filtered where logits are masked by the type's lowest value, at every temperature: such a token has a weight of 0, however far its
exponent is."""
import numpy as np
import pytest

from test_gpu_sample_filtered import check

LOWEST = np.finfo(np.float32).min


@pytest.mark.gpu
@pytest.mark.parametrize("more", [dict(), dict(k=[2000, 2000, 50, 300]), dict(p=[0.9, 0.5, 0.99, 0.999]), dict(m=[0.1, 1e-3, 0.5, 1e-30]),
                                  dict(k=[2000, 900, 20, 999], p=[0.9, 0.5, 0.99, 0.999], m=[0.0, 0.1, 0.0, 1e-6])])
@pytest.mark.parametrize("V", [333, 3001, 32000, 65533])
@pytest.mark.parametrize("temperature", [[1e-30, 1e-13, 1e-38, 0.7], [1e-45, 1e-20, 3e38, 1e10]])
def test_lowest_values(V, temperature, more):
    rng = np.random.default_rng(V)
    z = rng.standard_normal((4, 3, V)).astype(np.float32)
    z[:, 0][rng.random((4, V)) < 0.7] = LOWEST
    z[:, 1][rng.random((4, V)) < 0.995] = LOWEST
    z[:, 2] = LOWEST
    z[:, 2, V // 3], z[:2, 2, V // 2] = -LOWEST, 0.0
    check(z, rng.random((4, 3)).astype(np.float32), t=temperature, **more)

"""That the mean-square bounds of test_gpu_fp4_numerics.py see a lost plane: the 64-bit form with queries or probabilities of
fewer bits exceeds them."""
import numpy as np
import pytest
import torch

from fp4_ref import quantised
from tree_cases import rms


def _attend(q, K, V, scale, cut=lambda w: w):
    """One KV head, all keys visible; probabilities up to 1 as the kernels have them, cut in the numerator alone."""
    z = scale * (q @ K.T)
    w = np.exp(z - z.max(1, keepdims=True))
    return cut(w) @ V / w.sum(1, keepdims=True)


def _truncated(x, bits):
    m, e = np.frexp(x)
    return np.ldexp(np.trunc(m * 2.0 ** bits), e - bits)


def _bf16(x):
    return torch.from_numpy(x).to(torch.bfloat16).double().numpy()


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("keys", [34, 130, 1500])
def test_a_lost_plane_exceeds_the_bounds(keys, hd):
    rng = np.random.default_rng([keys, hd])
    spread = np.exp(rng.standard_normal((2, 1, hd)))
    K, V = quantised((rng.standard_normal((2, keys, hd)) * spread).astype(np.float32)).astype(np.float64)
    q = 0.5 * rng.standard_normal((40, hd)).astype(np.float32).astype(np.float64)
    o = _attend(q, K, V, hd ** -0.5)
    off = lambda x: rms(x - o) / rms(o)  # noqa: E731
    # fp32: two planes of eight bits each by truncation, of q, of the probabilities; three are all of their bits
    assert off(_attend(_truncated(q, 16), K, V, hd ** -0.5)) > 1e-6
    assert off(_attend(q, K, V, hd ** -0.5, lambda w: _truncated(w, 16))) > 1e-6
    assert off(_attend(_truncated(q, 24), K, V, hd ** -0.5, lambda w: _truncated(w, 24))) < 1e-7
    # bf16: one plane where two are meant
    q = _bf16(q)
    o = _attend(q, K, V, hd ** -0.5)
    own = rms(_bf16(o) - o)
    assert rms(_bf16(_attend(q, K, V, hd ** -0.5, _bf16)) - o) > 1.01 * own + 2.0 ** -16 * rms(o)

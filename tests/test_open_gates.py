"""gate_norm's gradient of wide open and of closed gates.

The sigmoid's slope e^-|z| / (1 + e^-|z|)^2 falls to zero on both sides, and the gradient
of z has to hold it relative to itself.  An fp32 kernel's e^-|z| is off by |z| EPS / 2
from its rounded exponent and an ulp of its own, 1 + e^-|z| by half of one, each of two
reciprocals by one: (|z| + 8) EPS in all, besides the norm's own error and the result's
rounding.  silu's slope s (1 + z (1 - s)) is held to the same relative to s (1 + |z| (1 - s)),
twice for its two parts.
"""

import numpy as np
import pytest

import layer_ref as ref
from gpu_harness import say
from test_norms import gate_inputs, np64, rounded

GATES = [0.0, 0.5, 4.0, 8.0, 9.5, 12.0, 15.0, 16.0, 16.7, 17.0, 18.0, 20.0, 25.0, 30.0, 60.0, 80.0]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("activation", ["sigmoid", "silu"])
def test_slope_of_open_and_closed_gates(activation, dtype):
    import paper_2609_32114_amd as P
    H, d, eps = 2, 96, 1e-6
    i = gate_inputs(2 * len(GATES), H, d, dtype, 5)
    jitter = np.random.default_rng(6).random((2 * len(GATES), H, d)) * 0.2
    i["z"] = rounded(np.array(GATES + [-z for z in GATES])[:, None, None] + jitter, dtype)
    _, dz, _ = P.gate_norm_backward(*(i[k].cuda() for k in ("dy", "o", "z", "w")), activation=activation, eps=eps)
    o, z, dy = (np64(i[k]).reshape(-1, d) for k in ("o", "z", "dy"))
    t = np.exp(-np.abs(z))
    small, large = t / (1 + t), 1 / (1 + t)
    s, c = np.where(z > 0, large, small), np.where(z > 0, small, large)  # the sigmoid and its complement
    n = dy * o / np.sqrt((o * o).mean(-1, keepdims=True) + eps) * np64(i["w"])
    k, kz = (d / 64 + 24) * ref.EPS, (np.abs(z) + 8) * ref.EPS
    slope, size = (s * c, s * c) if activation == "sigmoid" else (s * (1 + z * c), 2 * s * (1 + np.abs(z) * c))
    off = ref.excess(dz, (n * slope, np.abs(n) * (k * np.abs(slope) + kz * size)), dtype)
    say(f"[norm] {activation} slope {dtype}: {off:.3f}")
    assert off <= 1.0

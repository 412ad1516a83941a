"""The gate's factor and its derivative near and far from 0, in float32, each relative to itself.

Half steps (2^-24 of the number): the exponential 2 for the instruction (a whole step), 2 for what its rounded argument leaves; the sum with 1 one, its reciprocal
2, the products of these, with the gate and with y one each, 4 at most: 11 of a factor.  A derivative is a sum of two terms of such factors, s and x s (1 - s),
each 4 more: 16 of the sum of their sizes.  Numbers below the smallest normal one, 2^-126, may count as 0."""
import numpy as np
import pytest
import torch

from oracle import memory_oracle as oracle
from paper_2603_09221_amd import binding
from tests.memory_inputs import DEV, U, host

pytestmark = pytest.mark.gpu


def gates(count):
    """Both sides of 0, small numbers, all the way to where the exponential leaves float32's range."""
    gen = torch.Generator().manual_seed(count)
    near, far = torch.randn(count, generator=gen), torch.rand(count, generator=gen) * 200.0 - 100.0
    small = torch.randn(count, generator=gen) * 2.0 ** -20
    return torch.cat([near, far, small, torch.tensor([0.0, -0.0, 87.0, -87.0, 103.0, -103.0, 200.0, -200.0, 1e30, -1e30, 3e38, -3e38])])


@pytest.mark.parametrize("activation", ["silu", "sigmoid"])
@pytest.mark.parametrize("features", [40, 4096, 16384])
def test_each_gate_relative_to_itself(activation, features):
    x = gates(30000)
    x = x[:len(x) // features * features].reshape(-1, features).to(DEV)
    x[0, :12] = gates(1)[3:].to(DEV)
    one = torch.ones_like(x)
    r = host(binding.ttc_residual_norm(one, gate=x, activation=activation)["r"])
    got = binding.ttc_residual_norm_backward(one, gate=x, activation=activation, grad_r=one)
    X = np.clip(host(x), -700.0, 700.0)     # (exp(-700) is 0 here)
    act, s, c = oracle.act(X, activation)[0], oracle.act(X, "sigmoid")[0], oracle.act(-X, "sigmoid")[0]     # (1 - s would lose what c has)
    slope = s * c if activation == "sigmoid" else s + X * s * c
    if activation == "silu":
        act = act * np.where(np.abs(host(x)) > 700.0, np.abs(host(x)) / 700.0, 1.0)
    least = 2.0 ** -126 * (2 + np.abs(X))
    assert (np.abs(r - act) <= 11 * U * np.abs(act) + least).all(), float((np.abs(r - act) / (U * np.abs(act) + least)).max())
    assert np.array_equal(host(got["gy"]), r)
    size = s * c if activation == "sigmoid" else s + np.abs(X) * s * c
    off = np.abs(host(got["ggate"]) - slope)
    assert (off <= 16 * U * size + least).all(), float((off / (U * size + least)).max())

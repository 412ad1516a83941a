"""What bfloat16 results of linear attention, forward and gradients, lose beside their own rounding, against the float64 oracle.

The state that queries meet and the products of queries and keys are taken as two bfloat16 numbers each: the second holds what the first, off by
2^-8 at most, leaves, and is off by 2^-8 of that, so that 2^-16 is lost.  Every term of a result passes one of the two, beside the roundings to
float32 that attention_roundings counts: e <= size * (2^-16 + steps), size the same sum over magnitudes.  With R the rounding to bfloat16, y the
number before it and w the exact one, |R(y) - w| <= |R(y) - y| + e <= |R(w) - y| + e <= |R(w) - w| + 2 e, since no bfloat16 number is nearer to y
than R(y).  (Rounded to one bfloat16 number each, results are off by far more.)"""
import numpy as np
import pytest
import torch

from oracle import memory_oracle as oracle
from paper_2603_09221_amd import binding
from tests.memory_inputs import U, attention_roundings, host
from tests.test_gpu_linear_attention_backward import gradient_inputs

pytestmark = pytest.mark.gpu
LENGTHS = [[7], [31], [32, 9], [33], [64, 1, 40], [200], [900]]
HEADS = [(2, 1, 64, 64), (2, 2, 128, 128), (4, 2, 64, 128), (1, 1, 256, 256), (3, 3, 24, 200)]


def near(got, want, size, steps, name):
    rounded = torch.from_numpy(want).float().bfloat16().double().numpy()
    off, bound = np.abs(host(got) - want), np.abs(rounded - want) + 2 * size * (2.0 ** -16 + steps) + 2.0 ** -40 * np.abs(want) + 1e-40
    assert (off <= bound).all(), (name, float((off / bound).max()))


def magnitudes(args):
    return [np.abs(a) if isinstance(a, np.ndarray) and i != 3 else a for i, a in enumerate(args)]


@pytest.mark.parametrize("lengths", LENGTHS)
@pytest.mark.parametrize("heads,heads_qk,dk,dv", HEADS)
@pytest.mark.parametrize("states", [False, True])
def test_results(lengths, heads, heads_qk, dk, dv, states):
    (q, k, v, g, cu), _, first, _ = gradient_inputs(lengths, heads, heads_qk, dk, dv, torch.bfloat16, False, sum(lengths), states)
    got = binding.ttc_linear_attention(q, k, v, g, cu_q=cu, max_q=max(lengths), state=first)
    args = [host(t) for t in (q, k, v, g)] + [[int(i) for i in cu], dk ** -0.5] + ([host(first)] if states else [])
    near(got["out"], oracle.linear_attention(*args)[0], oracle.linear_attention(*magnitudes(args))[0], attention_roundings(dk, max(lengths)) * U, "out")


@pytest.mark.parametrize("lengths", [[1], [3, 6]] + LENGTHS)
@pytest.mark.parametrize("heads,heads_qk,dk,dv", HEADS)
@pytest.mark.parametrize("states", [False, True])
def test_gradients(lengths, heads, heads_qk, dk, dv, states):
    (q, k, v, g, cu), gout, first, glast = gradient_inputs(lengths, heads, heads_qk, dk, dv, torch.bfloat16, False, sum(lengths), states)
    got = binding.ttc_linear_attention_backward(q, k, v, g, gout, cu_q=cu, max_q=max(lengths), state=first, grad_state=glast)
    args = [host(t) for t in (q, k, v, g)] + [[int(i) for i in cu], dk ** -0.5, host(gout)] + ([host(first), host(glast)] if states else [])
    want, size = oracle.linear_attention_gradients(*args), oracle.linear_attention_gradients(*magnitudes(args))
    for name, w, s in zip(("gq", "gk", "gv"), want, size):
        near(got[name], w, s, attention_roundings(max(dk, dv), max(lengths)) * U, name)

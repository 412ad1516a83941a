"""Linear attention where tokens forget much and those behind them nothing, forward and backward, against the float64 oracle.

The weight between two tokens is exp of the decays between them, and of those alone: what the tokens before both have forgotten is in
neither's way.  Where all of 16 or 31 tokens forget strongly, the sums of decays from a chunk's beginning are thousands of times the difference
that counts.  Bounds are those of the other tests of linear attention: none counts a rounding for such a sum."""
import numpy as np
import pytest
import torch

from oracle import memory_oracle as oracle
from paper_2603_09221_amd import binding
from tests import test_gpu_linear_attention as forward
from tests import test_gpu_linear_attention_backward as backward
from tests.memory_inputs import attention_inputs, host

pytestmark = pytest.mark.gpu
CHUNK = 64


def strong_tokens(length, count, per_chunk=(0, 2)):
    """The first `count` tokens of the first and the third chunk, and what lies between the second's sixteens 0 and 2."""
    at = torch.zeros(length, dtype=torch.bool)
    for c in per_chunk:
        at[c * CHUNK:c * CHUNK + count] = True
    at[CHUNK + 3:CHUNK + 12] = True
    return at


@pytest.mark.parametrize("decay", [-20.0, -200.0, -float("inf")])
@pytest.mark.parametrize("count", [16, 31])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_tokens_behind_those_that_forget(decay, count, dtype):
    length = 3 * CHUNK + 59
    q, k, v, g, cu = attention_inputs([length], 2, 2, 64, 64, dtype, seed=count, rate=1e-3)
    g[strong_tokens(length, count).to(g.device)] = decay
    got = binding.ttc_linear_attention(q, k, v, g, cu_q=cu, max_q=length, want_state=True)
    forward.check(q, k, v, g, cu, got["out"], got["state"])


def check_gradients(x, gout, first, glast, got):
    """backward.check, but that first states' gradients below 2^-149, float32's smallest number, are 0 or that: a bound relative to exp(-200) of something
    is nothing that a float32 result could keep."""
    q, k, v, g, cu = x
    want = oracle.linear_attention_gradients(*[host(t) for t in (q, k, v)], host(g), [int(i) for i in cu], q.shape[2] ** -0.5, *[host(t) for t in (gout, first, glast)])[4]
    state, none = host(got["gstate"]), np.abs(want) < 2.0 ** -149
    assert (np.abs(state[none]) <= 2.0 ** -149).all()
    backward.check(x, gout, first, glast, {**got, "gstate": torch.from_numpy(np.where(none, want, state))})


@pytest.mark.parametrize("decay", [-20.0, -200.0, -float("inf")])
@pytest.mark.parametrize("count", [16, 31])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradients_of_tokens_behind_those_that_forget(decay, count, dtype):
    length = 3 * CHUNK + 59
    x, gout, first, glast = backward.gradient_inputs([length], 2, 2, 64, 64, dtype, False, count, True)
    g = x[3]
    g.mul_(1e-3)
    g[strong_tokens(length, count).to(g.device)] = decay
    got = binding.ttc_linear_attention_backward(*x[:4], gout, cu_q=x[4], max_q=length, state=first, grad_state=glast)
    check_gradients(x, gout, first, glast, got)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_decays_that_heads_have_for_good(dtype):
    """One that forgets all, one that forgets much, one a little, one nothing."""
    length = 2 * CHUNK + 40
    x, gout, first, glast = backward.gradient_inputs([length], 4, 2, 64, 64, dtype, True, 3, True)
    x[3].copy_(torch.tensor([-200.0, -20.0, -0.05, 0.0]))
    q, k, v, g, cu = x
    got = binding.ttc_linear_attention(q, k, v, g, cu_q=cu, max_q=length, state=first, want_state=True)
    forward.check(q, k, v, g, cu, got["out"], got["state"], first.double().cpu().numpy())
    got = binding.ttc_linear_attention_backward(q, k, v, g, gout, cu_q=cu, max_q=length, state=first, grad_state=glast)
    backward.check(x, gout, first, glast, got)


@pytest.mark.parametrize("decay", [-104.5, -200.0, -float("inf")])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("length", [40, 4 * CHUNK + 9])
def test_a_decay_that_leaves_nothing_has_no_gradient(decay, dtype, length):
    """dl/dg = exp(g) <R, S> is 0 where exp(g) is 0 in float32, below -104 (2^-150): not what is left of terms that cancel."""
    x, gout, first, glast = backward.gradient_inputs([length, 30], 2, 1, 64, 64, dtype, False, 11, True)
    q, k, v, g, cu = x
    none = torch.zeros(g.shape, dtype=torch.bool)
    none[::7, 0] = none[5::CHUNK, 1] = none[length:length + 1] = True
    g[none.to(g.device)] = decay
    got = binding.ttc_linear_attention_backward(q, k, v, g, gout, cu_q=cu, max_q=length, state=first, grad_state=glast)
    check_gradients(x, gout, first, glast, got)
    assert not got["glog_decay"].cpu()[none].any() and got["glog_decay"].cpu()[~none].all()
    fixed = torch.tensor([decay, -0.1], device=g.device)
    got = binding.ttc_linear_attention_backward(q, k, v, fixed, gout, cu_q=cu, max_q=length, state=first, grad_state=glast)["glog_decay"]
    assert got[0] == 0 and got[1] != 0


@pytest.mark.parametrize("length", [3, CHUNK, 150, 600])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_no_number_reaches_gradients_that_do_not_depend_on_it(length, dtype):
    """NaN and infinities in a token's query, key, value or result's gradient: other heads', other sequences' and the tokens' on the other side keep their
    bits; of the decays' gradients, which are sums along a sequence, other heads' and other sequences'."""
    x, gout, first, glast = backward.gradient_inputs([length, 20], 2, 2, 64, 64, dtype, False, 12, True)
    q, k, v, g, cu = x
    call = lambda: binding.ttc_linear_attention_backward(q, k, v, g, gout, cu_q=cu, max_q=max(length, 20), state=first, grad_state=glast)
    want = call()
    at = length * 2 // 3
    before, own, after = slice(0, at), slice(at, at + 1), slice(at + 1, length)
    keeps = {"q": dict(gq=(before, own, after), gk=(after,), gv=(after,)), "k": dict(gq=(before,), gk=(before, own, after), gv=(before, after)),
             "v": dict(gq=(before,), gk=(before, after), gv=(before, own, after)), "gout": dict(gq=(before, after), gk=(after,), gv=(after,))}
    for value in (float("nan"), float("inf"), -float("inf")):
        for name, t in (("q", q), ("k", k), ("v", v), ("gout", gout)):
            keep = t[at].clone()
            t[at, 0, 5] = value
            got = call()
            t[at] = keep
            for result in ("gq", "gk", "gv", "glog_decay"):
                assert torch.equal(got[result][:, 1], want[result][:, 1]) and torch.equal(got[result][length:], want[result][length:]), (name, result)
            assert torch.equal(got["gstate"][1], want["gstate"][1]) and torch.equal(got["gstate"][0, 1], want["gstate"][0, 1])
            for result, parts in keeps[name].items():
                for part in parts:
                    assert torch.equal(got[result][part, 0], want[result][part, 0]), (name, result, part)
            if name in ("k", "v"):
                assert torch.equal(got["gstate"], want["gstate"])


@pytest.mark.parametrize("heads,heads_qk", [(1, 1), (6, 3)])
@pytest.mark.parametrize("lengths", [[i % 4 for i in range(700)], [3] * 257, [1], [70] * 300])
def test_a_decay_for_good_over_many_sequences(lengths, heads, heads_qk):
    """Its gradient is the sum of those of all tokens: of as many segments as there are sequences, and more; the same bits every time."""
    x, gout, first, glast = backward.gradient_inputs(lengths, heads, heads_qk, 16, 24, torch.float32, True, 14, True)
    call = lambda: binding.ttc_linear_attention_backward(*x[:4], gout, cu_q=x[4], max_q=max(lengths), state=first, grad_state=glast)
    got = call()
    backward.check(x, gout, first, glast, got)
    assert torch.equal(call()["glog_decay"], got["glog_decay"])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradients_of_strong_and_weak_decays_beside_each_other(dtype):
    """-150 at every ninth token of one head, nothing fades in the second, a third forgets now and then and nothing else fades."""
    length = 4 * CHUNK + 20
    x, gout, first, glast = backward.gradient_inputs([length], 3, 3, 64, 64, dtype, False, 15, True)
    g = x[3]
    g[:, 0] = -1e-3
    g[::9, 0] = -150.0
    g[:, 1:] = 0.0
    g[17::50, 2] = -float("inf")
    got = binding.ttc_linear_attention_backward(*x[:4], gout, cu_q=x[4], max_q=length, state=first, grad_state=glast)
    check_gradients(x, gout, first, glast, got)


@pytest.mark.parametrize("length", [40, 3 * CHUNK + 7])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_decay_that_is_nan(length, dtype):
    """It reaches its own and later tokens of its head forward; of the gradients no other head's and no other sequence's, and no query's before it."""
    x, gout, first, glast = backward.gradient_inputs([length, 30], 2, 2, 64, 64, dtype, False, 16, True)
    q, k, v, g, cu = x
    call = lambda: binding.ttc_linear_attention_backward(q, k, v, g, gout, cu_q=cu, max_q=length, state=first, grad_state=glast)
    want, at = call(), length // 2
    g[at, 0] = float("nan")
    got = call()
    for result in ("gq", "gk", "gv", "glog_decay"):
        assert torch.equal(got[result][:, 1], want[result][:, 1]) and torch.equal(got[result][length:], want[result][length:]), result
    assert torch.equal(got["gq"][:at], want["gq"][:at]) and torch.isnan(got["gq"][at:length, 0]).all()
    assert torch.isnan(got["gk"][:at, 0]).all() and torch.isnan(got["gv"][:at, 0]).all() and torch.isnan(got["glog_decay"][at, 0])
    assert torch.equal(got["gstate"][1], want["gstate"][1]) and torch.equal(got["gstate"][0, 1], want["gstate"][0, 1])

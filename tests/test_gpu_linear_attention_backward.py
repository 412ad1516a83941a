"""Gradients of linear attention on the GPU (ttc_linear_attention_backward) against the float64 oracle, differences, and sums over shared heads.

Bounds as in test_gpu_linear_attention: the same sums over magnitudes, with the gradients' rows in the places of queries, keys and values.  A log
decay's gradient passes products of two such sums and a sum over tokens: twice the roundings, of the gradient by magnitudes plus the sums from
where its segment begins."""
import numpy as np
import pytest
import torch

from oracle import memory_oracle as oracle
from paper_2603_09221_amd import binding
from tests.memory_inputs import DEV, HALF, U, attention_inputs, attention_roundings, decays, host

pytestmark = pytest.mark.gpu


def gradient_inputs(lengths, heads, heads_qk, dk, dv, dtype, constant, seed, states):
    x = attention_inputs(lengths, heads, heads_qk, dk, dv, dtype, constant, seed)
    gen = torch.Generator().manual_seed(seed + 1)
    gout = torch.randn(x[2].shape, generator=gen).to(dtype).to(DEV)
    first, glast = (torch.randn((len(lengths), heads, dk, dv), generator=gen).to(DEV) if states else None for _ in range(2))
    return x, gout, first, glast


def check(x, gout, first, glast, got, kv_new=None):
    q, k, v, g, cu = x
    n, dk, dv = q.shape[0], q.shape[2], v.shape[2]
    bf16 = q.dtype == torch.bfloat16
    cu = [int(i) for i in cu]
    args = [host(t) for t in (q, k, v)] + [decays(g, n), cu, dk ** -0.5, host(gout)] + [None if t is None else host(t) for t in (first, glast)]
    want = oracle.linear_attention_gradients(*args)
    size = oracle.linear_attention_gradients(*[np.abs(a) if isinstance(a, np.ndarray) and i != 3 else a for i, a in enumerate(args)])
    longest = max(b - a for a, b in zip(cu, cu[1:]))
    steps = attention_roundings(max(dk, dv), longest) * U
    for name, w, s in zip(("gq", "gk", "gv"), want, size):
        off = np.abs(host(got[name]) - w)
        bound = s * (steps + (2.0 ** -8 + 2.0 ** -15 if bf16 else 0.0)) + HALF[q.dtype] * np.abs(w) + 1e-40
        assert (off <= bound).all(), (name, float((off / bound).max()))
        assert np.linalg.norm(off) <= np.linalg.norm(w) * (1.5 * 2.0 ** -8 if bf16 else 4 * (steps * U) ** 0.5) + 1e-30, name
    gg, sg = want[3], size[3]
    # a sum over the segment's earlier tokens reaches every later one
    reach = np.stack([np.concatenate([np.cumsum(sg[a:b, h]) for a, b in zip(cu, cu[1:])]) for h in range(g.shape[-1])], 1) if n else sg
    if g.dim() == 1:
        gg, reach = gg.sum(0), reach.sum(0)
    off = np.abs(host(got["glog_decay"]) - gg)
    assert (off <= 2 * steps * reach + 1e-40).all(), float((off / (2 * steps * reach + 1e-40)).max())
    if g.dim() == 2:
        assert np.linalg.norm(off) <= np.linalg.norm(gg) * 8 * (steps * U) ** 0.5 + 1e-30
    if first is not None:
        off = np.abs(host(got["gstate"]) - want[4])
        assert (off <= size[4] * steps + 1e-40).all()
        assert np.linalg.norm(off) <= np.linalg.norm(want[4]) * 4 * (steps * U) ** 0.5


@pytest.mark.parametrize("lengths,heads,heads_qk,dk,dv", [
    ([1], 1, 1, 64, 64), ([64], 2, 1, 128, 128), ([65, 0, 3], 3, 3, 8, 24), ([5, 0, 1, 130], 4, 2, 80, 72), ([150], 2, 2, 256, 256), ([100, 64], 2, 1, 128, 256),
    ([200], 4, 1, 256, 40), ([600], 2, 2, 64, 128)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("constant,states", [(False, False), (False, True), (True, True)])
def test_against_oracle(lengths, heads, heads_qk, dk, dv, dtype, constant, states):
    x, gout, first, glast = gradient_inputs(lengths, heads, heads_qk, dk, dv, dtype, constant, sum(lengths), states)
    got = binding.ttc_linear_attention_backward(*x[:4], gout, cu_q=x[4], max_q=max(lengths), state=first, grad_state=glast)
    check(x, gout, first, glast, got)


def test_many_heads_and_sequences_without_segments():
    """Enough of both that a sequence is not cut."""
    lengths = [70, 1, 129] * 12
    x, gout, first, glast = gradient_inputs(lengths, 16, 16, 64, 64, torch.float32, False, 3, True)
    got = binding.ttc_linear_attention_backward(*x[:4], gout, cu_q=x[4], max_q=129, state=first, grad_state=glast)
    cu = [int(i) for i in x[4]]
    few = slice(0, 3)
    part = {k: v[:cu[3]] if k != "gstate" else v[:3] for k, v in got.items()}
    check([t[:cu[3]] for t in x[:4]] + [cu[:4]], gout[:cu[3]], first[few], glast[few], part)


@pytest.mark.parametrize("lengths", [[70] * 90, [(i * 7) % 5 if i % 3 else 0 for i in range(150)] + [900] + [0] * 20 + [66]])
def test_many_sequences(lengths):
    """More sequences than a wavefront has lanes, alike and far from it."""
    x, gout, first, glast = gradient_inputs(lengths, 2, 2, 16, 24, torch.float32, False, 5, True)
    got = binding.ttc_linear_attention_backward(*x[:4], gout, cu_q=x[4], max_q=max(lengths), state=first, grad_state=glast)
    check(x, gout, first, glast, got)


def test_single_tokens_and_no_tokens():
    x, gout, first, glast = gradient_inputs([1] * 9, 2, 2, 64, 64, torch.float32, False, 4, True)
    got = binding.ttc_linear_attention_backward(*x[:4], gout, state=first, grad_state=glast)
    check(x, gout, first, glast, got)
    cu = torch.zeros(3, dtype=torch.int32, device=DEV)
    got = binding.ttc_linear_attention_backward(*(t[:0] for t in x[:4]), gout[:0], cu_q=cu, max_q=0, state=first[:2], grad_state=glast[:2])
    assert torch.equal(got["gstate"], glast[:2]) and got["gq"].shape == (0, 2, 64)
    got = binding.ttc_linear_attention_backward(*(t[:0] for t in x[:3]), x[3][0], gout[:0], cu_q=cu[:1], max_q=0)
    assert not got["glog_decay"].any()


def test_against_differences():
    """Of the float32 forward pass: a step h of one number moves the loss by h times the gradient, but for curvature (of log decays alone; the loss is linear
    in every other number; h^2/6 of the third derivative, which is below the loss by magnitudes) and for the losses' roundings."""
    x, gout, first, glast = gradient_inputs([70, 3], 2, 1, 16, 24, torch.float32, False, 5, True)
    q, k, v, g, cu = x
    got = binding.ttc_linear_attention_backward(q, k, v, g, gout, cu_q=cu, max_q=70, state=first, grad_state=glast)

    def loss():
        y = binding.ttc_linear_attention(q, k, v, g, cu_q=cu, max_q=70, state=first, want_state=True)
        return float((y["out"].double() * gout.double()).sum() + (y["state"].double() * glast.double()).sum())

    out, last = oracle.linear_attention(*[np.abs(host(t)) for t in (q, k, v)], host(g), [0, 70, 73], 0.25, np.abs(host(first)))
    size = (out * np.abs(host(gout))).sum() + (last * np.abs(host(glast))).sum()
    rng = np.random.default_rng(6)
    for t, name, h in ((q, "gq", 0.5), (k, "gk", 0.5), (v, "gv", 0.5), (g, "glog_decay", 2.0 ** -5), (first, "gstate", 0.5)):
        for _ in range(12):
            i = tuple(int(rng.integers(0, s)) for s in t.shape)
            keep = float(t[i])
            t[i] = keep + h
            up, above = loss(), float(t[i])
            t[i] = keep - h
            down, below = loss(), float(t[i])
            t[i] = keep
            slack = attention_roundings(24, 70) ** 0.5 * 2 * U * size / h + (h * h / 6 * size if t is g else 0.0)
            assert abs((up - down) / (above - below) - float(got[name][i])) <= slack, name


def test_beginnings_by_rule_have_no_gradient_and_shared_rows_add_up():
    lengths = [40, 90, 10]
    x, gout, first, glast = gradient_inputs(lengths, 4, 1, 32, 32, torch.float32, False, 7, True)
    q, k, v, g, cu = x
    kv_len = torch.tensor([100, 90, 11], dtype=torch.int32, device=DEV)
    row = torch.tensor([2, 0, 9], dtype=torch.int32, device=DEV)     # the third lies outside
    got = binding.ttc_linear_attention_backward(q, k, v, g, gout, cu_q=cu, max_q=90, state=first, state_row=row, kv_len=kv_len, grad_state=glast)
    began = torch.zeros_like(first)
    began[0] = first[2]
    assert not got["gstate"][1].any() and not got["gstate"][2].any()
    full = binding.ttc_linear_attention_backward(q, k, v, g, gout, cu_q=cu, max_q=90, state=began, grad_state=glast)
    for name in ("gq", "gk", "gv", "glog_decay"):
        assert torch.equal(got[name], full[name]), name
    assert torch.equal(got["gstate"][0], full["gstate"][0])
    apart = binding.ttc_linear_attention_backward(q.expand(-1, 4, -1), k.expand(-1, 4, -1), v, g, gout, cu_q=cu, max_q=90, state=began, grad_state=glast)
    for name in ("gq", "gk"):
        one, sum_ = host(got[name])[:, 0], host(apart[name]).sum(1)
        assert np.abs(one - sum_).max() <= 4 * U * np.abs(host(apart[name])).sum(1).max()
    each = host(full["glog_decay"])
    fixed = binding.ttc_linear_attention_backward(q, k, v, g[0], gout, cu_q=cu, max_q=90, state=began, grad_state=glast)["glog_decay"]
    spread = binding.ttc_linear_attention_backward(q, k, v, g[0].expand(140, 4).contiguous(), gout, cu_q=cu, max_q=90, state=began, grad_state=glast)
    assert fixed.shape == (4,) and np.abs(host(fixed) - host(spread["glog_decay"]).sum(0)).max() <= 140 * U * np.abs(host(spread["glog_decay"])).sum(0).max()
    assert each.shape == (140, 4)


def test_rows_of_nobody_and_strides():
    x, gout, _, _ = gradient_inputs([150], 4, 2, 64, 40, torch.bfloat16, False, 8, False)
    q, k, v, g, _ = x
    cu = torch.tensor([10, 80, 139], dtype=torch.int32, device=DEV)
    names = {"gq": q, "gk": k, "gv": v, "glog_decay": g}
    out = {name: torch.full(t.shape, 7.0, dtype=t.dtype, device=DEV) for name, t in names.items()}
    got = binding.ttc_linear_attention_backward(q, k, v, g, gout, cu_q=cu, max_q=70, out=out)
    for name in names:
        assert (got[name][:10] == 7).all() and (got[name][139:] == 7).all(), name
    fused = torch.zeros((150, 1 + 4 * 64 + 8 * 40), dtype=torch.bfloat16, device=DEV)
    a, b, c, d = (fused[:, at:at + h * e].unflatten(1, (h, e)) for at, h, e in ((1, 2, 64), (129, 2, 64), (257, 4, 40), (417, 4, 40)))
    for to, t in ((a, q), (b, k), (c, v), (d, gout)):
        to.copy_(t)
    again = binding.ttc_linear_attention_backward(a, b, c, g, d, cu_q=cu, max_q=70)
    for name in names:
        assert torch.equal(again[name][10:139], got[name][10:139]), name


def test_captured_and_replayed_beside_an_eager_graph():
    """autograd over both calls, and a captured backward pass, replayed with other work between: every replay has the eager call's bits."""
    class Linear(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v, g, cu):
            ctx.save_for_backward(q, k, v, g, cu)
            return binding.ttc_linear_attention(q, k, v, g, cu_q=cu, max_q=300)["out"]

        @staticmethod
        def backward(ctx, grad):
            q, k, v, g, cu = ctx.saved_tensors
            out = binding.ttc_linear_attention_backward(q, k, v, g, grad, cu_q=cu, max_q=300)
            return out["gq"], out["gk"], out["gv"], out["glog_decay"], None

    x, gout, _, _ = gradient_inputs([300, 20], 2, 1, 64, 64, torch.float32, False, 9, False)
    q, k, v, g = (t.requires_grad_() for t in x[:4])
    Linear.apply(q, k, v, g, x[4]).backward(gout)
    plain = [t.detach() for t in (q, k, v, g)]
    call = lambda **kw: binding.ttc_linear_attention_backward(*plain, gout, cu_q=x[4], max_q=300, **kw)
    want = call()
    for t, name in ((q, "gq"), (k, "gk"), (v, "gv"), (g, "glog_decay")):
        assert torch.equal(t.grad, want[name])
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for _ in range(3):
        for t in out.values():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for name in out:
            assert torch.equal(out[name], want[name])
        plain[1].mul_(-1.0)
        want = call()

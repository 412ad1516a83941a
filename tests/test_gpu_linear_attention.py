"""Linear attention with decays on the GPU (ttc_linear_attention) against the float64 oracle.

A result is a sum over magnitudes of the same call (scale, queries, keys and values by their sizes): it may be off by half a step of that for
each rounding that it passes.  For bfloat16 the products of queries and keys of a chunk are rounded to 8 bits (2^-8 of the size), what queries meet
of the state to 16 (2^-15: the second part is cut off), results to 8.  These are bounds of the worst case; in the norm roundings of either sign
leave at most 1.5 steps' share of the largest of them, for float32 the root of their number."""
import numpy as np
import pytest
import torch

from oracle import memory_oracle as oracle
from paper_2603_09221_amd import binding
from tests.memory_inputs import DEV, HALF, U, attention_inputs, attention_roundings, decays, host

pytestmark = pytest.mark.gpu


def check(q, k, v, g, cu, got, state=None, first=None, scale=None):
    """out (and last states) against the oracle; first: the sequences' first states (float64)."""
    n, dk = q.shape[0], q.shape[2]
    scale = dk ** -0.5 if scale is None else scale
    x, cu, bf16 = [host(t) for t in (q, k, v)], [int(i) for i in cu], q.dtype == torch.bfloat16
    g = decays(g, n)
    want, last = oracle.linear_attention(*x, g, cu, scale, first)
    size, states = oracle.linear_attention(*[np.abs(t) for t in x], g, cu, abs(scale), None if first is None else np.abs(first))
    steps = attention_roundings(dk, max([b - a for a, b in zip(cu, cu[1:])] + [1])) * U
    own = cu[0], cu[-1]
    off = np.abs(host(got) - want)[own[0]:own[1]]
    bound = (size * (steps + (2.0 ** -8 + 2.0 ** -15 if bf16 else 0.0)) + HALF[q.dtype] * np.abs(want))[own[0]:own[1]] + 1e-40
    assert (off <= bound).all(), float((off / bound).max())
    if off.size and np.abs(want).max() > 0:
        assert np.linalg.norm(off) <= np.linalg.norm(want[own[0]:own[1]]) * (1.5 * 2.0 ** -8 if bf16 else 4 * steps ** 0.5 * U ** 0.5)
    if state is not None:
        off = np.abs(host(state) - last)
        assert (off <= states * steps + 1e-40).all()
        assert np.linalg.norm(off) <= np.linalg.norm(last) * 4 * steps ** 0.5 * U ** 0.5 + 1e-40
    return want, last


SIZES = [  # lengths, heads, heads_qk, dk, dv
    ([1], 1, 1, 64, 64), ([63], 2, 2, 64, 64), ([64], 2, 1, 128, 128), ([65], 3, 3, 8, 8), ([5, 0, 1, 130], 4, 2, 80, 72), ([200], 2, 2, 256, 256),
    ([129, 64], 2, 1, 128, 256), ([300], 1, 1, 256, 40), ([7, 6, 5, 8, 1, 0, 2], 5, 5, 32, 136), ([2, 3, 4, 1, 0], 6, 2, 128, 64), ([700], 2, 2, 64, 128)]


@pytest.mark.parametrize("lengths,heads,heads_qk,dk,dv", SIZES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("constant", [False, True])
def test_against_oracle(lengths, heads, heads_qk, dk, dv, dtype, constant):
    q, k, v, g, cu = attention_inputs(lengths, heads, heads_qk, dk, dv, dtype, constant, seed=sum(lengths) + dk)
    out = binding.ttc_linear_attention(q, k, v, g, cu_q=cu, max_q=max(lengths), want_state=True)
    check(q, k, v, g, cu, out["out"], out["state"])


@pytest.mark.parametrize("most", [5, 6, 7, 15, 16, 17])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_few_tokens_on_both_sides_of_the_rules(most, dtype):
    """Sequences that one kernel goes through token by token and the other in chunks."""
    lengths = [most, 0, 1, most - 2, 3]
    q, k, v, g, cu = attention_inputs(lengths, 4, 2, 64, 72, dtype, seed=most)
    first = torch.randn((5, 4, 64, 72), generator=torch.Generator().manual_seed(most)).to(q.device)
    out = binding.ttc_linear_attention(q, k, v, g, cu_q=cu, max_q=most, state=first, want_state=True)
    check(q, k, v, g, cu, out["out"], out["state"], host(first))


@pytest.mark.parametrize("dk,dv", [(64, 64), (128, 128), (256, 256), (24, 200)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_single_tokens_with_rows_of_a_pool(dk, dv, dtype):
    """Rows in any order, one outside the pool, sequences that begin anew by their length; in place, other rows untouched."""
    q, k, v, g, _ = attention_inputs([7], 6, 3, dk, dv, dtype, seed=dk)
    pool = torch.randn((9, 6, dk, dv), generator=torch.Generator().manual_seed(1)).to(DEV)
    row = torch.tensor([8, 2, -1, 0, 5, 9, 3], dtype=torch.int32, device=DEV)
    kv_len = torch.tensor([5, 1, 4, 0, 2, 7, 100], dtype=torch.int32, device=DEV)
    first = np.zeros((7, 6, dk, dv))
    for s in (0, 4, 6):
        first[s] = host(pool[int(row[s])])
    start = pool.clone()
    out = binding.ttc_linear_attention(q, k, v, g, state=pool, state_row=row, kv_len=kv_len, out={"state": pool})
    kept = [s for s in range(7) if s not in (2, 5)]
    last = torch.zeros((7, 6, dk, dv), device=DEV)
    last[kept] = pool[row[kept].long()]
    _, want = oracle.linear_attention(*[host(t) for t in (q, k, v, g)], list(range(8)), dk ** -0.5, first)
    check(q, k, v, g, range(8), out["out"], None, first)
    assert (np.abs(host(last) - want)[kept] <= 8 * U * (np.abs(want[kept]) + np.abs(first[kept])) + 8 * U).all()
    for r in (1, 4, 6, 7):
        assert torch.equal(pool[r], start[r])
    again = binding.ttc_linear_attention(q, k, v, g, state=start, state_row=row, kv_len=kv_len, out={"state": start.clone()})
    assert torch.equal(again["state"], pool) and torch.equal(again["out"], out["out"])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("heads", [1, 40])      # one head of one sequence is cut into segments, forty are less so
def test_a_prompt_in_pieces(dtype, heads):
    """One call, and pieces of odd lengths that go on from each other's states, single tokens among them."""
    n, dk, dv = 1000, 64, 96
    q, k, v, g, cu = attention_inputs([n], heads, heads, dk, dv, dtype, seed=heads)
    whole = binding.ttc_linear_attention(q, k, v, g, cu_q=cu, max_q=n, want_state=True)
    few = slice(0, 1) if heads > 1 else slice(None)
    check(q[:, few], k[:, few], v[:, few], g[:, few], cu, whole["out"][:, few], whole["state"][:, few])
    pool, at, outs = torch.full((1, heads, dk, dv), float("nan"), device=DEV), 0, []
    for m in (1, 63, 2, 64, 65, 300, 1, 4, 5, 495):
        at += m
        c = torch.tensor([0, m], dtype=torch.int32, device=DEV)
        part = slice(at - m, at)
        outs.append(binding.ttc_linear_attention(q[part], k[part], v[part], g[part], cu_q=c, max_q=m, state=pool, out={"state": pool},
                                                 kv_len=torch.tensor([at], dtype=torch.int32, device=DEV))["out"])
    assert at == n
    y, x = torch.cat(outs), whole["out"]
    steps = attention_roundings(dk, n) * U
    size = torch.from_numpy(oracle.linear_attention(*[np.abs(host(t[:, few])) for t in (q, k, v)], host(g[:, few]), [0, n], dk ** -0.5)[0])
    assert ((y - x)[:, few].double().cpu().abs() <= 2 * size * (steps + (2.0 ** -7 if dtype == torch.bfloat16 else 0.0))).all()
    assert float((pool - whole["state"]).norm() / whole["state"].norm()) <= 8 * (steps * U) ** 0.5


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides_alignment_and_rows_of_nobody(dtype):
    """Queries, keys and values where a fused projection left them, at any offset, results into rows of a wider tensor: the same bits; rows that no
    sequence has and entries between heads stay."""
    lengths, heads, dk, dv = [70, 3, 40], 3, 64, 40
    q, k, v, g, cu = attention_inputs([20] + lengths + [9], heads, heads, dk, dv, dtype, seed=2)
    cu = torch.tensor([20, 90, 93, 133], dtype=torch.int32, device=DEV)
    want = binding.ttc_linear_attention(q, k, v, g, cu_q=cu, max_q=70, out={"out": torch.zeros_like(v)})["out"]
    for first in (0, 1, 8):
        fused = torch.zeros((q.shape[0], heads * (2 * dk + dv) + 16), dtype=dtype, device=DEV)
        a, b, c = (fused[:, first:][:, x:x + heads * d].unflatten(1, (heads, d)) for x, d in ((0, dk), (heads * dk, dk), (2 * heads * dk, dv)))
        a.copy_(q), b.copy_(k), c.copy_(v)
        room = torch.full((q.shape[0], heads, dv + 5), 7.0, dtype=dtype, device=DEV)
        got = binding.ttc_linear_attention(a, b, c, g, cu_q=cu, max_q=70, out={"out": room[..., :dv]})["out"]
        assert torch.equal(got[20:133], want[20:133])
        assert (room[..., dv:] == 7).all() and (room[:20] == 7).all() and (room[133:] == 7).all()
    wide = torch.zeros((q.shape[0], 2 * heads), device=DEV)[:, ::2]
    wide.copy_(g)
    assert torch.equal(binding.ttc_linear_attention(q, k, v, wide, cu_q=cu, max_q=70, out={"out": torch.zeros_like(v)})["out"], want)
    across = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v)]
    assert torch.equal(binding.ttc_linear_attention(*across, g, cu_q=cu, max_q=70, out={"out": torch.zeros_like(v)})["out"], want)


def test_tokens_beyond_max_q_and_wild_row_numbers_are_left_out():
    q, k, v, g, _ = attention_inputs([100], 2, 2, 64, 64, torch.float32, seed=4)
    cu = torch.tensor([-5, 50, 40, 100, 4000], dtype=torch.int32, device=DEV)
    room = torch.full_like(v, 7.0)
    got = binding.ttc_linear_attention(q, k, v, g, cu_q=cu, max_q=30, want_state=True, out={"out": room})
    check(q[:30], k[:30], v[:30], g[:30], [0, 30], got["out"][:30], got["state"][:1])
    assert (room[30:40] == 7).all() and (room[70:] == 7).all() and not got["state"][1].any() and not got["state"][3].any()
    check(q[40:70], k[40:70], v[40:70], g[40:70], [0, 30], got["out"][40:70], got["state"][2:3])


@pytest.mark.parametrize("length", [3, 64, 150, 600])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_no_number_reaches_earlier_tokens(length, dtype):
    """NaN and infinities in queries, keys, values of one token: earlier tokens' results and other heads' keep their bits."""
    q, k, v, g, cu = attention_inputs([length, 20], 2, 2, 64, 64, dtype, seed=5)
    call = lambda: binding.ttc_linear_attention(q, k, v, g, cu_q=cu, max_q=length, want_state=True, out={"out": torch.zeros_like(v)})
    want = call()       # (the second sequence's tokens beyond max_q are not written)
    at = length * 2 // 3
    for value in (float("nan"), float("inf"), -float("inf")):
        for t in (q, k, v):
            keep = t[at].clone()
            t[at, 0, 5] = value
            got = call()
            t[at] = keep
            assert torch.equal(got["out"][:at], want["out"][:at]) and torch.equal(got["out"][:, 1], want["out"][:, 1])
            assert torch.equal(got["out"][length:], want["out"][length:]) and torch.equal(got["state"][1], want["state"][1])
            if t is v:      # one column of it
                bad = ~torch.isfinite(got["out"][at:length, 0])
                assert bad[:, 5].all() and not bad[:, :5].any() and not bad[:, 6:].any()
            else:
                assert not torch.isfinite(got["out"][at, 0]).any()
            if t is q:
                assert torch.equal(got["out"][at + 1:], want["out"][at + 1:])


def test_decays_of_zero_infinity_and_nan():
    for length in (3, 130):
        q, k, v, g, cu = attention_inputs([length], 3, 3, 64, 64, torch.float32, seed=6)
        g[:, 0] = 0.0                       # nothing fades
        g[length // 2, 1] = -float("inf")   # begins anew
        g[length // 2, 2] = float("nan")
        got = binding.ttc_linear_attention(q, k, v, g, cu_q=cu, max_q=length, want_state=True)
        fine = slice(0, 2)
        check(q[:, fine], k[:, fine], v[:, fine], g[:, fine].clamp(min=-500.0), cu, got["out"][:, fine], got["state"][:, fine])
        assert torch.isnan(got["out"][length // 2:, 2]).all() and not torch.isnan(got["out"][:length // 2, 2]).any()


def test_strong_and_weak_decays_beside_each_other():
    """Weights are differences of sums: -150 of one token must not cost the next ones their digits."""
    q, k, v, g, cu = attention_inputs([256], 2, 2, 64, 64, torch.float32, seed=7, rate=1e-3)
    g[::9] = -150.0
    got = binding.ttc_linear_attention(q, k, v, g, cu_q=cu, max_q=256, want_state=True)
    check(q, k, v, g, cu, got["out"], got["state"])


def test_many_sequences():
    """More sequences than a wavefront has lanes, most of them empty, one cut into segments."""
    lengths = [(i * 7) % 5 if i % 3 else 0 for i in range(150)] + [1400] + [0] * 20 + [3]
    q, k, v, g, cu = attention_inputs(lengths, 2, 1, 32, 32, torch.float32, seed=8)
    got = binding.ttc_linear_attention(q, k, v, g, cu_q=cu, max_q=1400, want_state=True)
    check(q, k, v, g, cu, got["out"], got["state"])


def test_many_sequences_of_one_length():
    lengths = [130] * 70
    q, k, v, g, cu = attention_inputs(lengths, 1, 1, 16, 16, torch.float32, seed=9)
    got = binding.ttc_linear_attention(q, k, v, g, cu_q=cu, max_q=130, want_state=True)
    check(q, k, v, g, cu, got["out"], got["state"])


def test_no_tokens_leave_states_as_they_are():
    state = torch.randn((3, 2, 16, 24), device=DEV)
    q, v, g = torch.zeros((0, 2, 16), device=DEV), torch.zeros((0, 2, 24), device=DEV), torch.zeros((0, 2), device=DEV)
    cu, kv_len = torch.zeros(4, dtype=torch.int32, device=DEV), torch.tensor([3, 0, 9], dtype=torch.int32, device=DEV)
    for most in (0, 1, 500):
        got = binding.ttc_linear_attention(q, q, v, g, cu_q=cu, max_q=most, state=state, kv_len=kv_len, want_state=True)["state"]
        assert torch.equal(got[0], state[0]) and torch.equal(got[2], state[2]) and not got[1].any()
    assert binding.ttc_linear_attention(q, q, v, g)["out"].shape == (0, 2, 24)


def test_another_stream_a_captured_graph_and_one_workspace():
    """Eager calls, calls on another stream, and replays with other work between, two graphs sharing one workspace: the same bits."""
    q, k, v, g, cu = attention_inputs([900], 2, 2, 64, 64, torch.bfloat16, seed=9)
    state = torch.randn((1, 2, 64, 64), device=DEV)
    call = lambda **kw: binding.ttc_linear_attention(q, k, v, g, cu_q=cu, max_q=900, state=state, **kw)
    want = call(want_state=True)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    got = call(want_state=True, stream=stream)
    stream.synchronize()
    assert torch.equal(got["out"], want["out"]) and torch.equal(got["state"], want["state"])
    workspace = torch.empty(1 << 24, dtype=torch.uint8, device=DEV)
    graphs, outs = [], []
    for _ in range(2):
        out = {"out": torch.zeros_like(v), "state": torch.zeros_like(state)}
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(out=out, workspace=workspace)
        graphs.append(graph)
        outs.append(out)
    for i in range(4):
        for graph, out in zip(graphs, outs):
            out["out"].zero_(), out["state"].zero_()
            workspace.random_(0, 256)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out["out"], want["out"]) and torch.equal(out["state"], want["state"])
        q.mul_(-1.0)
        want = call(want_state=True)

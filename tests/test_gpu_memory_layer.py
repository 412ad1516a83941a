"""Places, norms and linear attention together, as a memory layer is served and trained, against the float64 oracles in the same order; the example's
layer with one in it."""
import numpy as np
import pytest
import torch

from examples import hybrid_layer
from oracle import memory_oracle as oracle
from paper_2603_09221_amd import binding
from tests.memory_inputs import DEV, U, attention_roundings, host

pytestmark = pytest.mark.gpu

HEADS, DK, DV, PAGE, SLOTS = 2, 32, 48, 16, 5
FEATURES = HEADS * (2 * DK + 2 * DV)
SIZES = [HEADS * DK, HEADS * DK, HEADS * DV, HEADS * DV]


def split(h):
    """queries, keys, values and gates of normed features (the keys about as long as 1)"""
    at = np.cumsum([0] + SIZES)
    q, k, v, gate = (h[:, a:b] for a, b in zip(at, at[1:]))
    return q.reshape(len(h), HEADS, DK), k.reshape(len(h), HEADS, DK) * DK ** -0.5, v.reshape(len(h), HEADS, DV), gate


def layer(x, g, **kw):
    h = binding.ttc_residual_norm(x, pre="rms")["h"]
    q, k, v, gate = split(h)
    o = binding.ttc_linear_attention(q, k, v, g, **kw)["out"]
    return o, binding.ttc_residual_norm(o.view(len(x), -1), gate=gate, activation="silu", post="rms", groups=HEADS)["r"]


def layer_oracle(x, g):
    """The layer on one sequence's tokens in float64, and bounds of its float32 errors, to first order.

    h: a sum over the features and 8 roundings more, of each number.  Results of the attention: its own roundings, and those of the three factors of
    each product, of the sum of magnitudes.  The norm: an error E of o gives (E_i + |z_i| rms(E)) / rms(o), and a sum and 8 roundings of z.  silu has a
    slope of at most 1.1 and rounds four times."""
    n, cu = len(x), [0, len(x)]
    _, h = oracle.residual_norm(x, pre="rms")
    q, k, v, gate = split(h)
    gs = np.broadcast_to(g, (n, HEADS))
    o, _ = oracle.linear_attention(q, k, v, gs, cu, DK ** -0.5)
    size, _ = oracle.linear_attention(np.abs(q), np.abs(k), np.abs(v), gs, cu, DK ** -0.5)
    r, _ = oracle.residual_norm(o.reshape(n, -1), gate=gate, activation="silu", post="rms", groups=HEADS)
    of_h = (FEATURES + 8) * U
    e = size * (attention_roundings(DK, n) * U + 3 * of_h)
    rms = np.sqrt((o ** 2).mean(-1, keepdims=True) + 1e-5)
    z = o / rms
    of_z = ((e + np.abs(z) * np.sqrt((e ** 2).mean(-1, keepdims=True))) / rms + np.abs(z) * (DV + 8) * U).reshape(n, -1)
    a, _ = oracle.act(gate, "silu")
    return r, np.abs(a) * of_z + np.abs(z).reshape(n, -1) * (1.1 * np.abs(gate) * of_h + 4 * U * np.abs(a)) + U * np.abs(r)


def test_requests_come_and_go():
    """Prompts of several lengths beside single tokens, then captured steps in which requests end, wait and begin: every token's result as if its
    request had been given whole, and every token on a page of its own."""
    rng = np.random.default_rng(0)
    pages = 40
    table = torch.full((SLOTS, 20), -1, dtype=torch.int32, device=DEV)
    free = torch.from_numpy(rng.permutation(pages).astype(np.int32)).to(DEV)
    count, length = torch.tensor([pages], dtype=torch.int32, device=DEV), torch.zeros(SLOTS, dtype=torch.int32, device=DEV)
    states = torch.full((SLOTS + 3, HEADS, DK, DV), float("nan"), device=DEV)       # rows as they were left
    row = torch.tensor([6, 0, 3, 7, 2], dtype=torch.int32, device=DEV)
    decay = torch.tensor([-0.01, -1.5], device=DEV)
    new, x = torch.zeros(SLOTS, dtype=torch.int32, device=DEV), torch.zeros((SLOTS + 2, FEATURES), device=DEV)
    on_pages = torch.full((pages * PAGE,), -1, dtype=torch.int64, device=DEV)
    requests, ids = [None] * SLOTS, iter(range(10 ** 6))

    def serve(x, max_q):
        at = binding.ttc_kv_place(length, new, table, PAGE, len(x), pages=pages, free=free, free_count=count, out={"kv_len": length, "free_count": count})
        o, r = layer(x, decay, cu_q=at["cu_q"], max_q=max_q, state=states, state_row=row, kv_len=length, out={"state": states, "out": torch.zeros(
            (len(x), HEADS, DV), device=DEV)})
        return at, r

    def turn(asked, run, rows):
        """Tokens for the slots that ask, on the host and the device; then what `run` gives for them against the oracle."""
        given = []
        for s, n in enumerate(asked):
            if n < 0:
                requests[s] = None
            elif n > 0:
                old = requests[s] or (np.zeros((0, FEATURES)), [])
                more = rng.standard_normal((n, FEATURES)).astype(np.float32)
                requests[s] = np.concatenate([old[0], more]), old[1] + [next(ids) for _ in range(n)]
                given.append((s, more))
        feed = np.concatenate([m for _, m in given] + [np.full((rows - sum(len(m) for _, m in given), FEATURES), 1.0, dtype=np.float32)])
        new.copy_(torch.tensor(asked, dtype=torch.int32))
        at, r = run(torch.from_numpy(feed).to(DEV))
        torch.cuda.synchronize()
        got, first, slots = host(r), 0, at["slots"].cpu()
        for s, m in given:
            tokens, own = requests[s]
            want, bound = layer_oracle(tokens.astype(np.float64), host(decay))
            off = np.abs(got[first:first + len(m)] - want[-len(m):])
            assert (off <= bound[-len(m):]).all(), (asked, s, float((off / bound[-len(m):]).max()))
            on_pages[slots[first:first + len(m)].to(DEV)] = torch.tensor(own[-len(m):], device=DEV)
            first += len(m)
        assert (slots[first:] == -1).all() and int(at["missing"]) == 0
        held, places = table.cpu().numpy(), on_pages.cpu().numpy()
        for s in range(SLOTS):
            assert int(length[s]) == (len(requests[s][1]) if requests[s] else 0)
            if requests[s]:
                p = np.arange(len(requests[s][1]))
                assert np.array_equal(places[held[s, p // PAGE] * PAGE + p % PAGE], requests[s][1])

    for asked in ([70, 0, 3, 130, 1], [1, 65, 1, 0, 17], [1, 1, -1, 1, 1], [0, 2, 90, -1, 4]):
        turn(asked, lambda t: serve(t, max(asked)), sum(max(n, 0) for n in asked) + 3)
    before = [(t, t.clone()) for t in (table, free, count, length, states)]
    new.fill_(1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        serve(x, 1)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        at, r = serve(x, 1)
    for t, old in before:
        t.copy_(old)

    def replay(feed):
        x.copy_(feed)
        graph.replay()
        return at, r

    for asked in ([1, 1, 1, 1, 1], [1, -1, 1, 0, 1], [1, 1, 1, 1, -1], [0, 1, 1, 1, 1], [1, 1, 1, 1, 1]):
        turn(asked, replay, SLOTS + 2)


@pytest.mark.parametrize("lengths", [[1], [5, 0, 130], [64, 200]])
def test_trained_through(lengths):
    """Gradients through norm, attention, gated norm and residual, one call's results given to the next, against the oracle's in the same order.

    Each call's results are within 1e-5 of their norm (the bounds of its own test, of the sizes here); a norm's gradient, a product's or a decay's lets
    what it is given count by less than ten times, and there are three calls on the way: 3e-4."""
    gen = torch.Generator().manual_seed(sum(lengths))
    n, cu = sum(lengths), np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    y, x, w = (torch.randn((n, f), generator=gen).to(DEV) for f in (FEATURES, FEATURES, HEADS * DV))
    wx = torch.randn((n, FEATURES), generator=gen).to(DEV)
    g = -torch.rand((n, HEADS), generator=gen).to(DEV)
    gain = (1 + 0.1 * torch.randn(FEATURES, generator=gen)).to(DEV)
    at = dict(cu_q=torch.from_numpy(cu).to(DEV), max_q=max(lengths))
    first = dict(residual=x, pre="layer", pre_gain=gain)
    last = dict(activation="silu", post="rms", groups=HEADS)

    a = binding.ttc_residual_norm(y, **first)
    q, k, v, gate = split(a["h"])
    o = binding.ttc_linear_attention(q, k, v, g, **at)["out"].view(n, -1)
    b = binding.ttc_residual_norm_backward(o, gate=gate, grad_r=w, **last)      # of the loss sum(w * r) + sum(wx * a["r"])
    c = binding.ttc_linear_attention_backward(q, k, v, g, b["gy"].view(n, HEADS, DV), **at)
    gh = torch.cat([c["gq"].view(n, -1), c["gk"].view(n, -1) * DK ** -0.5, c["gv"].view(n, -1), b["ggate"]], dim=1)
    d = binding.ttc_residual_norm_backward(y, grad_r=wx, grad_h=gh, **first)
    got = dict(y=d["gy"], x=d["gresidual"], gain=d["gpre_gain"], g=c["glog_decay"])

    Y, X, W, WX, G, GAIN = (host(t) for t in (y, x, w, wx, g, gain))
    _, h = oracle.residual_norm(Y, residual=X, pre="layer", pre_gain=GAIN)
    q, k, v, gate = split(h)
    o, _ = oracle.linear_attention(q, k, v, G, cu, DK ** -0.5)
    b = oracle.residual_norm(o.reshape(n, -1), gate=gate, gr=W, **last)
    gq, gk, gv, gg, _ = oracle.linear_attention_gradients(q, k, v, G, cu, DK ** -0.5, b["gy"].reshape(n, HEADS, DV))
    gh = np.concatenate([gq.reshape(n, -1), gk.reshape(n, -1) * DK ** -0.5, gv.reshape(n, -1), b["ggate"]], axis=1)
    d = oracle.residual_norm(Y, residual=X, pre="layer", pre_gain=GAIN, gr=WX, gh=gh)
    want = dict(y=d["gy"], x=d["gresidual"], gain=d["gpre_gain"], g=gg)
    for name, t in got.items():
        assert np.linalg.norm(host(t) - want[name]) <= 3e-4 * np.linalg.norm(want[name]) + 1e-30, name


@pytest.mark.parametrize("sequences,prompt,steps,heads", [(1, 1, 3, 1), (4, 300, 20, 4), (7, 259, 70, 2)])
def test_the_examples_layer(sequences, prompt, steps, heads, capsys):
    """Steps from a captured graph against the same tokens as one prompt: 2e-2 in the norm, as without the memory layer, whose results are rounded to
    bfloat16 like the others."""
    off = hybrid_layer.main(["--sequences", str(sequences), "--prompt", str(prompt), "--steps", str(steps), "--features", "256", "--memory", str(heads)])
    print(capsys.readouterr().out)
    assert off < 2e-2


def test_replays_of_the_examples_layer_equal_eager_steps():
    made = hybrid_layer.HybridLayer(256, longest=512, memory_heads=2)
    gen = torch.Generator(device=DEV).manual_seed(3)
    first = torch.randn((53, 256), generator=gen, device=DEV).bfloat16()
    a, b = (hybrid_layer.Sequences(made, 2, 512, page=16) for _ in range(2))
    assert torch.equal(hybrid_layer.prompt(made, a, first, [33, 20]), hybrid_layer.prompt(made, b, first, [33, 20]))
    step, one = hybrid_layer.Step(made, a, 256), torch.ones(2, dtype=torch.int32, device=DEV)
    for i in range(4):
        new = torch.randn((2, 256), generator=gen, device=DEV).bfloat16()
        got = step.replay(new).clone()
        at = b.grow(one, 2)
        want = made.forward(new, b.cache, at["slots"], at["positions"], b.pages, b.length, states=b.states)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(a.cache, b.cache) and torch.equal(a.length, b.length) and torch.equal(a.states, b.states)


def test_rows_beyond_what_32_bits_count():
    """Rows of one wide tensor, the last of them more than 2^32 entries behind the first, give the bits of the same rows side by side."""
    tokens, step, heads, d = 33000, 1 << 17, 2, 64
    wide = torch.empty((tokens, step), dtype=torch.bfloat16, device=DEV)
    gen = torch.Generator(device=DEV).manual_seed(1)
    near = torch.randn((tokens, 5 * heads * d), generator=gen, device=DEV).bfloat16()
    near[:, heads * d:2 * heads * d] *= d ** -0.5
    wide[:, :5 * heads * d] = near
    g = -torch.rand((tokens, heads), generator=gen, device=DEV)
    at = dict(cu_q=torch.tensor([0, 1, 900, tokens - 70, tokens], dtype=torch.int32, device=DEV), max_q=tokens)
    results = []
    for x in (near, wide):
        q, k, v, gout, gate = (x[:, i * heads * d:(i + 1) * heads * d] for i in range(5))
        by_heads = [t.unflatten(1, (heads, d)) for t in (q, k, v, gout)]
        place = torch.zeros_like(x[:, 5 * heads * d:6 * heads * d]) if x is near else wide[:, 5 * heads * d:6 * heads * d].zero_()
        got = binding.ttc_linear_attention(*by_heads[:3], g, out={"out": place.unflatten(1, (heads, d))} if x is wide else None, want_state=True, **at)
        back = binding.ttc_linear_attention_backward(*by_heads[:3], g, by_heads[3], **at)
        norm = binding.ttc_residual_norm(q, residual=k, gate=gate, post="rms", groups=heads, pre="layer", out={"r": place} if x is wide else None)
        grads = binding.ttc_residual_norm_backward(q, residual=k, gate=gate, post="rms", groups=heads, pre="layer", grad_h=v, grad_r=gout)
        results.append([got["state"]] + [norm["r"].clone(), norm["h"]] + list(back.values()) + list(grads.values()))
        if x is near:
            out = got["out"].clone()
        else:
            again = binding.ttc_linear_attention(*by_heads[:3], g, out={"out": place.unflatten(1, (heads, d))}, **at)["out"]
            assert torch.equal(again.flatten(1), out.flatten(1))
    for a, b in zip(*results):
        assert torch.equal(a, b)

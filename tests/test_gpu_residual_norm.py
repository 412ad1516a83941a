"""The norms, gate and residual scale around a block on the GPU (ttc_residual_norm and its gradients) against the float64 oracle.

Every result comes from a few sums over a row, of float32 numbers, and products and quotients of them.  A normed entry is (x - m) / s: where a
row's entries lie close together in relation to their mean, a difference is known to half a step of the mean.  Inputs are of size 1 with spread of
size 1, for which 64 half steps of the largest entry of a row bound all roundings of a forward result, and 64 of the largest product of gradient and
factors those of a gradient; sums over tokens add half a step a token of the sum of magnitudes."""
import numpy as np
import pytest
import torch

from oracle import memory_oracle as oracle
from paper_2603_09221_amd import binding
from tests.memory_inputs import DEV, HALF, U, host

pytestmark = pytest.mark.gpu
VECTORS = ("post_gain", "post_offset", "residual_gain", "pre_gain", "pre_offset")


def inputs(tokens, features, dtype, post, pre, gate, residual, vectors, seed=0):
    gen = torch.Generator().manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=gen)
    x = dict(y=(rand(tokens, features) + 0.3).to(dtype).to(DEV), gate=rand(tokens, features).to(dtype).to(DEV) if gate else None,
             residual=rand(tokens, features).to(dtype).to(DEV) if residual else None)
    for name in VECTORS:
        there = vectors and (not name.startswith("po") or post) and (not name.startswith("pr") or pre)
        x[name] = (rand(features) * 0.3 + (0.0 if "offset" in name else 1.0)).to(DEV) if there else None
    return x


def doubles(x):
    return {k: None if t is None else host(t) for k, t in x.items()}


def near(got, want, dtype, scale=None):
    """Row by row: 64 half steps of the row's largest number (of `scale`), half a step of the result's type."""
    largest = np.abs(want if scale is None else scale).max(-1, keepdims=True)
    bound = 64 * U * largest + HALF[dtype] * np.abs(want) * 1.01 + 1e-38
    off = np.abs(host(got) - want)
    assert (off <= bound).all(), float((off / bound).max())


CASES = [  # tokens, features, groups
    (1, 1, 1), (3, 7, 1), (5, 64, 1), (9, 100, 1), (4, 512, 1), (2, 513, 1), (6, 1024, 16), (5, 1500, 1), (3, 2048, 8), (2, 2056, 1), (3, 4096, 1), (2, 5000, 1),
    (2, 8192, 64), (1, 16384, 1), (3, 16384, 2), (300, 96, 1), (7, 960, 10), (5, 24, 3), (3, 1600, 5), (2, 6144, 2), (130, 320, 4)]


@pytest.mark.parametrize("tokens,features,groups", CASES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("post,pre,activation,residual,vectors", [("rms", "rms", "silu", True, True), ("layer", "layer", "sigmoid", True, False),
                                                                   ("layer", None, "identity", False, True), (None, "rms", None, True, True)])
def test_against_oracle(tokens, features, groups, dtype, post, pre, activation, residual, vectors):
    if post == "layer" and features // groups == 1 or pre == "layer" and features < 8:
        return      # the norm of one number is 0 whatever it is; of a few it can be a small difference over a smaller one
    x = inputs(tokens, features, dtype, post, pre, activation, residual, vectors, seed=features)
    kw = dict(activation=activation or "silu", post=post, pre=pre, scale=0.7, groups=groups)
    got = binding.ttc_residual_norm(**x, **kw)
    r, h = oracle.residual_norm(**doubles(x), **kw)
    near(got["r"], r, dtype)
    if pre:
        near(got["h"], h, dtype)
    else:
        assert got["h"] is None
    gen = torch.Generator().manual_seed(1)
    gr = torch.randn((tokens, features), generator=gen).to(dtype).to(DEV)
    gh = torch.randn((tokens, features), generator=gen).to(dtype).to(DEV) if pre else None
    got = binding.ttc_residual_norm_backward(grad_r=gr, grad_h=gh, **x, **kw)
    d = doubles(x)
    want = oracle.residual_norm(**d, **kw, gr=host(gr), gh=None if gh is None else host(gh))
    assert set(got) == {"g" + k for k, t in x.items() if t is not None}
    # sizes: gradients before their differences are taken
    unit_r = oracle._unit(r, pre, 1e-5, 1) if pre else None
    total = np.abs(host(gr)) + (np.abs(host(gh)) * np.abs(d["pre_gain"] if vectors else 1.0) * (1 + np.abs(unit_r[0])) * unit_r[1] if pre else 0.0)
    total = np.broadcast_to(total.max(-1, keepdims=True), total.shape)
    by = 0.7 * (np.abs(d["residual_gain"]) if vectors else np.ones(features))
    act, slope = oracle.act(d["gate"], kw["activation"]) if activation else (np.ones_like(d["y"]), None)
    unit, inverse = oracle._unit(d["y"], post, 1e-5, groups) if post else (d["y"], np.ones_like(d["y"]))
    z = unit * (d["post_gain"] if post and vectors else 1.0) + (d["post_offset"] if post and vectors else 0.0)
    gain = np.abs(d["post_gain"]) if post and vectors else np.ones(features)
    sizes = {"gresidual": total, "ggate": total * by * (1 + np.abs(z)) * (1 if slope is None else 1 + np.abs(slope)), "gy": total * by * np.abs(act).max() * gain * (1 + np.abs(unit).max()) ** 2 * inverse}
    for name in ("gy", "ggate", "gresidual"):
        if name in got:
            near(got[name], want[name], dtype, sizes[name])
    gz = total * by * np.abs(act)
    of = {"gpost_gain": gz * (1 + np.abs(unit)), "gpost_offset": gz, "gresidual_gain": 0.7 * total * np.abs(act) * (1 + np.abs(z))}
    if pre:
        of.update(gpre_gain=np.abs(host(gh)) * (1 + np.abs(unit_r[0])), gpre_offset=np.abs(host(gh)))
    for name, size in of.items():
        if name in got:
            off = np.abs(host(got[name]) - want[name])
            assert (off <= (64 + tokens) * U * size.sum(0) + 1e-38).all(), name


@pytest.mark.parametrize("features", [4096, 5000, 8192, 16384])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_many_wide_rows(features, dtype):
    """Several rows to a workgroup; and gains without offsets, which are those with offsets of 0: an addition of 0 rounds nothing, so that only the
    order of roundings could differ (64 half steps, as against the oracle)."""
    test_against_oracle(530, features, 1, dtype, "rms", "rms", "silu", True, True)
    x = inputs(530, features, dtype, "rms", "layer", True, True, True, seed=2)
    gen = torch.Generator().manual_seed(3)
    gr, gh = (torch.randn((530, features), generator=gen).to(dtype).to(DEV) for _ in range(2))
    kw = dict(post="rms", pre="layer", grad_r=gr, grad_h=gh)
    zeros = {**x, "post_offset": torch.zeros_like(x["post_gain"]), "pre_offset": torch.zeros_like(x["post_gain"])}
    want = binding.ttc_residual_norm_backward(**zeros, **kw)
    got = binding.ttc_residual_norm_backward(**{**x, "post_offset": None, "pre_offset": None}, **kw)
    assert set(want) - set(got) == {"gpost_offset", "gpre_offset"}
    for name in ("gy", "ggate", "gresidual"):
        near(got[name], host(want[name]), dtype, np.abs(host(gr)) + 8 * np.abs(host(gh)))
    for name in ("gpost_gain", "gresidual_gain", "gpre_gain"):
        off, size = np.abs(host(got[name]) - host(want[name])), 530 * 8 * (np.abs(host(gr)).max() + 8 * np.abs(host(gh)).max())
        assert (off <= 64 * U * size).all(), name


def test_parts_and_no_parts():
    """Only h, only r, nothing but a copy; gradients with grad_r left out."""
    x = inputs(5, 256, torch.float32, "rms", "rms", True, True, True)
    kw = dict(post="rms", pre="rms", scale=1.3)
    both = binding.ttc_residual_norm(**x, **kw)
    y = x["y"]
    assert torch.equal(binding.ttc_residual_norm(y)["r"], y)
    plain = binding.ttc_residual_norm(y, pre="layer")
    assert torch.equal(plain["r"], y)
    near(plain["h"], oracle.residual_norm(host(y), pre="layer")[1], torch.float32)
    g = torch.randn_like(y)
    zero = torch.zeros_like(y)
    one = binding.ttc_residual_norm_backward(grad_h=g, **x, **kw)
    two = binding.ttc_residual_norm_backward(grad_h=g, grad_r=zero, **x, **kw)
    for name in one:
        assert torch.equal(one[name], two[name]), name
    assert torch.equal(binding.ttc_residual_norm_backward(y, grad_r=g)["gy"], g)
    # r in place of the residual, h in place of the gate
    r, h = x["residual"].clone(), x["gate"].clone()
    binding.ttc_residual_norm(**{**x, "residual": r, "gate": h}, **kw, out={"r": r, "h": h})
    assert torch.equal(r, both["r"]) and torch.equal(h, both["h"])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("features", [96, 1000, 3000])
def test_strides_alignment_and_a_gate_for_all(dtype, features):
    x = inputs(6, features, dtype, "layer", "rms", True, True, True, seed=2)
    kw = dict(post="layer", pre="rms", scale=0.5)
    want = binding.ttc_residual_norm(**x, **kw)
    g = torch.randn((2, 6, features), device=DEV).to(dtype)
    back = binding.ttc_residual_norm_backward(grad_r=g[0], grad_h=g[1], **x, **kw)
    for shift in (0, 1, 3):
        room = {k: torch.full((6, features + 9), 7.0, dtype=dtype, device=DEV) for k in ("y", "gate", "residual", "r", "h", "gr", "gh")}
        view = {k: t[:, shift:shift + features] for k, t in room.items()}
        for k in ("y", "gate", "residual"):
            view[k].copy_(x[k])
        view["gr"].copy_(g[0]), view["gh"].copy_(g[1])
        moved = {**x, **{k: view[k] for k in ("y", "gate", "residual")}}
        got = binding.ttc_residual_norm(**moved, **kw, out={"r": view["r"], "h": view["h"]})
        assert torch.equal(got["r"], want["r"]) and torch.equal(got["h"], want["h"])
        for k in ("r", "h"):
            assert (room[k][:, :shift] == 7).all() and (room[k][:, shift + features:] == 7).all()
        again = binding.ttc_residual_norm_backward(grad_r=view["gr"], grad_h=view["gh"], **moved, **kw)
        for name in back:
            assert torch.equal(again[name], back[name]), name
    one = x["gate"][:1].expand(6, -1)
    spread = {**x, "gate": one.contiguous()}
    a, b = (binding.ttc_residual_norm(**{**x, "gate": t}, **kw) for t in (one, spread["gate"]))
    assert torch.equal(a["r"], b["r"]) and torch.equal(a["h"], b["h"])
    a, b = (binding.ttc_residual_norm_backward(grad_r=g[0], grad_h=g[1], **{**x, "gate": t}, **kw) for t in (one, spread["gate"]))
    for name in a:
        assert torch.equal(a[name], b[name]), name


def test_far_gates_zero_rows_and_nan():
    y = torch.randn((6, 128), device=DEV)
    y[1] = 0.0
    gate = torch.tensor([0.0, 100.0, -100.0, float("inf"), -float("inf"), 1.0], device=DEV)[:, None].expand(6, 128).contiguous()
    for activation, limit in (("silu", [0.0, 100.0, 0.0, float("inf"), 0.0]), ("sigmoid", [0.5, 1.0, 0.0, 1.0, 0.0])):
        one = torch.ones_like(y)
        r = binding.ttc_residual_norm(one, gate=gate, activation=activation)["r"]
        assert torch.allclose(r[:5, 0], torch.tensor(limit, device=DEV), rtol=4 * U, atol=1e-30)
        g = binding.ttc_residual_norm_backward(one, grad_r=one, gate=gate, activation=activation)["ggate"]
        assert torch.allclose(g[:5, 0], torch.tensor([0.5, 1, 0, 1, 0] if activation == "silu" else [0.25, 0, 0, 0, 0], device=DEV), rtol=4 * U, atol=1e-30)
    for kind in ("rms", "layer"):
        h = binding.ttc_residual_norm(y, pre=kind)["h"]
        assert not h[1].any() and torch.isfinite(h).all()
        assert torch.isfinite(binding.ttc_residual_norm_backward(y, grad_h=y, pre=kind)["gy"]).all()
    y[3, 5] = float("nan")      # its own row alone
    for features in (128, 64):
        got = binding.ttc_residual_norm(y[:, :features], post="rms", pre="layer")
        assert torch.isnan(got["h"][3]).all() and torch.isfinite(got["h"][[0, 1, 2, 4, 5]]).all()


def test_against_differences():
    """Central differences of the float32 forward pass: curvature h^2 / 6 times a third derivative of size 10 at most here, and roundings of the loss over h."""
    x = inputs(2, 32, torch.float32, "layer", "rms", True, True, True, seed=3)
    kw = dict(post="layer", pre="rms", scale=0.7, groups=2, activation="sigmoid")
    gr, gh = torch.randn((2, 2, 32), device=DEV).unbind(0)
    got = binding.ttc_residual_norm_backward(grad_r=gr, grad_h=gh, **x, **kw)

    def loss():
        y = binding.ttc_residual_norm(**x, **kw)
        return float((y["r"].double() * gr.double()).sum() + (y["h"].double() * gh.double()).sum())

    h = 2.0 ** -6
    for name, t in x.items():
        for at in ([0, 3], [1, 31]):
            i = tuple(at[-t.dim():])
            keep = float(t[i])
            t[i] = keep + h
            up, above = loss(), float(t[i])
            t[i] = keep - h
            down, below = loss(), float(t[i])
            t[i] = keep
            assert abs((up - down) / (above - below) - float(got["g" + name][i])) <= 64 * 10 * h * h / 6 + 128 * 16 * U / h, name


def test_many_tokens_streams_and_replays():
    """More rows than one turn of the workgroups; another stream; a captured call replayed with other work between."""
    x = inputs(5000, 72, torch.bfloat16, "rms", "rms", True, True, True, seed=4)
    kw = dict(post="rms", pre="rms")
    g = torch.randn((2, 5000, 72), device=DEV).bfloat16()
    call = lambda **more: binding.ttc_residual_norm_backward(grad_r=g[0], grad_h=g[1], **x, **kw, **more)
    want = call()
    doubled = oracle.residual_norm(**doubles(x), **kw, gr=host(g[0]), gh=host(g[1]))
    for name in ("gpost_gain", "gresidual_gain", "gpre_gain"):
        off = host(want[name]) - doubled[name]
        assert np.linalg.norm(off) <= 32 * U * np.linalg.norm(doubled[name]), name
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    other = call(stream=stream)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
        forward = binding.ttc_residual_norm(**x, **kw)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        eager = binding.ttc_residual_norm(**x, **kw)
        for name in want:
            assert torch.equal(out[name], want[name]) and torch.equal(other[name], want[name])
        assert torch.equal(forward["r"], eager["r"]) and torch.equal(forward["h"], eager["h"])


def test_no_tokens():
    x = inputs(0, 64, torch.float32, "rms", "rms", True, True, True)
    got = binding.ttc_residual_norm(**x, post="rms", pre="rms")
    assert got["r"].shape == (0, 64) and got["h"].shape == (0, 64)
    got = binding.ttc_residual_norm_backward(grad_h=x["y"], **x, post="rms", pre="rms")
    for name in VECTORS:
        assert got["g" + name].shape == (64,) and not got["g" + name].any()

"""Rotary positions on the GPU (ttc_rope, ttc_rope_backward, ttc_rope_table) against the float64 oracle.  An entry is two products and a
sum, each rounded to float32: at most 2^-23 (|a c| + |b s|) off for the two roundings that it passes, half a step of its type more where
that is bfloat16 (of 8 significant bits: 2^-8 of it at most)."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as oracle
from paper_2603_09221_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def host(t):
    return t.detach().cpu().double().numpy()


def table_of(rows, rot, **kw):
    freqs, scale = binding.rope_frequencies(rot, **kw)
    return binding.ttc_rope_table(rows, freqs, scale=scale, device=DEV), freqs.numpy(), scale


def bound(x, positions, table, layout, bf16):
    """How far an entry may be off: the same rotation of magnitudes by magnitudes."""
    mags = np.abs(table) * np.array([1.0, -1.0])    # cos a - (-sin) b: everything adds up
    size = np.abs(oracle.rope(np.abs(x), positions, mags, layout)) + np.abs(oracle.rope(np.abs(x), positions, np.abs(table), layout))
    return size * (2.0 ** -23 + (2.0 ** -8 if bf16 else 0.0)) + 1e-45


SHAPES = [(1, 1, 64, 64), (1, 32, 128, 128), (37, 5, 128, 64), (300, 3, 80, 80), (65, 2, 96, 24), (5, 7, 2, 2), (9, 3, 7, 4), (33, 4, 256, 256),
          (16, 2, 64, 0), (700, 40, 128, 128), (12, 3, 20, 10)]


@pytest.mark.parametrize("tokens,heads,d,rot", SHAPES)
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_against_oracle_and_back(tokens, heads, d, rot, layout, dtype):
    gen = torch.Generator(device=DEV).manual_seed(tokens + heads + d + rot)
    x = torch.randn((tokens, heads, d), generator=gen, device=DEV).to(dtype)
    pos = torch.randint(0, 500, (tokens,), generator=gen, device=DEV)
    table = table_of(500, rot)[0] if rot else torch.empty((500, 0, 2), device=DEV)
    few = min(tokens, 40)       # (the oracle turns pair by pair)
    y, back = binding.ttc_rope(x, pos, table, layout=layout), binding.ttc_rope_backward(x, pos, table, layout=layout)
    for got, backward in ((y, False), (back, True)):
        want = oracle.rope(host(x[:few]), host(pos[:few]).astype(int), host(table), layout, backward)
        off = np.abs(host(got[:few]) - want)
        assert (off <= bound(host(x[:few]), host(pos[:few]).astype(int), host(table), layout, dtype == torch.bfloat16)).all(), off.max()
    # all tokens: turning back gives the tokens again (two rotations' roundings, of lengths that a rotation keeps)
    again = binding.ttc_rope_backward(y, pos, table, layout=layout)
    size = x.float().abs().amax() * 2
    assert float((again.float() - x.float()).abs().max()) <= float(size) * (2.0 ** -21 if dtype == torch.float32 else 2.0 ** -7)
    assert torch.equal(y[..., rot:], x[..., rot:])


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides_alignment_and_in_place_give_the_same_bits(layout, dtype):
    gen = torch.Generator(device=DEV).manual_seed(3)
    fused = torch.randn((50, 12 * 64 + 3), generator=gen, device=DEV).to(dtype)
    pos = torch.randint(0, 99, (50,), generator=gen, device=DEV)
    table = table_of(99, 32)[0]
    for first in (0, 1, 3):     # rows that begin anywhere
        x = fused[:, first:first + 640].unflatten(1, (10, 64))
        want = binding.ttc_rope(x.contiguous(), pos, table, layout=layout)
        assert torch.equal(binding.ttc_rope(x, pos, table, layout=layout), want)
        across = torch.randn((10, 50, 64), generator=gen, device=DEV).to(dtype)
        out = across.transpose(0, 1)
        binding.ttc_rope(x, pos, table, layout=layout, out=out)
        assert torch.equal(out, want)
        copy = fused.clone()
        view = copy[:, first:first + 640].unflatten(1, (10, 64))
        binding.ttc_rope(view, pos, table, layout=layout, out=view)
        assert torch.equal(view, want)
        assert torch.equal(copy[:, :first], fused[:, :first]) and torch.equal(copy[:, first + 640:], fused[:, first + 640:])
    uneven = torch.empty(table.numel() + 2, device=DEV)[2:].view(table.shape)     # a table that is 8-byte aligned only
    uneven.copy_(table)
    x = fused[:, :640].unflatten(1, (10, 64)).contiguous()
    assert torch.equal(binding.ttc_rope(x, pos, uneven, layout=layout), binding.ttc_rope(x, pos, table, layout=layout))


def test_positions_outside_the_table_give_nan_in_the_rotated_entries():
    x = torch.randn((4, 2, 64), device=DEV)
    table = table_of(10, 32)[0]
    y = binding.ttc_rope(x, torch.tensor([0, -1, 10, 9], device=DEV), table)
    assert torch.isnan(y[1:3, :, :32]).all() and torch.equal(y[..., 32:], x[..., 32:])
    assert torch.equal(y[0], x[0]) and not torch.isnan(y[3]).any()


@pytest.mark.parametrize("kw", [{}, dict(scaling="linear", factor=4.0), dict(scaling="base", factor=8.0),
                                dict(scaling="bands", factor=4.0, trained=4096)])
def test_table(kw):
    """Angles in float64: an entry is rounded once (2^-25 of the scale at most), and cos, sin of an angle of 10^6 are some 1e-10 off."""
    rows = 1 << 20
    table, freqs, scale = table_of(rows, 32, **kw)
    some = np.concatenate([np.arange(50), np.random.default_rng(1).integers(0, rows, 500), [rows - 1]])
    angle = some[:, None] * freqs
    want = scale * np.stack([np.cos(angle), np.sin(angle)], -1)
    assert np.abs(host(table[torch.from_numpy(some).to(DEV)]) - want).max() <= scale * 2.0 ** -24


def test_gradient_against_differences():
    """dl/dx of l = sum of g times the rotated x, by central differences of the float32 forward pass: it is linear, so a step of 1
    leaves only roundings, each below 2^-23 of the largest entry times two, in a sum of 2 entries."""
    gen = torch.Generator(device=DEV).manual_seed(9)
    x, g = torch.randn((2, 3, 2, 12), generator=gen, device=DEV).unbind(0)
    pos, table = torch.tensor([3, 77, 12], device=DEV), table_of(100, 8)[0]
    grad = host(binding.ttc_rope_backward(g, pos, table))
    for i in np.ndindex(3, 2, 12):
        step = torch.zeros_like(x)
        step[i] = 1.0
        up, down = (host(binding.ttc_rope(x + s * step, pos, table)) for s in (1, -1))
        assert abs(((up - down) * host(g)).sum() / 2 - grad[i]) <= 40 * 2.0 ** -23


def test_another_stream_and_no_tokens():
    x = torch.randn((64, 4, 64), device=DEV)
    pos, table = torch.arange(64, device=DEV), table_of(64, 64)[0]
    want = binding.ttc_rope(x, pos, table)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    got = binding.ttc_rope(x, pos, table, stream=stream)
    stream.synchronize()
    assert torch.equal(got, want)
    assert binding.ttc_rope(x[:0], pos[:0], table).shape == (0, 4, 64)

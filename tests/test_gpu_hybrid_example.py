"""The example of a served layer: single tokens replayed from a captured graph against the same tokens as one prompt.  The two differ in the
rounding of their projections and weights to bfloat16 (8 significant bits, 2^-8 each), some of which a key's code or a block's exponent answers to
with a step of its own: 2e-2 in the norm of a layer's output."""
import pytest
import torch

from examples import hybrid_layer
from paper_2603_09221_amd import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sequences,prompt,steps", [(1, 1, 3), (4, 300, 20), (7, 259, 70)])
def test_steps_against_one_prompt(sequences, prompt, steps, capsys):
    off = hybrid_layer.main(["--sequences", str(sequences), "--prompt", str(prompt), "--steps", str(steps), "--features", "256"])
    print(capsys.readouterr().out)
    assert off < 2e-2


def test_replays_equal_eager_steps():
    """Every replay, with other work between, gives the bits of the same call made eagerly on a cache of its own."""
    layer = hybrid_layer.HybridLayer(256, longest=512)
    gen = torch.Generator(device="cuda:0").manual_seed(3)
    x = torch.randn((2, 40, 256), generator=gen, device="cuda:0").bfloat16()
    lengths, features = [33, 20], 256
    a, b = (hybrid_layer.Sequences(layer, 2, 512, page=16) for _ in range(2))
    first = torch.cat([x[0, :33], x[1, :20]])
    assert torch.equal(hybrid_layer.prompt(layer, a, first, lengths), hybrid_layer.prompt(layer, b, first, lengths))
    step = hybrid_layer.Step(layer, a, features)
    each = torch.arange(2, device="cuda:0")
    for i in range(5):
        new = torch.randn((2, features), generator=gen, device="cuda:0").bfloat16()
        got = step.replay(new).clone()
        position = b.length.long()
        b.length += 1
        want = layer.forward(new, b.cache, b.place(each, position), position, b.pages, b.length)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(a.cache, b.cache) and torch.equal(a.length, b.length)


def test_training_reads_the_same_positions():
    """The rotation that serving has inside its append is ttc_rope's, whose gradient autograd can be given."""
    class Rope(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, positions, table):
            ctx.save_for_backward(positions, table)
            return binding.ttc_rope(x, positions, table)

        @staticmethod
        def backward(ctx, grad):
            return binding.ttc_rope_backward(grad, *ctx.saved_tensors), None, None

    layer = hybrid_layer.HybridLayer(256, longest=64)
    x = torch.randn((9, 2, 128), device="cuda:0", requires_grad=True)
    positions = torch.arange(9, device="cuda:0") * 7
    w = torch.randn((9, 2, 128), device="cuda:0")
    y = Rope.apply(x, positions, layer.table)
    (y * w).sum().backward()
    # the transpose: <w, R x> = <R^T w, x>, of 2304 products of about 1, each side of them rounded to 2^-22 of the largest
    left, right = float((y.detach().double() * w.double()).sum()), float((x.grad.double() * x.detach().double()).sum())
    assert abs(left - right) <= 2304 * 16 * 2.0 ** -22

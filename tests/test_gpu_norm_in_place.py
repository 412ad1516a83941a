"""Gradients of the norms around a block written over what they come from: the bits of results of their own."""
import pytest
import torch

from paper_2603_09221_amd import binding
from tests.memory_inputs import DEV
from tests.test_gpu_residual_norm import inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,features", [(700, 96), (1300, 1000), (600, 3000), (530, 5000), (300, 16384)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("post,pre", [("rms", "layer"), (None, None)])
def test_gradients_in_place(tokens, features, dtype, post, pre):
    """More rows than workgroups, so that one has its next row under way while it writes."""
    x = inputs(tokens, features, dtype, post, pre, True, True, True, seed=features)
    gen = torch.Generator().manual_seed(3)
    gr, gh = (torch.randn((tokens, features), generator=gen).to(dtype).to(DEV) for _ in range(2))
    kw = dict(post=post, pre=pre)
    if pre is None:
        gh = None
    want = binding.ttc_residual_norm_backward(**x, grad_r=gr, grad_h=gh, **kw)
    rows = {"y": x["y"], "gate": x["gate"], "residual": x["residual"], "grad_r": gr, "grad_h": gh}
    for places in (("y", "gate", "residual"), ("grad_r", "residual", "y"), ("gate", "y", "grad_r"), ("residual", "grad_h" if pre else "y", "gate")):
        own = {name: None if t is None else t.clone() for name, t in rows.items()}
        out = {result: own[place] for result, place in zip(("gy", "ggate", "gresidual"), places)}
        got = binding.ttc_residual_norm_backward(**{**x, **own}, **kw, out=out)
        for name in want:
            assert torch.equal(got[name], want[name]), (places, name)
        assert all(got[result] is own[place] for result, place in zip(("gy", "ggate", "gresidual"), places))

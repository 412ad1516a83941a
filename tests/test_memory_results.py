"""Tensors in `out` that a call of the memory layers, the norms or the places would hand back unwritten: refused, before anything else of the GPU's."""
import pytest
import torch

from paper_2603_09221_amd import binding
from tests.test_memory_boundary import i32, linear_args, place_call


@pytest.mark.parametrize("call", [
    lambda: binding.ttc_residual_norm(torch.zeros(3, 64), out={"h": torch.zeros(3, 64)}),
    lambda: binding.ttc_residual_norm(torch.zeros(3, 64), pre="rms", out={"r": torch.zeros(3, 64), "z": torch.zeros(3, 64)}),
    lambda: binding.ttc_residual_norm_backward(torch.zeros(3, 64), grad_r=torch.zeros(3, 64), out={"ggate": torch.zeros(3, 64)}),
    lambda: binding.ttc_residual_norm_backward(torch.zeros(3, 64), grad_r=torch.zeros(3, 64), post="rms", out={"gpost_gain": torch.zeros(64)}),
    lambda: binding.ttc_linear_attention(**linear_args(), out={"lse": torch.zeros(6, 4)}),
    lambda: binding.ttc_linear_attention_backward(**linear_args(), grad_out=torch.zeros(6, 4, 32), out={"gstate": torch.zeros(2, 4, 64, 32)}),
    lambda: place_call(free=None, free_count=None, out={"free_count": i32(1)}),
    lambda: place_call(free=None, free_count=None, out={"missing": i32(1)})])
def test_results_that_the_call_does_not_have(call):
    with pytest.raises(ValueError, match="has no result"):
        call()


@pytest.mark.parametrize("call", [
    lambda: binding.ttc_residual_norm(torch.zeros(3, 64), out={"r": torch.zeros(3, 64), "h": None}),
    lambda: binding.ttc_linear_attention(**linear_args(), out={"out": None, "state": None}),
    lambda: place_call(free=None, free_count=None, out={"missing": None, "slots": None})])
def test_names_without_tensors_are_none(call):
    """What a call gave back is taken as the next one's `out`."""
    with pytest.raises(ValueError, match="on a GPU"):
        call()

"""What the Python entry points of positions, cache and attention refuse before a launch, beyond test_attention_boundary.  No GPU."""
import pytest
import torch

from paper_2603_09221_amd import binding


def call(**change):
    q, cache = torch.zeros(3, 8, 128), torch.zeros(4, 2, 64 * 136, dtype=torch.uint8)
    a = dict(q=q, cache=cache, block_table=torch.zeros(3, 4, dtype=torch.int32), kv_len=torch.zeros(3, dtype=torch.int32))
    return binding.ttc_attention(**{**a, **change})


def test_host_memory_is_not_handed_to_a_kernel():
    """Arguments that fit, but lie on the host."""
    k, cache, slots = torch.zeros(3, 2, 128), torch.zeros(4, 2, 64 * 136, dtype=torch.uint8), torch.zeros(3, dtype=torch.int64)
    table = torch.zeros(8, 64, 2)
    for refused in (lambda: call(), lambda: binding.ttc_kv_append(cache, k, k, slots), lambda: binding.ttc_kv_append(cache, k, k, slots, slots, table, q=k),
                    lambda: binding.ttc_kv_read(cache, slots, 128), lambda: binding.ttc_rope(k, slots, table),
                    lambda: binding.ttc_rope_backward(k, slots, table, out=k), lambda: binding.ttc_rope_table(8, torch.ones(4), device="cpu")):
        with pytest.raises(ValueError, match="on a GPU"):
            refused()


def test_numbers_that_a_descriptor_would_cut_off():
    """2^32 + 5 is not 5."""
    cu = torch.zeros(4, dtype=torch.int32)
    wide = torch.empty((3, 1 << 25), dtype=torch.int32)     # room for 2^31 tokens (never touched)
    for change in (dict(window=(1 << 32) + 5), dict(window=1 << 31), dict(cu_q=cu, max_q=(1 << 32) + 1), dict(block_table=wide, max_kv=1 << 31)):
        with pytest.raises(ValueError, match="32 bits"):
            call(**change)

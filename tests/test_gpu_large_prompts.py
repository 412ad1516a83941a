"""Positions and the cache on the GPU at the sizes where a thread takes several heads or tokens, and where results are written past the caches: against
the float64 oracle, and against the same call in small pieces, whose threads take one each."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as oracle
from paper_2603_09221_amd import binding
from tests.test_gpu_kv_cache import check_bytes, host, some_slots, some_tokens

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
N = 4099


def compute_units():
    return torch.cuda.get_device_properties(0).multi_processor_count


@pytest.mark.parametrize("heads_q,heads,d,rot,page", [(6, 1, 128, 128, 64), (6, 5, 64, 64, 16), (10, 2, 256, 256, 32), (10, 5, 128, 40, 256), (9, 4, 64, 24, 32)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_append_of_many_tokens(heads_q, heads, d, rot, page, layout, dtype):
    # two workgroups of four entries a thread to each compute unit: from here on a thread takes four heads, or tokens
    assert N * (heads_q + 2 * heads) * (d // 8) >= 2 * 256 * 4 * compute_units()
    pages = N // page + 5
    k, v = some_tokens(N, heads, d, dtype, d + rot, spread=0.5)
    q = some_tokens(N, heads_q, d, dtype, 7)[0]
    gen = torch.Generator(device=DEV).manual_seed(2)
    pos = torch.randint(0, 4000, (N,), generator=gen, device=DEV)
    pos[5], pos[N - 1] = -3, 4000
    table = binding.ttc_rope_table(4000, binding.rope_frequencies(rot)[0], device=DEV)
    slots = some_slots(N, pages, page, 1)
    slots[::11], slots[N - 2] = -1, pages * page
    before = torch.randint(0, 256, (pages, heads, binding.ttc_kv_page_bytes(d, page)), generator=gen, device=DEV, dtype=torch.uint8)
    cache = before.clone()
    got = binding.ttc_kv_append(cache, k, v, slots, pos, table, layout=layout, q=q)
    want = binding.ttc_rope(q, pos, table, layout=layout)
    assert torch.equal(got.nan_to_num(123.0), want.nan_to_num(123.0))
    check_bytes(cache, before, d, host(binding.ttc_rope(k.float(), pos, table, layout=layout)), host(v), slots)
    # in small pieces: a NaN block's codes, which stand for nothing, included
    pieces, part = before.clone(), torch.empty_like(q)
    for at in range(0, N, 500):
        to = slice(at, at + 500)
        assert 500 * (heads_q + 2 * heads) * (d // 8) < 2 * 256 * 4 * compute_units()
        part[to] = binding.ttc_kv_append(pieces, k[to], v[to], slots[to], pos[to], table, layout=layout, q=q[to])
    assert torch.equal(pieces, cache) and torch.equal(part.nan_to_num(123.0), got.nan_to_num(123.0))
    # rows that begin anywhere, queries in place
    wide = torch.zeros((N, (heads_q + 2 * heads) * d + 1), device=DEV, dtype=dtype)
    rows = wide[:, 1:].unflatten(1, (heads_q + 2 * heads, d))
    rows[:, :heads_q], rows[:, heads_q:-heads], rows[:, -heads:] = q, k, v
    other = before.clone()
    binding.ttc_kv_append(other, rows[:, heads_q:-heads], rows[:, -heads:], slots, pos, table, layout=layout, q=rows[:, :heads_q], q_out=rows[:, :heads_q])
    assert torch.equal(other, cache) and torch.equal(rows[:, :heads_q].nan_to_num(123.0), got.nan_to_num(123.0))
    assert torch.equal(rows[:, -heads:], v) and not wide[:, 0].any()
    # queries in place on rows that allow wide accesses
    same = q.clone()
    other = before.clone()
    binding.ttc_kv_append(other, k, v, slots, pos, table, layout=layout, q=same, q_out=same)
    assert torch.equal(other, cache) and torch.equal(same.nan_to_num(123.0), got.nan_to_num(123.0))


@pytest.mark.parametrize("d,page", [(64, 16), (128, 64), (256, 128)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_read_of_many_tokens(d, page, dtype):
    """Results of more than 16 MiB: every code and every exponent, NaN's among them."""
    heads = 2048 // d
    pages = N // page + 3
    gen = torch.Generator(device=DEV).manual_seed(d)
    cache = torch.randint(0, 256, (pages, heads, binding.ttc_kv_page_bytes(d, page)), generator=gen, device=DEV, dtype=torch.uint8)
    slots = some_slots(N, pages, page, 3)
    slots[::9], slots[N - 1] = -1, pages * page
    got = binding.ttc_kv_read(cache, slots, d, dtype=dtype)
    assert sum(t.numel() * t.element_size() for t in got) >= 16 << 20
    real = ((slots >= 0) & (slots < pages * page)).cpu().numpy()
    for g, w in zip(got, oracle.tokens(cache.cpu().numpy(), d)):
        want = np.zeros(g.shape)
        want[real] = w[slots.cpu().numpy()[real]]
        np.testing.assert_array_equal(host(g), want)
    for at in range(0, N, 300):
        piece = binding.ttc_kv_read(cache, slots[at:at + 300], d, dtype=dtype)
        for g, w in zip(got, piece):
            assert torch.equal(g[at:at + 300].nan_to_num(123.0), w.nan_to_num(123.0))


@pytest.mark.parametrize("heads,d,rot", [(18, 128, 128), (7, 256, 128), (41, 64, 64), (18, 128, 48)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rotation_of_many_tokens(heads, d, rot, layout, dtype):
    tokens, vec = 4 * N, 8 if dtype == torch.bfloat16 else 4
    units = rot // 2 // vec + (d - rot) // vec if layout == "half" else d // vec    # pieces of a head that a thread owns
    assert tokens * units * -(-heads // 4) >= 256 * compute_units() > 64 * units * -(-heads // 4)
    gen = torch.Generator(device=DEV).manual_seed(heads)
    x = torch.randn((tokens, heads, d), generator=gen, device=DEV).to(dtype)
    pos = torch.randint(0, 500, (tokens,), generator=gen, device=DEV)
    pos[7] = 500
    table = binding.ttc_rope_table(500, binding.rope_frequencies(rot)[0], device=DEV)
    for call, backward in ((binding.ttc_rope, False), (binding.ttc_rope_backward, True)):
        got = call(x, pos, table, layout=layout)
        for at in (0, 64, 5000, tokens - 61):
            to = slice(at, at + 64)
            assert torch.equal(got[to].nan_to_num(123.0), call(x[to].contiguous(), pos[to], table, layout=layout).nan_to_num(123.0))
        few = slice(tokens - 12, tokens)
        want = oracle.rope(host(x[few]), host(pos[few]).astype(int), host(table), layout, backward)
        size = 2 * np.abs(host(x[few])).max()
        # two roundings to float32 of products of at most `size`, one to bfloat16
        assert np.abs(host(got[few]) - want).max() <= size * (2.0 ** -23 + (2.0 ** -8 if dtype == torch.bfloat16 else 0.0))
        same = x.clone()
        call(same, pos, table, layout=layout, out=same)
        assert torch.equal(same.nan_to_num(123.0), got.nan_to_num(123.0))

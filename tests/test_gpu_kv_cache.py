"""The cache of 4-bit codes on the GPU (ttc_kv_append, ttc_kv_read) against the float64 oracle.  Without positions the bytes are the
oracle's; with them the rotated key is the float32 numbers that ttc_rope gives, quantised like any others."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as oracle
from paper_2603_09221_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NUMPY = {torch.float32: np.float64, torch.bfloat16: np.float64}


def host(t):
    return t.detach().cpu().double().numpy()


def some_tokens(tokens, heads, d, dtype, seed, spread=1.0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn((2, tokens, heads, d), generator=gen, device=DEV)
    x *= torch.exp(spread * torch.randn((2, tokens, heads, 1), generator=gen, device=DEV))
    return x.to(dtype).unbind(0)


def some_slots(tokens, pages, page, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randperm(pages * page, generator=gen, device=DEV)[:tokens]


def check_bytes(cache, before, d, k, v, slots):
    """The whole cache: the tokens' codes and exponents, and every other byte as it was."""
    got, old = oracle.parts(cache.cpu().numpy(), d), oracle.parts(before.cpu().numpy(), d)
    page = got[0].shape[2]
    slots = slots.cpu().numpy()
    real = (slots >= 0) & (slots < got[0].shape[0] * page)
    want = [p.copy() for p in old]
    for i, x in ((0, k), (1, v)):
        codes, e = oracle.quantise(x[real])
        full = e == 255
        want[i][slots[real] // page, :, slots[real] % page] = codes
        want[i + 2][slots[real] // page, :, slots[real] % page] = e
        for g in (got, want):       # a NaN block's codes stand for nothing
            t = g[i][slots[real] // page, :, slots[real] % page]
            g[i][slots[real] // page, :, slots[real] % page] = np.where(np.repeat(full, 32, -1), 0, t)
    for g, w, name in zip(got, want, ("keys", "values", "keys' exponents", "values' exponents")):
        np.testing.assert_array_equal(g, w, err_msg=name)


@pytest.mark.parametrize("tokens,heads,d,page", [(1, 1, 64, 16), (1, 8, 128, 64), (33, 3, 128, 16), (77, 5, 64, 32), (100, 2, 256, 128), (513, 2, 128, 256),
                                                 (31, 1, 256, 16)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_bytes_without_positions(tokens, heads, d, page, dtype):
    pages = tokens // page + 3
    k, v = some_tokens(tokens, heads, d, dtype, tokens + d)
    slots = some_slots(tokens, pages, page, tokens)
    slots[::7] = -1
    if tokens > 8:
        slots[3] = pages * page     # one past the cache
    cache = torch.randint(0, 256, (pages, heads, binding.ttc_kv_page_bytes(d, page)), device=DEV, dtype=torch.uint8)
    before = cache.clone()
    assert binding.ttc_kv_append(cache, k, v, slots) is None
    check_bytes(cache, before, d, host(k), host(v), slots)
    for out_dtype in (torch.float32, torch.bfloat16):
        rk, rv = binding.ttc_kv_read(cache, slots, d, dtype=out_dtype)
        for got, x in ((rk, k), (rv, v)):
            want = oracle.numbers(*oracle.quantise(host(x)))
            want[((slots < 0) | (slots >= pages * page)).cpu().numpy()] = 0.0
            np.testing.assert_array_equal(host(got), want)


def test_rounding_at_ties_and_at_the_ends_of_the_range():
    """Every tie of two codes with both signs, blocks of zeros, of denormal numbers, of the largest ones, of NaN and infinity."""
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.0, -0.0])
    row = np.zeros((12, 64), np.float32)
    row[0, :9], row[0, 31], row[0, 32:41], row[0, 63] = ties, 6.0, -ties, -4.0
    row[1, 0], row[1, 32] = 7.0, 6.9999995
    row[2, 5] = 1e-45
    row[3, :5], row[3, 40] = np.arange(5) * 1e-40, 1.1754944e-38
    row[4, 1], row[4, 33] = 3.4028235e38, 3.0e38
    row[5, 2], row[5, 40] = np.nan, -np.inf
    row[6, 2], row[6, 3] = np.inf, 1.0
    row[7] = np.linspace(-6, 6, 64)
    row[8] = np.float32(2.0) ** np.linspace(-140, 120, 64).astype(np.int32)
    row[9, ::2] = -1e-30
    row[10, :32] = np.nextafter(np.float32(1.75), np.float32(0)) * np.float32(4)
    row[11, 7] = 1.5 * 2.0 ** 127
    x = torch.from_numpy(row)[:, None].to(DEV)
    cache = torch.zeros((1, 1, binding.ttc_kv_page_bytes(64, 16)), device=DEV, dtype=torch.uint8)
    slots = torch.arange(12, device=DEV)
    binding.ttc_kv_append(cache, x, x.flip(0).contiguous(), slots)
    check_bytes(cache, torch.zeros_like(cache), 64, host(x), host(x.flip(0)), slots)
    k, v = binding.ttc_kv_read(cache, slots, 64, dtype=torch.float32)
    np.testing.assert_array_equal(host(k), oracle.numbers(*oracle.quantise(host(x))))
    np.testing.assert_array_equal(host(v), oracle.numbers(*oracle.quantise(host(x.flip(0)))))


@pytest.mark.parametrize("d,rot", [(64, 64), (128, 128), (128, 64), (256, 256), (64, 24), (64, 20), (128, 2), (256, 12)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_positions_on_the_way(d, rot, layout, dtype):
    tokens, heads, group, page, pages = 53, 3, 2, 32, 4
    k, v = some_tokens(tokens, heads, d, dtype, d + rot, spread=0.5)
    q = some_tokens(tokens, heads * group, d, dtype, 7)[0]
    gen = torch.Generator(device=DEV).manual_seed(2)
    pos = torch.randint(0, 4000, (tokens,), generator=gen, device=DEV)
    pos[5], pos[6] = -3, 4000
    table = binding.ttc_rope_table(4000, binding.rope_frequencies(rot)[0], scale=1.1, device=DEV)
    slots = some_slots(tokens, pages, page, 1)
    cache = torch.zeros((pages, heads, binding.ttc_kv_page_bytes(d, page)), device=DEV, dtype=torch.uint8)
    got_q = binding.ttc_kv_append(cache, k, v, slots, pos, table, layout=layout, q=q)
    assert torch.equal(got_q.nan_to_num(123.0), binding.ttc_rope(q, pos, table, layout=layout).nan_to_num(123.0))
    turned = binding.ttc_rope(k.float(), pos, table, layout=layout)
    check_bytes(cache, torch.zeros_like(cache), d, host(turned), host(v), slots)
    # every key within half a step of the oracle's rotation
    want = oracle.rope(host(k), pos.cpu().numpy(), host(table), layout)
    read = host(binding.ttc_kv_read(cache, slots, d, dtype=torch.float32)[0])
    e = oracle.quantise(want)[1]
    scale = np.repeat(np.where(e == 255, np.nan, np.exp2(e - 127.0)), 32, -1)
    y = np.abs(want) / scale
    step = np.where(y <= 2, 0.25, np.where(y <= 4, 0.5, 1.0)) * (1 + 2.0 ** -18)
    fine = np.isfinite(y)
    assert fine.mean() > 0.9 and (np.abs(read - want)[fine] <= (step * scale)[fine]).all()
    # strides, rows that begin anywhere, queries in place: the same bytes and bits
    wide = torch.zeros((tokens, (heads * (group + 2)) * d + 1), device=DEV, dtype=dtype)
    part = wide[:, 1:].unflatten(1, (heads * (group + 2), d))
    part[:, :heads * group], part[:, heads * group:-heads], part[:, -heads:] = q, k, v
    other = torch.zeros_like(cache)
    out = binding.ttc_kv_append(other, part[:, heads * group:-heads], part[:, -heads:], slots, pos, table, layout=layout, q=part[:, :heads * group],
                                q_out=part[:, :heads * group])
    assert torch.equal(other, cache) and torch.equal(out.nan_to_num(123.0), got_q.nan_to_num(123.0))


def test_one_token_at_a_time_fills_the_same_cache():
    tokens, heads, d, page = 70, 2, 128, 16
    k, v = some_tokens(tokens, heads, d, torch.bfloat16, 4)
    table = binding.ttc_rope_table(100, binding.rope_frequencies(d)[0], device=DEV)
    pos = torch.arange(tokens, device=DEV)
    at_once, one_by_one = binding.make_kv_cache(6, heads, d, page), binding.make_kv_cache(6, heads, d, page)
    binding.ttc_kv_append(at_once, k, v, pos + 5, pos, table)
    for t in range(tokens):
        binding.ttc_kv_append(one_by_one, k[t:t + 1], v[t:t + 1], pos[t:t + 1] + 5, pos[t:t + 1], table)
    assert torch.equal(at_once, one_by_one)


def test_slots_whose_offsets_pass_32_bits():
    heads, d, page = 8, 128, 256
    pages = (1 << 32) // (heads * binding.ttc_kv_page_bytes(d, page)) + 3
    cache = torch.zeros((pages, heads, binding.ttc_kv_page_bytes(d, page)), device=DEV, dtype=torch.uint8)
    k, v = some_tokens(4, heads, d, torch.bfloat16, 4)
    slots = torch.tensor([0, pages * page - 1, pages * page // 2 + 1, pages * page - page - 3], device=DEV)
    binding.ttc_kv_append(cache, k, v, slots)
    rk, rv = binding.ttc_kv_read(cache, slots, d, dtype=torch.float32)
    np.testing.assert_array_equal(host(rk), oracle.numbers(*oracle.quantise(host(k))))
    np.testing.assert_array_equal(host(rv), oracle.numbers(*oracle.quantise(host(v))))


def test_captured_append_replays_on_new_tokens():
    tokens, heads, d, page = 8, 2, 64, 16
    table = binding.ttc_rope_table(64, binding.rope_frequencies(d)[0], device=DEV)
    k, v = (t.clone() for t in some_tokens(tokens, heads, d, torch.bfloat16, 1))
    q, pos = k.clone(), torch.arange(tokens, device=DEV)
    slots, cache, q_out = pos.clone(), binding.make_kv_cache(3, heads, d, page), torch.empty_like(q)
    binding.ttc_kv_append(cache, k, v, slots, pos, table, q=q, q_out=q_out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.ttc_kv_append(cache, k, v, slots, pos, table, q=q, q_out=q_out)
    for step in range(3):
        a, b = some_tokens(tokens, heads, d, torch.bfloat16, 10 + step)
        k.copy_(a), v.copy_(b), q.copy_(b), pos.copy_(torch.arange(tokens, device=DEV) + 3 * step), slots.copy_(pos + step)
        eager = cache.clone()
        want = binding.ttc_kv_append(eager, k, v, slots, pos, table, q=q)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(cache, eager) and torch.equal(q_out, want)

"""Attention over the cache on the GPU where a call is at an edge: memory that was never written, a scale of 0, a cache without pages, bounds wider
than the call, replays on a workspace that nobody clears.  Bounds on errors are those of test_gpu_cached_attention; which kernel a case
takes is asked of the plan."""
import numpy as np
import pytest
import torch

from paper_2603_09221_amd import binding
from tests.attention_plan import describe, plan
from tests.test_gpu_cached_attention import DEV, TYPES, Setup, host

pytestmark = pytest.mark.gpu
MANY = [(torch.bfloat16, 64), (torch.bfloat16, 128), (torch.float32, 64)]   # what the kernel for many rows takes
FEW = [(t, d) for t in TYPES for d in (64, 128, 256)]


def planned(s, window=0, causal=True, max_kv=None):
    """The plan of the call that Setup `s` makes."""
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    heads = s.raw.shape[1]
    return plan(describe(len(s.kv_len), int(s.cu[-1]), s.q.shape[1], heads, s.d, s.page, s.dtype == torch.bfloat16, max(s.new),
                         max_kv or s.table.shape[1] * s.page, window, causal, s.pages), cus)


def few(dtype, d, seed=11):
    s = Setup([200, 150, 1, 63], [20, 1, 1, 5], 2, 3, d, 16, dtype, seed=seed)
    assert not planned(s).prompt
    return s


def many(dtype, d, seed=11):
    s = Setup([430, 200], [380, 200], 8, 8, d, 16, dtype, seed=seed)
    assert planned(s).prompt
    return s


CASES = [(few, *c) for c in FEW] + [(many, *c) for c in MANY]


def put_exponents(s, k, v):
    c, e = s.page * s.d, s.page * s.d // 32
    s.raw[..., c:c + e], s.raw[..., c + e:] = k.reshape(*s.raw.shape[:2], e), v.reshape(*s.raw.shape[:2], e)


@pytest.mark.parametrize("make,dtype,d", CASES)
def test_bytes_that_were_never_written_have_no_influence(make, dtype, d):
    """Tokens that no row sees hold exponents of 253 to 255 and any codes; so does page 0, which no sequence has, beside a page outside the cache."""
    s = make(dtype, d)
    rng = np.random.default_rng(1)
    s.raw = np.concatenate([s.raw[:1], s.raw])
    s.raw[0, :, s.page * s.d:] = 254
    s.table[s.table >= 0] += 1
    s.pages += 1
    s.table[0, 2] = -1
    exps = s.raw[..., s.page * s.d:]
    unseen = exps == 255
    exps[unseen] = rng.integers(253, 256, unseen.sum())
    s.check(binding.ttc_attention(**s.gpu()))
    s.check(binding.ttc_attention(**s.gpu(), window=70), window=70)
    s.check(binding.ttc_attention(**s.gpu(), causal=False), causal=False)


@pytest.mark.parametrize("exponent", [253, 254])
@pytest.mark.parametrize("make,dtype,d", CASES)
def test_exponents_above_252_are_nan_to_the_rows_that_see_them(make, dtype, d, exponent):
    s = make(dtype, d)
    k, v = s.exponents()
    k[s.table[0, 190 // 16], 1, 190 % 16, d // 32 - 1] = exponent       # keys of token 190, values of token 140 of the second sequence
    v[s.table[1, 140 // 16], 0, 140 % 16 // 4, 1, 140 % 4] = exponent
    put_exponents(s, k, v)
    (out, _, _), _ = s.oracle(window=30)
    assert 0 < np.isnan(out).mean() < 0.2
    s.check(binding.ttc_attention(**s.gpu(), window=30), window=30)
    slots = torch.tensor([int(s.table[0, 190 // 16]) * 16 + 190 % 16, int(s.table[1, 140 // 16]) * 16 + 140 % 16], device=DEV)
    for t in TYPES:
        rk, rv = (host(x) for x in binding.ttc_kv_read(torch.from_numpy(s.raw).to(DEV), slots, d, dtype=t))
        assert np.isnan(rk[0, 1, -32:]).all() and np.isnan(rv[1, 0, 32:64]).all()
        assert np.isnan(rk).sum() == 32 and np.isnan(rv).sum() == 32


@pytest.mark.parametrize("scale", [0.0, -0.0])
@pytest.mark.parametrize("make,dtype,d", CASES)
def test_a_scale_of_0_gives_the_mean_of_what_is_seen(make, dtype, d, scale):
    s = make(dtype, d)
    s.scale = scale
    s.table[0, 1] = -1
    s.check(binding.ttc_attention(**s.gpu()))
    s.check(binding.ttc_attention(**s.gpu(), window=50), window=50)
    s.check(binding.ttc_attention(**s.gpu(), causal=False), causal=False)


@pytest.mark.parametrize("make,dtype,d", [(few, torch.bfloat16, 128), (many, torch.bfloat16, 128), (many, torch.float32, 64)])
def test_nan_with_a_scale_of_0(make, dtype, d):
    """0 times NaN: a query or a key that is NaN makes NaN of the rows that have it or see it."""
    s = make(dtype, d)
    s.scale = 0.0
    k, v = s.exponents()
    k[s.table[0, 190 // 16], 1, 190 % 16, 1] = 255
    put_exponents(s, k, v)
    clean, s.q[3, 2, 5] = s.q.clone(), float("nan")
    got = binding.ttc_attention(**s.gpu(), window=30)
    assert torch.isnan(got["out"][3, 2]).all() and torch.isnan(got["lse"][3, 2])
    s.q = clean     # without the query's NaN: every other row as it is, and this one's from the oracle (bounds are taken from the queries)
    (out, lse, _), _ = s.oracle(window=30)
    got["out"][3, 2], got["lse"][3, 2] = torch.from_numpy(out[3, 2]).to(got["out"]), float(lse[3, 2])
    s.check(got, window=30)


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_without_being_told_and_a_wider_bound(dtype):
    """Through the C interface: no cu_q, so one row each, with max_q = 4: 384 sequences of 100 rows of a cache head, every one of them answered."""
    s = Setup([i % 70 for i in range(384)], [1] * 384, 1, 100, 64, 16, dtype, seed=3)
    a = s.gpu()
    want = binding.ttc_attention(a["q"], a["cache"], a["block_table"], a["kv_len"], scale=s.scale)
    s.check(want)
    lib, tokens, heads_q = binding.load(), *a["q"].shape[:2]
    for max_q in (4, 1, 37):
        out, lse = torch.full_like(a["q"], 77.0), torch.full((tokens, heads_q), 77.0, device=DEV)
        att = binding.Attention(binding.KvCache(a["cache"].data_ptr(), s.pages, 1, s.d, s.page), 384, tokens, heads_q, 1 if dtype == torch.bfloat16 else 0, 1, 0, s.scale, max_q,
                                a["block_table"].shape[1] * s.page, a["q"].data_ptr(), out.data_ptr(), lse.data_ptr(), heads_q * s.d, s.d,
                                heads_q * s.d, s.d, None, a["kv_len"].data_ptr(), a["block_table"].data_ptr(), a["block_table"].stride(0))
        work = torch.empty(max(lib.ttc_attention_workspace_bytes(att), 16), dtype=torch.uint8, device=DEV)
        assert lib.ttc_attention(att, work.data_ptr(), work.numel(), torch.cuda.current_stream().cuda_stream) == 0
        torch.cuda.synchronize()
        assert not (out == 77.0).any() and not (lse == 77.0).any()
        s.check({"out": out, "lse": lse})


@pytest.mark.parametrize("dtype,d", MANY)
def test_a_bound_on_new_tokens_far_above_what_there_is(dtype, d):
    s = Setup([29 * i % 97 + 3 for i in range(39)] + [1100], [i % 2 for i in range(39)] + [1050], 8, 4, d, 16, dtype, seed=d)
    a = s.gpu()
    p = plan(describe(40, int(s.cu[-1]), 32, 8, d, 16, dtype == torch.bfloat16, 1 << 19, s.table.shape[1] * 16))
    assert p.fits and p.prompt
    s.check(binding.ttc_attention(**{**a, "max_q": 1 << 19}))


@pytest.mark.parametrize("dtype,d", MANY)
def test_nan_missing_pages_and_negative_scale_where_rows_are_many(dtype, d):
    s = many(dtype, d, seed=5)
    k, v = s.exponents()
    k[s.table[0, 180 // 16], 1, 180 % 16, 1] = 255
    v[s.table[1, 75 // 16], 2, 75 % 16 // 4, 0, 75 % 4] = 255
    s.table[0, 3], s.table[1, 1] = -1, s.pages
    put_exponents(s, k, v)
    (out, _, _), _ = s.oracle(window=100)
    assert 0 < np.isnan(out).mean() < 0.2
    s.check(binding.ttc_attention(**s.gpu(), window=100), window=100)
    s.scale = -0.25
    got = binding.ttc_attention(**s.gpu())
    s.q, s.scale = -s.q, 0.25
    s.check(got)


@pytest.mark.parametrize("dtype,d", MANY)
@pytest.mark.parametrize("kv_len,new,group,window", [
    ([500, 260], [300, 100], 11, 130),
    ([37 * i % 101 + 9 for i in range(150)], [12 * i % 17 for i in range(150)], 16, 0),     # more sequences than a wavefront has lanes
    ([140, 300, 128], [128, 126, 125], 11, 0)])
def test_many_rows_by_the_plan(kv_len, new, group, window, dtype, d):
    s = Setup(kv_len, new, 8, group, d, 32, dtype, seed=len(new) + d)
    assert planned(s, window).prompt
    s.check(binding.ttc_attention(**s.gpu(), window=window), window=window)


@pytest.mark.parametrize("dtype", TYPES)
def test_replays_on_a_workspace_that_nobody_clears(dtype):
    """A captured call carries the same mark every time: what it left in the workspace must not be taken for this replay's parts.  Behind
    every replay no mark is left."""
    s = Setup([3000, 20, 2500], [1, 1, 1], 2, 4, 128, 64, dtype)
    a = s.gpu()
    p = planned(s)
    assert p.shared and p.workgroups > 8
    work = torch.zeros(p.workspace, dtype=torch.uint8, device=DEV)
    got = {k: v.clone() for k, v in binding.ttc_attention(**a).items()}
    binding.ttc_attention(**a, out=got, workspace=work)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.ttc_attention(**a, out=got, workspace=work)
    for step in range(6):
        a["q"].copy_(torch.randn(a["q"].shape, device=DEV))
        a["kv_len"].copy_(torch.tensor([3000 - 400 * step, 20 - step, 2500 - 300 * step], dtype=torch.int32))
        want = binding.ttc_attention(**a)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])
        assert not work[-2 * 8 * p.workgroups:].any()


def test_a_table_with_room_for_more_tokens_than_a_sequence_may_have():
    """max_kv is what the table has room for where the caller names none: 2^32 tokens here, of which a sequence has 300."""
    s = Setup([300, 64], [1, 1], 1, 4, 64, 256, torch.bfloat16)
    a = s.gpu()
    want = binding.ttc_attention(**a)
    wide = torch.full((2, 1 << 24), -1, dtype=torch.int32, device=DEV)
    wide[:, :a["block_table"].shape[1]] = a["block_table"]
    s.check(want)
    s.check(binding.ttc_attention(**{**a, "block_table": wide}))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("new", [1, 600])
def test_a_cache_without_pages_holds_nothing(dtype, new):
    """Lengths and a table, but no page: what the plan makes of it (lengths of 0) is tested without a GPU."""
    cache = binding.make_kv_cache(0, 8, 64, 16, device=DEV)
    q = torch.randn((2 * new, 64, 64), device=DEV).to(dtype)
    p = plan(describe(2, 2 * new, 64, 8, 64, 16, dtype == torch.bfloat16, new, 160, pages=0))
    assert p.max_kv == 0 and bool(p.prompt) == (new > 1)
    cu = torch.tensor([0, new, 2 * new], dtype=torch.int32, device=DEV)
    for causal in (True, False):
        got = binding.ttc_attention(q, cache, torch.zeros((2, 10), dtype=torch.int32, device=DEV), torch.tensor([150, 9], dtype=torch.int32, device=DEV),
                                    cu_q=cu, max_q=new, causal=causal)
        assert (got["out"] == 0).all() and torch.isneginf(got["lse"]).all()

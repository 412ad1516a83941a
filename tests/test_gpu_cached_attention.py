"""Attention over the cache on the GPU (ttc_attention) against the float64 oracle on the same bytes.

How far an entry may be off follows from the arithmetic (u = 2^-24): a score is a float32 sum of d exact products, (d + 4) u times the
sum of their magnitudes at most, scaling and maximum included; so a weight is off by e = twice that in proportion, an entry of out by
2 e of size = sum weight |value|.  Sums over the context pass at most 64 + n / 16 roundings one after the other.  With bfloat16
queries a weight and the result are rounded once each to 8 significant bits (2^-8 at most)."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as oracle
from paper_2603_09221_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


def host(t):
    return t.detach().cpu().double().numpy()


class Setup:
    """Sequences of kv_len tokens with the last `new` of each as queries, on pages in any order; what no sequence uses is random bytes,
    NaN among them."""

    def __init__(self, kv_len, new, heads, group, d, page, dtype, seed=0, spare=2, size=1.0):
        rng = np.random.default_rng(seed)
        self.kv_len, self.new, self.d, self.page, self.dtype = list(kv_len), list(new), d, page, dtype
        count = [-(-n // page) for n in kv_len]
        self.pages, width = sum(count) + spare, max(max(count), 1) + 1
        raw = rng.integers(0, 256, (self.pages, heads, page * (d + d // 16)), dtype=np.uint8)
        exps = raw[..., page * d:]
        exps[...] = rng.integers(122, 128, exps.shape)      # numbers of about 1
        order = rng.permutation(self.pages).astype(np.int32)
        self.table = np.full((len(kv_len), width), -1, np.int32)
        at = 0
        for i, c in enumerate(count):
            self.table[i, :c] = order[at:at + c]
            at += c
        self.raw, used = raw, np.zeros((self.pages, page), bool)
        for i, n in enumerate(kv_len):
            for j in range(n):
                used[self.table[i, j // page], j % page] = True
        self.spoil(~used)
        self.cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        # queries of such a size that scores are some units wide
        self.q = torch.from_numpy(size * rng.standard_normal((int(self.cu[-1]), heads * group, d)) * 8 / d ** 0.5).to(dtype)
        self.scale = 0.25

    def exponents(self):
        """views of the keys' and the values' exponents, (pages, heads, page, d/32) and (pages, heads, page/4, d/32, 4)"""
        p, h, n = self.raw.shape
        c, e = self.page * self.d, self.page * self.d // 32
        return self.raw[..., c:c + e].reshape(p, h, self.page, -1), self.raw[..., c + e:].reshape(p, h, self.page // 4, self.d // 32, 4)

    def spoil(self, where):
        """NaN into the tokens (pages, page) that `where` says"""
        p, h, n = self.raw.shape
        c, e = self.page * self.d, self.page * self.d // 32
        k = self.raw[..., c:c + e].reshape(p, h, self.page, -1).copy()
        v = self.raw[..., c + e:].reshape(p, h, self.page // 4, self.d // 32, 4).copy()
        k[np.broadcast_to(where[:, None, :, None], k.shape)] = 255
        four = where.reshape(p, 1, self.page // 4, 1, 4)
        v[np.broadcast_to(four, v.shape)] = 255
        self.raw[..., c:c + e], self.raw[..., c + e:] = k.reshape(p, h, e), v.reshape(p, h, e)

    def gpu(self):
        return dict(q=self.q.to(DEV), cache=torch.from_numpy(self.raw).to(DEV), block_table=torch.from_numpy(self.table).to(DEV),
                    kv_len=torch.tensor(self.kv_len, dtype=torch.int32, device=DEV), cu_q=torch.from_numpy(self.cu).to(DEV), max_q=max(self.new),
                    scale=self.scale)

    def oracle(self, causal=True, window=0):
        k, v = oracle.tokens(self.raw, self.d)
        return oracle.attention(host(self.q), k, v, self.table, self.kv_len, self.cu, self.page, self.pages, self.scale, causal, window), k

    def check(self, got, causal=True, window=0):
        (out, lse, size), k = self.oracle(causal, window)
        longest = max(max(self.kv_len), 1)
        key = np.nan_to_num(np.abs(k)).max()
        score = self.scale * np.abs(host(self.q)).sum(-1).max(initial=0.0) * key
        e = 2 * (self.d + 4) * U * score
        bf16 = self.dtype == torch.bfloat16
        tol = (2 * e + (64 + longest / 16) * U + (2.0 ** -8 if bf16 else 0.0)) * size + (2.0 ** -8 if bf16 else U) * np.abs(out) + 1e-30
        g = host(got["out"])
        assert np.array_equal(np.isnan(g), np.isnan(out))
        off = np.abs(g - out)
        worst = np.nanmax(off / tol, initial=0.0)
        print("largest error %.3g, %.3f of the bound" % (np.nanmax(off, initial=0.0), worst))
        assert worst <= 1.0
        l = host(got["lse"])
        assert np.array_equal(np.isneginf(l), np.isneginf(lse)) and np.array_equal(np.isnan(l), np.isnan(lse))
        fine = np.isfinite(lse)
        assert (np.abs(l - lse)[fine] <= e / 2 + (64 + longest / 16) * U + 4 * U * np.abs(lse[fine])).all()


TYPES = [torch.bfloat16, torch.float32]
DECODE = [0, 1, 15, 16, 17, 63, 64, 65, 127, 255, 256, 257, 700]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads,group,d,page", [(2, 4, 128, 64), (1, 1, 64, 16), (3, 3, 64, 32), (1, 16, 128, 16), (2, 7, 256, 128), (1, 20, 64, 256),
                                                (5, 1, 256, 16)])
def test_one_token_each(heads, group, d, page, dtype):
    s = Setup(DECODE, [1] * len(DECODE), heads, group, d, page, dtype, seed=d + group)
    a = s.gpu()
    s.check(binding.ttc_attention(**a))
    del a["cu_q"], a["max_q"]
    s.check(binding.ttc_attention(**a))     # a row each without being told
    s.check(binding.ttc_attention(**a, max_kv=700))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kv_len,new,heads,group,d,page", [
    ([5, 40, 3, 200, 64], [5, 3, 7, 200, 0], 2, 4, 128, 16),      # a whole prompt, a few tokens, more queries than keys, none at all
    ([129, 64, 1], [129, 33, 1], 1, 3, 64, 32),
    ([300, 77], [260, 77], 2, 1, 128, 64),
    ([90, 20], [50, 20], 1, 6, 256, 16),
    ([520], [519], 1, 2, 64, 256),
    ([33, 600, 1], [9, 70, 1], 2, 16, 64, 16)])
def test_prompts(kv_len, new, heads, group, d, page, dtype):
    s = Setup(kv_len, new, heads, group, d, page, dtype, seed=sum(new))
    s.check(binding.ttc_attention(**s.gpu()))
    s.check(binding.ttc_attention(**s.gpu(), causal=False), causal=False)


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 64), (torch.bfloat16, 128), (torch.float32, 64)])
@pytest.mark.parametrize("kv_len,new,heads,group,page,window", [
    ([150, 37, 300, 0, 64, 1, 65], [150, 33, 120, 3, 64, 1, 2], 8, 16, 16, 0),    # prompts, chunks, more queries than keys, empty rows
    ([129, 400], [129, 200], 16, 8, 256, 0),
    ([700, 64, 63, 128, 40], [90, 64, 63, 127, 70], 8, 16, 32, 50),               # windows shorter than a step
    ([500, 200], [300, 1], 8, 11, 64, 130)])
def test_many_rows(kv_len, new, heads, group, page, window, dtype, d):
    """Enough tiles of 128 rows for the kernel that is made for them."""
    s = Setup(kv_len, new, heads, group, d, page, dtype, seed=sum(new) + d)
    assert heads * (sum(new) * group // 128) >= 192
    s.check(binding.ttc_attention(**s.gpu(), window=window), window=window)
    if not window:
        s.check(binding.ttc_attention(**s.gpu(), causal=False), causal=False)


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 64), (torch.bfloat16, 128), (torch.float32, 64)])
@pytest.mark.parametrize("kv_len,new,heads,group", [
    ([140, 300, 128, 129], [128] * 4, 8, 8),                           # the same number of tiles each, contexts of other lengths
    ([140, 300, 128], [127, 128, 121], 8, 8),                          # and of an odd number of sequences
    ([140, 300, 128], [128, 126, 125], 8, 11),
    ([200, 190], [200, 190], 8, 11),
    ([37 * i % 101 + 9 for i in range(150)], [9 * i % 14 for i in range(150)], 3, 16),
    ([200, 90], [200, 90], 8, 11),
    ([37 * i % 101 + 9 for i in range(150)], [7 * i % 13 for i in range(150)], 3, 16)])   # more sequences than a wavefront has lanes, some without rows
def test_many_rows_in_tiles_of_many_sequences(kv_len, new, heads, group, dtype, d):
    s = Setup(kv_len, new, heads, group, d, 32, dtype, seed=len(new) + d)
    s.check(binding.ttc_attention(**s.gpu()))


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.float32, 64)])
@pytest.mark.parametrize("new,group", [(1, 20), (1, 64), (3, 21), (2, 32), (6, 16), (8, 16), (1, 128)])
def test_a_few_rows_of_each_of_many_sequences(new, group, dtype, d):
    """Rows for part of a tile, or for one, of 260 sequences."""
    lengths = [17 * i % 91 for i in range(260)]
    s = Setup(lengths, [new] * 260, 1, group, d, 16, dtype, seed=new * group)
    s.check(binding.ttc_attention(**s.gpu()))
    if new == 1:
        s.check(binding.ttc_attention(**{k: v for k, v in s.gpu().items() if k not in ("cu_q", "max_q")}))


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 64), (torch.bfloat16, 128), (torch.float32, 64)])
def test_many_rows_with_nan_missing_pages_and_negative_scale(dtype, d):
    s = Setup([300, 150], [250, 150], 8, 8, d, 16, dtype, seed=5)
    k, v = s.exponents()
    k[s.table[0, 180 // 16], 1, 180 % 16, 1] = 255              # keys of token 180, values of token 75 of the other sequence
    v[s.table[1, 75 // 16], 2, 75 % 16 // 4, 0, 75 % 4] = 255
    s.table[0, 3], s.table[1, 1] = -1, s.pages
    c, e = s.page * s.d, s.page * s.d // 32
    s.raw[..., c:c + e], s.raw[..., c + e:] = k.reshape(*s.raw.shape[:2], e), v.reshape(*s.raw.shape[:2], e)
    (out, _, _), _ = s.oracle(window=100)
    assert 0 < np.isnan(out).mean() < 0.2
    s.check(binding.ttc_attention(**s.gpu(), window=100), window=100)
    s.scale = -0.25
    got = binding.ttc_attention(**s.gpu())
    s.q, s.scale = -s.q, 0.25
    s.check(got)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("window", [1, 2, 17, 64, 100, 5000])
def test_windows(window, dtype):
    s = Setup([400, 63, 129, 1000], [150, 1, 129, 2], 2, 3, 64, 16, dtype, seed=window)
    s.check(binding.ttc_attention(**s.gpu(), window=window), window=window)
    s = Setup([400, 0, 64, 1], [1] * 4, 1, 8, 128, 64, dtype, seed=window)
    s.check(binding.ttc_attention(**s.gpu(), window=window), window=window)


@pytest.mark.parametrize("dtype", TYPES)
def test_long_contexts_are_shared_and_joined(dtype):
    s = Setup([5000, 1, 4097, 2048], [1, 1, 1, 1], 1, 4, 64, 32, dtype)
    s.check(binding.ttc_attention(**s.gpu()))
    s = Setup([6000], [3], 2, 2, 128, 64, dtype)
    s.check(binding.ttc_attention(**s.gpu()))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads,group,d,page", [(1, 5, 64, 16), (2, 16, 128, 64), (1, 3, 256, 32)])
def test_many_sequences_share_a_long_context(heads, group, d, page, dtype):
    """More sequences and row tiles than a wavefront has lanes, some of them empty, beside contexts that several workgroups divide; and the short
    ones alone, which take a workgroup each."""
    lengths = [37 * i % 301 for i in range(70)]
    s = Setup(lengths[:35] + [2900] + lengths[35:] + [0, 1500], [(i + 1) % 4 for i in range(73)], heads, group, d, page, dtype, seed=d)
    s.check(binding.ttc_attention(**s.gpu()))
    s.check(binding.ttc_attention(**s.gpu(), window=1900), window=1900)
    s = Setup(lengths, [i % 4 for i in range(70)], heads, group, d, page, dtype, seed=d)
    s.check(binding.ttc_attention(**s.gpu()))


@pytest.mark.parametrize("dtype", TYPES)
def test_nan_reaches_the_rows_that_see_it_only(dtype):
    """A token whose keys (or values) are NaN: earlier tokens' rows, and rows whose window has passed it, have no trace of it."""
    for part, window in (("key", 0), ("key", 9), ("value", 0), ("value", 9)):
        s = Setup([100, 70], [60, 70], 2, 3, 128, 16, dtype, seed=5)
        k, v = s.exponents()
        page, t = s.table[0, 75 // 16], 75 % 16
        if part == "key":
            k[page, 1, t, 2] = 255
        else:
            v[page, 1, t // 4, 2, t % 4] = 255      # entries 64 .. 95 of one head
        c, e = s.page * s.d, s.page * s.d // 32
        s.raw[..., c:c + e], s.raw[..., c + e:] = k.reshape(*s.raw.shape[:2], e), v.reshape(*s.raw.shape[:2], e)
        (out, _, _), _ = s.oracle(window=window)
        assert 0 < np.isnan(out).mean() < 0.5
        s.check(binding.ttc_attention(**s.gpu(), window=window), window=window)


def test_large_and_small_scores():
    """Scores some hundreds apart: all but the largest weights vanish, nothing overflows."""
    for dtype in TYPES:
        s = Setup([300, 40], [1, 40], 1, 4, 64, 16, dtype, size=60.0)
        s.check(binding.ttc_attention(**s.gpu()))
        s = Setup([300, 40], [1, 40], 1, 4, 64, 16, dtype, size=0.0)
        s.check(binding.ttc_attention(**s.gpu()))
        s = Setup([300, 40], [1, 40], 1, 4, 64, 16, dtype)
        s.scale = -0.25
        got = binding.ttc_attention(**s.gpu())
        s.q, s.scale = -s.q, 0.25
        s.check(got)


@pytest.mark.parametrize("dtype", TYPES)
def test_pages_outside_the_cache_hold_nothing(dtype):
    s = Setup([200, 150], [20, 1], 1, 4, 64, 16, dtype)
    s.table[0, 3], s.table[1, 0], s.table[0, 12] = -7, s.pages, 1 << 30
    s.check(binding.ttc_attention(**s.gpu()))


@pytest.mark.parametrize("dtype", TYPES)
def test_strides_alignment_streams_and_outputs_of_the_caller(dtype):
    s = Setup([77, 300, 9], [12, 1, 9], 2, 3, 128, 32, dtype)
    a = s.gpu()
    want = binding.ttc_attention(**a)
    n, h, d = a["q"].shape
    for first in (0, 1, 5):
        wide = torch.zeros((n, h * d + 9), dtype=dtype, device=DEV)
        q = wide[:, first:first + h * d].unflatten(1, (h, d))
        q.copy_(a["q"])
        out = {"out": torch.full((h, n, d + first), 7.0, dtype=dtype, device=DEV)[..., first:].transpose(0, 1),
               "lse": torch.empty((n, h), device=DEV)}
        got = binding.ttc_attention(**{**a, "q": q}, out=out)
        assert got["out"] is out["out"] and torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    got = binding.ttc_attention(**a, stream=stream)
    stream.synchronize()
    assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])
    got = binding.ttc_attention(**a, want_lse=False)
    assert "lse" not in got and torch.equal(got["out"], want["out"])
    # a table whose rows lie apart, and only some of whose columns are meant
    wide = torch.full((3, a["block_table"].shape[1] + 6), 123456, dtype=torch.int32, device=DEV)
    wide[:, :-6] = a["block_table"]
    got = binding.ttc_attention(**{**a, "block_table": wide[:, :-6]})
    assert torch.equal(got["out"], want["out"])


def test_lengths_that_do_not_fit_stay_inside():
    """More tokens than max_kv, more new tokens than max_q, row numbers outside q: read as the bounds say, rows left out keep their values."""
    s = Setup([64, 64], [1, 1], 1, 4, 64, 16, torch.float32)
    a = s.gpu()
    a["kv_len"] = torch.tensor([5000, -4], dtype=torch.int32, device=DEV)
    s.kv_len, keep = [64, 0], s.table
    s.check(binding.ttc_attention(**a, max_kv=64))
    s = Setup([64, 64], [8, 8], 1, 4, 64, 16, torch.float32)
    a = s.gpu()
    out = {"out": torch.full(a["q"].shape, 3.0, device=DEV)}
    got = binding.ttc_attention(**{**a, "max_q": 5, "cu_q": torch.tensor([0, 8, 99], dtype=torch.int32, device=DEV)}, out=out)
    full = binding.ttc_attention(**a)
    for first in (0, 8):
        assert (got["out"][first + 5:first + 8] == 3.0).all()
    assert torch.equal(got["out"][:5], full["out"][:5])


def test_offsets_that_pass_32_bits():
    heads, d, page = 8, 128, 256
    nbytes = binding.ttc_kv_page_bytes(d, page)
    pages = (1 << 32) // (heads * nbytes) + 4
    cache = torch.zeros((pages, heads, nbytes), device=DEV, dtype=torch.uint8)
    s = Setup([700, 30], [1, 4], heads, 2, d, page, torch.bfloat16, spare=0)
    a = s.gpu()
    cache[pages - s.pages:] = a["cache"]
    want = binding.ttc_attention(**a)
    table = torch.where(a["block_table"] >= 0, a["block_table"] + pages - s.pages, -1).int()
    got = binding.ttc_attention(**{**a, "cache": cache, "block_table": table})
    assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])


@pytest.mark.parametrize("dtype", TYPES)
def test_equal_calls_give_equal_bits_and_graphs_replay(dtype):
    s = Setup([3000, 20, 500], [1, 1, 1], 2, 4, 128, 64, dtype)
    a = s.gpu()
    first = binding.ttc_attention(**a)
    need_out = {k: v.clone() for k, v in first.items()}
    work = torch.empty(1 << 26, dtype=torch.uint8, device=DEV)
    binding.ttc_attention(**a, out=need_out, workspace=work)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.ttc_attention(**a, out=need_out, workspace=work)
    for step in range(3):
        a["q"].copy_(torch.randn(a["q"].shape, device=DEV))
        a["kv_len"].copy_(torch.tensor([3000 - 700 * step, 20 - step, 500 - step], dtype=torch.int32))
        want = binding.ttc_attention(**a)
        again = binding.ttc_attention(**a)
        assert torch.equal(want["out"], again["out"]) and torch.equal(want["lse"], again["lse"])
        work.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(need_out["out"], want["out"]) and torch.equal(need_out["lse"], want["lse"])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_cache_filled_and_read_in_one_sequence_of_calls(dtype, layout):
    """Prompts appended and answered, then single tokens, each step against the oracle on the cache's own bytes and the turned queries."""
    heads, group, d, page = 2, 4, 128, 16
    gen = torch.Generator(device=DEV).manual_seed(1)
    table = binding.ttc_rope_table(256, binding.rope_frequencies(d)[0], device=DEV)
    cache = binding.make_kv_cache(20, heads, d, page)
    order = torch.randperm(20, generator=gen, device=DEV)
    pages = order.view(2, 10).int()
    length = [0, 0]
    for new in ([37, 90], [1, 1], [5, 0], [1, 1]):
        pos = torch.cat([torch.arange(n, n + m, device=DEV) for n, m in zip(length, new)])
        seq = torch.repeat_interleave(torch.arange(2, device=DEV), torch.tensor(new, device=DEV))
        slots = pages[seq, pos // page].long() * page + pos % page
        x = torch.randn((sum(new), heads * (group + 2), d), generator=gen, device=DEV).to(dtype)
        q = binding.ttc_kv_append(cache, x[:, heads * group:-heads], x[:, -heads:], slots, pos, table, layout=layout, q=x[:, :heads * group])
        length = [n + m for n, m in zip(length, new)]
        cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        got = binding.ttc_attention(q, cache, pages, torch.tensor(length, dtype=torch.int32, device=DEV), cu_q=torch.from_numpy(cu).to(DEV),
                                    max_q=max(new))
        s = Setup.__new__(Setup)
        s.kv_len, s.new, s.d, s.page, s.dtype, s.pages, s.cu = length, new, d, page, dtype, 20, cu
        s.raw, s.table, s.q, s.scale = cache.cpu().numpy(), pages.cpu().numpy(), q.cpu(), d ** -0.5
        s.check(got)

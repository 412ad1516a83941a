"""Places of new tokens in a paged cache (ttc_kv_place) on the GPU against the oracle, number for number."""
import numpy as np
import pytest
import torch

from oracle import memory_oracle as oracle
from paper_2603_09221_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(values):
    return torch.tensor(np.asarray(values), dtype=torch.int32, device=DEV)


def setup(past, new, page, spare, seed=0, width=None):
    """A table whose held pages are drawn from the cache, and the list of the others; `spare` pages more than the new tokens need."""
    rng = np.random.default_rng(seed)
    held = [-(-p // page) for p in past]
    need = sum(max(0, -(-(p + max(n, 0)) // page) - h) for p, n, h in zip(past, new, held) if n >= 0)
    pages = sum(held) + max(0, need + spare) + 3
    order = rng.permutation(pages)
    width = width or max([1] + [-(-(p + max(n, 0)) // page) for p, n in zip(past, new)])
    table = np.full((len(past), width), -1, dtype=np.int32)
    at = 0
    for s, h in enumerate(held):
        table[s, :h] = order[at:at + h]
        at += h
    count = max(0, need + spare)
    free = np.full(pages, -7, dtype=np.int32)
    free[:count] = order[at:at + count]
    return table, pages, free, count


def check(past, new, page, tokens, spare=3, seed=0, stride=0, with_list=True, in_place=False):
    table, pages, free, count = setup(past, new, page, spare, seed)
    want = oracle.place(past, new, table, page, tokens, pages, free if with_list else None, count)
    wide = torch.full((len(past), table.shape[1] + stride), 99, dtype=torch.int32, device=DEV)
    on = wide[:, :table.shape[1]]
    on.copy_(torch.from_numpy(table))
    past_t, listed, count_t = i32(past), i32(free), i32([count])
    kw = dict(free=listed, free_count=count_t) if with_list else {}
    out = {"kv_len": past_t, **({"free_count": count_t} if with_list else {})} if in_place else None
    got = binding.ttc_kv_place(past_t, i32(new), on, page, tokens, pages=pages, out=out, **kw)
    for name in ("cu_q", "kv_len", "positions", "slots", "sequence"):
        assert np.array_equal(got[name].cpu().numpy(), want[name]), name
    assert np.array_equal(on.cpu().numpy(), want["table"]) and (wide[:, table.shape[1]:] == 99).all()
    if with_list:
        assert np.array_equal(listed.cpu().numpy(), want["free"]) and int(got["free_count"]) == want["free_count"] and int(got["missing"]) == want["missing"]


@pytest.mark.parametrize("page", [1, 16, 48, 64, 256])
@pytest.mark.parametrize("stride,in_place", [(0, False), (3, True)])
def test_single_tokens(page, stride, in_place):
    rng = np.random.default_rng(page)
    for n in (1, 3, 64, 65, 1000):
        past = rng.integers(0, 300, n)
        new = np.where(rng.random(n) < 0.2, -1, rng.integers(0, 2, n))
        check(past, new, page, max(0, int(new.clip(0).sum())) + 4, seed=n, stride=stride, in_place=in_place)


@pytest.mark.parametrize("page", [16, 64])
def test_prompts(page):
    """Beyond what one workgroup places itself, and more sequences than it adds up at once."""
    rng = np.random.default_rng(1)
    for n, most in ((1, 9000), (7, 2000), (70, 150), (1500, 9), (2100, 5), (3000, 1)):
        past = rng.integers(0, 200, n)
        new = np.where(rng.random(n) < 0.1, -1, rng.integers(0, most + 1, n))
        check(past, new, page, int(new.clip(0).sum()), seed=n)
        check(past, new, page, int(new.clip(0).sum()) + 17, seed=n, in_place=True)


def test_lists_that_run_out_and_lists_that_grow():
    past, new = [0, 70, 500, 64, 10], [200, 60, -1, 1, 130]
    for spare in (-1, -2, -4, -100, 0):
        check(past, new, 64, 391, spare=spare)
    check([3000] * 6, [-1] * 6, 16, 2)                       # everything given back
    check([0, 0, 0], [0, 0, 0], 16, 0)
    check([5, 6], [100, 100], 16, 150)                       # rows for some of the tokens alone
    check([5, 6], [-1, 100], 16, 150, with_list=False)
    check([5, 600] * 900, [-3, 1] * 900, 16, 900, with_list=False)


def test_lengths_pages_and_numbers_beyond_their_limits():
    """Negative and large lengths, table entries and listed pages outside the cache, more tokens than the table has columns."""
    table = i32([[0, 1, -1], [7, 99, 5], [-4, 2, 3], [6, -1, -1]])
    free = i32([50, -3, 4, 8])
    past, new = [-9, 40, 48, 3], [20, -1, 30, 2_000_000_000]
    want = oracle.place(past, new, table.cpu().numpy(), 16, 100, 9, free.cpu().numpy(), 3)
    count = i32([3])
    got = binding.ttc_kv_place(i32(past), i32(new), table, 16, 100, pages=9, free=free, free_count=count)
    for name in ("cu_q", "kv_len", "positions", "slots", "sequence"):
        assert np.array_equal(got[name].cpu().numpy(), want[name]), name
    assert np.array_equal(table.cpu().numpy(), want["table"]) and np.array_equal(free.cpu().numpy(), want["free"])
    # a list count beyond the list, and below 0
    for n in (400, -5):
        again = binding.ttc_kv_place(i32([0]), i32([20]), i32([[-1, -1]]), 16, 20, pages=9, free=i32([1, 2, 3]), free_count=i32([n]))
        assert int(again["free_count"]) == (1 if n > 0 else 0) and int(again["missing"]) == (0 if n > 0 else 2)


def test_nobody():
    got = binding.ttc_kv_place(i32([]), i32([]), torch.zeros((0, 4), dtype=torch.int32, device=DEV), 16, 5, pages=9, free=i32([1, 2]), free_count=i32([2]))
    assert got["cu_q"].tolist() == [0] and got["slots"].tolist() == [-1] * 5 and got["positions"].tolist() == [0] * 5 and int(got["free_count"]) == 2


def test_a_replayed_step_goes_on_by_itself():
    """Lengths, table and list in place: every replay is the next step, as the oracle takes it; another stream gives the same."""
    rng = np.random.default_rng(3)
    n, page, pages = 40, 16, 400
    past = rng.integers(0, 50, n)
    table, pages, free, count = setup(past, [100] * n, page, 40)
    past_t, on, listed, count_t, new = i32(past), i32(table), i32(free), i32([count]), i32([1] * n)
    out = {"kv_len": past_t, "free_count": count_t}
    call = lambda **kw: binding.ttc_kv_place(past_t, new, on, page, n + 3, pages=pages, free=listed, free_count=count_t, out=out, **kw)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    call(stream=stream)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    want = oracle.place(past, [1] * n, table, page, n + 3, pages, free, count)
    for step in range(6):
        asked = np.ones(n, dtype=np.int64)
        asked[step::7] = -1 if step % 2 else 0
        new.copy_(torch.from_numpy(asked))
        want = oracle.place(want["kv_len"], asked, want["table"], page, n + 3, pages, want["free"], want["free_count"])
        graph.replay()
        torch.cuda.synchronize()
        for name in ("cu_q", "kv_len", "positions", "slots", "sequence"):
            assert np.array_equal(got[name].cpu().numpy(), want[name]), (step, name)
        assert np.array_equal(on.cpu().numpy(), want["table"]) and np.array_equal(listed.cpu().numpy(), want["free"])
        assert int(count_t) == want["free_count"]

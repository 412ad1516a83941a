"""C-ABI boundary of include/ttc_attention.h without a GPU: the library exports what the header declares, and bad arguments are refused
before the device is touched."""
import ctypes
import os
import re

import pytest
import torch

from paper_2603_09221_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
FAKE = 0x1000   # never read: every call below is refused, or has nothing to do


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return binding.load()


def test_exports_match_header(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ttc_attention.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(ttc_[a-z_0-9]+)\s*\(", text)))
    assert names == sorted(binding.ATTENTION_EXPORTS)
    for name in names:
        assert hasattr(lib, name), name


def test_structures_have_the_headers_size(lib, tmp_path):
    """Field by field the sizes of the descriptors, as a C compiler lays them out."""
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include "ttc_attention.h"\nint main(void) { printf("%zu %zu %zu %zu", sizeof(ttc_rope_t), '
                   'sizeof(ttc_kv_cache_t), sizeof(ttc_kv_append_t), sizeof(ttc_attention_t)); return 0; }\n')
    import subprocess
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "sizes")], check=True)
    got = subprocess.run([str(tmp_path / "sizes")], capture_output=True, text=True, check=True).stdout.split()
    assert [int(g) for g in got] == [ctypes.sizeof(s) for s in (binding.Rope, binding.KvCache, binding.KvAppend, binding.Attention)]


def _fill(s, **kw):
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def rope(**kw):
    s = binding.Rope(4, 2, 64, 64, 0, 0, FAKE, 2 * FAKE, 128, 64, 128, 64, FAKE, FAKE, 16)
    return _fill(s, **kw)


@pytest.mark.parametrize("want,change", [
    (INVALID, dict(tokens=-1)), (INVALID, dict(heads=0)), (INVALID, dict(d=0)), (INVALID, dict(rot=3)), (INVALID, dict(rot=66)),
    (INVALID, dict(rot=-2)), (INVALID, dict(dtype=2)), (INVALID, dict(layout=2)), (INVALID, dict(x=None)), (INVALID, dict(y=None)),
    (INVALID, dict(x=FAKE + 2)), (INVALID, dict(positions=None)), (INVALID, dict(table=None)), (INVALID, dict(table=FAKE + 4)),
    (INVALID, dict(table_rows=0)), (INVALID, dict(y=FAKE, y_token=256)), (UNSUPPORTED, dict(heads=1 << 25)), (OK, dict(tokens=0))])
def test_rope_refusals(lib, want, change):
    for call in (lib.ttc_rope, lib.ttc_rope_backward):
        assert call(rope(**change), None) == want
        assert call(None, None) == INVALID


def test_rope_table_refusals(lib):
    assert lib.ttc_rope_table(None, 4, 4, FAKE, 1.0, None) == INVALID
    assert lib.ttc_rope_table(FAKE, 4, 4, None, 1.0, None) == INVALID
    assert lib.ttc_rope_table(FAKE, -1, 4, FAKE, 1.0, None) == INVALID
    assert lib.ttc_rope_table(FAKE, 4, 4, FAKE, float("inf"), None) == INVALID
    assert lib.ttc_rope_table(None, 0, 4, None, 1.0, None) == OK


CACHE = dict(data=FAKE, pages=4, heads=2, d=128, page=64)
BAD_CACHES = [(INVALID, dict(pages=-1)), (INVALID, dict(heads=0)), (INVALID, dict(data=None)), (INVALID, dict(data=FAKE + 8)),
              (UNSUPPORTED, dict(d=96)), (UNSUPPORTED, dict(page=48)), (UNSUPPORTED, dict(page=8)), (UNSUPPORTED, dict(page=512))]


def cache(**kw):
    return _fill(binding.KvCache(), **{**CACHE, **kw})


def test_page_bytes(lib):
    for d in (64, 128, 256):
        for page in (16, 32, 64, 128, 256):
            assert binding.ttc_kv_page_bytes(d, page) == page * d * 2 // 2 + 2 * page * d // 32
    for d, page in ((32, 64), (128, 0), (128, -16), (128, 24), (0, 64)):
        assert binding.ttc_kv_page_bytes(d, page) == 0


def append(**kw):
    s = binding.KvAppend(cache=cache(), tokens=4, dtype=1, rot=128, layout=0, k=FAKE, v=FAKE, k_token=256, k_head=128, v_token=256,
                         v_head=128, slots=FAKE, positions=FAKE, table=FAKE, table_rows=8)
    return _fill(s, **kw)


@pytest.mark.parametrize("want,change", [(w, dict(cache=cache(**c))) for w, c in BAD_CACHES] + [
    (INVALID, dict(tokens=-1)), (INVALID, dict(dtype=7)), (INVALID, dict(k=None)), (INVALID, dict(v=None)), (INVALID, dict(k=FAKE + 1)),
    (INVALID, dict(slots=None)), (INVALID, dict(rot=130)), (INVALID, dict(rot=1)), (INVALID, dict(positions=None)), (INVALID, dict(table=None)),
    (INVALID, dict(q=FAKE)), (INVALID, dict(q_out=FAKE)), (INVALID, dict(q=FAKE, q_out=2 * FAKE, heads_q=0)),
    (INVALID, dict(q=FAKE, q_out=FAKE, heads_q=2, q_token=256, q_head=128, q_out_token=512, q_out_head=128)),
    (UNSUPPORTED, dict(q=FAKE, q_out=2 * FAKE, heads_q=70000)), (UNSUPPORTED, dict(tokens=1 << 27)), (OK, dict(tokens=0))])
def test_append_refusals(lib, want, change):
    assert lib.ttc_kv_append(append(**change), None) == want
    assert lib.ttc_kv_append(None, None) == INVALID


def test_read_refusals(lib):
    for want, c in BAD_CACHES:
        assert lib.ttc_kv_read(cache(**c), FAKE, 4, 0, FAKE, FAKE, None) == want
    assert lib.ttc_kv_read(None, FAKE, 4, 0, FAKE, FAKE, None) == INVALID
    assert lib.ttc_kv_read(cache(), None, 4, 0, FAKE, FAKE, None) == INVALID
    assert lib.ttc_kv_read(cache(), FAKE, -4, 0, FAKE, FAKE, None) == INVALID
    assert lib.ttc_kv_read(cache(), FAKE, 4, 3, FAKE, FAKE, None) == INVALID
    assert lib.ttc_kv_read(cache(), FAKE, 4, 0, FAKE + 8, FAKE, None) == INVALID
    assert lib.ttc_kv_read(cache(), FAKE, 0, 0, FAKE, FAKE, None) == OK


def attention(**kw):
    s = binding.Attention(cache=cache(), sequences=3, tokens=3, heads_q=8, dtype=1, causal=1, window=0, scale=0.1, max_q=1, max_kv=200,
                          q=FAKE, out=2 * FAKE, lse=None, q_token=1024, q_head=128, out_token=1024, out_head=128, cu_q=None, kv_len=FAKE,
                          block_table=FAKE, table_stride=4)
    return _fill(s, **kw)


@pytest.mark.parametrize("want,change", [(w, dict(cache=cache(**c))) for w, c in BAD_CACHES] + [
    (INVALID, dict(sequences=-1)), (INVALID, dict(tokens=-1)), (INVALID, dict(dtype=2)), (INVALID, dict(causal=2)), (INVALID, dict(window=-1)),
    (INVALID, dict(window=4, causal=0)), (INVALID, dict(scale=float("nan"))), (INVALID, dict(heads_q=7)), (INVALID, dict(heads_q=0)),
    (INVALID, dict(max_q=-1)), (INVALID, dict(max_kv=-1)), (UNSUPPORTED, dict(max_kv=(1 << 30) + 1)), (UNSUPPORTED, dict(max_q=1 << 29)),
    (UNSUPPORTED, dict(sequences=1 << 24)), (INVALID, dict(q=None)), (INVALID, dict(out=None)), (INVALID, dict(out=FAKE)),
    (INVALID, dict(q=FAKE + 1)), (INVALID, dict(lse=FAKE + 2)), (INVALID, dict(kv_len=None)), (INVALID, dict(block_table=None)),
    (INVALID, dict(table_stride=-1)), (INVALID, dict(tokens=4)), (OK, dict(tokens=0)), (OK, dict(sequences=0)), (OK, dict(max_q=0))])
def test_attention_refusals(lib, want, change):
    assert lib.ttc_attention(attention(**change), FAKE, 1 << 40, None) == want
    assert lib.ttc_attention(None, FAKE, 1 << 40, None) == INVALID


def test_attention_workspace(lib):
    long = attention(sequences=1, tokens=1, max_kv=100000)
    need = lib.ttc_attention_workspace_bytes(long)
    assert need > 0
    assert lib.ttc_attention(long, None, 0, None) == WORKSPACE
    assert lib.ttc_attention(long, FAKE, need - 1, None) == WORKSPACE
    assert lib.ttc_attention(long, FAKE + 8, need, None) == WORKSPACE
    assert lib.ttc_attention_workspace_bytes(attention(max_kv=64)) == 0
    assert lib.ttc_attention_workspace_bytes(attention(heads_q=7)) == 0


def test_wrapper_refuses_tensors_that_do_not_fit():
    q, k = torch.zeros(3, 8, 128), torch.zeros(3, 2, 128)
    c = torch.zeros(4, 2, 64 * 136, dtype=torch.uint8)
    table, lens = torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    slots, rope_table = torch.zeros(3, dtype=torch.int64), torch.zeros(8, 64, 2)
    ok = dict(q=q, cache=c, block_table=table, kv_len=lens)
    for change in (dict(q=q.half()), dict(q=q[0]), dict(q=q.transpose(0, 2)), dict(cache=c.float()), dict(cache=c[..., :-1]), dict(block_table=table.long()),
                   dict(kv_len=lens.long()), dict(kv_len=lens[:2]), dict(max_kv=257), dict(cu_q=torch.zeros(4, dtype=torch.int32)),
                   dict(cu_q=torch.zeros(3, dtype=torch.int32), max_q=1), dict(block_table=table[:2]),
                   dict(out={"out": q.bfloat16()}), dict(out={"out": q, "lse": torch.zeros(3, 7)})):
        with pytest.raises(ValueError):
            binding.ttc_attention(**{**ok, **change})
    for args, kw in (((c, k, k[:2], slots), {}), ((c, k, k, slots.int()), {}), ((c, k[:, :1], k[:, :1], slots), {}), ((c, k, k.bfloat16(), slots), {}),
                     ((c, k, k, slots, None, rope_table[..., 0]), {}), ((c, k, k, slots, slots, torch.zeros(8, 65, 2)), {}), ((c, k, k, slots), dict(q_out=q)),
                     ((c, k, k, slots, slots, rope_table), dict(layout="other"))):
        with pytest.raises((ValueError, AttributeError)):
            binding.ttc_kv_append(*args, **kw)
    for args, kw in (((q, slots[:2], rope_table), {}), ((q, slots.int(), rope_table), {}), ((q.double(), slots, rope_table), {}),
                     ((q, slots, rope_table.double()), {}), ((q, slots, rope_table), dict(out=q[:, :4])), ((q, slots, rope_table), dict(layout="x"))):
        with pytest.raises(ValueError):
            binding.ttc_rope(*args, **kw)
    with pytest.raises(ValueError):
        binding.ttc_kv_read(c, slots, 128, dtype=torch.float16)
    with pytest.raises(ValueError):
        binding.make_kv_cache(4, 2, 96, 64, device="cpu")

"""C-ABI boundary of include/ttc_memory.h and of ttc_kv_place without a GPU: exports, the descriptors' sizes, what is refused before the
device is touched, by the entry points and by their wrappers."""
import ctypes
import os
import re
import subprocess

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
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ttc_memory.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(ttc_[a-z_0-9]+)\s*\(", text)))
    assert names == sorted(binding.MEMORY_EXPORTS)
    for name in names:
        assert hasattr(lib, name), name


def test_structures_have_the_headers_layout(tmp_path):
    """Sizes and every field's place, as a C compiler lays them out."""
    of = {"ttc_kv_place_t": binding.KvPlace, "ttc_linear_attention_t": binding.LinearAttention,
          "ttc_linear_attention_backward_t": binding.LinearAttentionBackward, "ttc_residual_norm_t": binding.ResidualNorm,
          "ttc_residual_norm_backward_t": binding.ResidualNormBackward}
    lines = []
    for name, s in of.items():
        lines.append('printf("%%zu\\n", sizeof(%s));' % name)
        lines += ['printf("%%zu\\n", offsetof(%s, %s));' % (name, f[0]) for f in s._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "ttc_attention.h"\n#include "ttc_memory.h"\nint main(void) { %s return 0; }\n'
                   % "\n".join(lines))
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "layout")], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True, check=True).stdout.split()]
    want = []
    for s in of.values():
        want.append(ctypes.sizeof(s))
        want += [getattr(s, f[0]).offset for f in s._fields_]
    assert got == want


def _fill(s, kw):
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def place(**kw):
    return _fill(binding.KvPlace(4, 8, 16, 64, 3, FAKE, FAKE, FAKE, 3, FAKE, 16, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE), kw)


@pytest.mark.parametrize("want,change", [
    (INVALID, dict(sequences=-1)), (INVALID, dict(tokens=-1)), (INVALID, dict(pages=-1)), (INVALID, dict(width=-1)), (UNSUPPORTED, dict(page=0)),
    (UNSUPPORTED, dict(page=65537)), (UNSUPPORTED, dict(sequences=1 << 30)), (UNSUPPORTED, dict(tokens=1 << 30)), (UNSUPPORTED, dict(pages=1 << 31)),
    (INVALID, dict(past=None)), (INVALID, dict(new_tokens=None)), (INVALID, dict(block_table=None)), (INVALID, dict(table_stride=-1)),
    (INVALID, dict(table_stride=2)), (INVALID, dict(cu_q=None)), (INVALID, dict(kv_len=None)), (INVALID, dict(positions=None)),
    (INVALID, dict(slots=None)), (INVALID, dict(slots=FAKE + 4)), (INVALID, dict(sequence=FAKE + 2)), (INVALID, dict(free_count=None)),
    (INVALID, dict(free_count_out=None)), (INVALID, dict(free_capacity=-1)), (INVALID, dict(missing=FAKE + 1))])
def test_place_refusals(lib, want, change):
    assert lib.ttc_kv_place(place(**change), None) == want
    assert lib.ttc_kv_place(None, None) == INVALID


def linear(**kw):
    s = binding.LinearAttention(sequences=2, tokens=600, heads=4, heads_qk=2, dk=64, dv=128, dtype=1, max_q=500, scale=0.1, q=FAKE, k=FAKE, v=FAKE,
                                out=2 * FAKE, q_token=128, q_head=64, k_token=128, k_head=64, v_token=512, v_head=128, out_token=512, out_head=128,
                                log_decay=FAKE, g_token=4, g_head=1, cu_q=FAKE, state_in=FAKE, state_out=FAKE, state_rows=2)
    return _fill(s, kw)


SIZES = [(INVALID, dict(sequences=-1)), (INVALID, dict(tokens=-1)), (INVALID, dict(heads=0)), (INVALID, dict(heads=3)), (INVALID, dict(heads_qk=0)),
         (INVALID, dict(dtype=2)), (INVALID, dict(max_q=-1)), (INVALID, dict(scale=float("nan"))), (UNSUPPORTED, dict(dk=4)), (UNSUPPORTED, dict(dk=60)),
         (UNSUPPORTED, dict(dk=264)), (UNSUPPORTED, dict(dv=0)), (UNSUPPORTED, dict(dv=512)), (UNSUPPORTED, dict(tokens=1 << 31)),
         (UNSUPPORTED, dict(heads=1 << 24)), (INVALID, dict(cu_q=None)), (INVALID, dict(q=None)), (INVALID, dict(k=None)), (INVALID, dict(v=None)),
         (INVALID, dict(log_decay=None)), (INVALID, dict(q=FAKE + 1)), (INVALID, dict(log_decay=FAKE + 2)), (INVALID, dict(cu_q=FAKE + 2)),
         (INVALID, dict(state_in=FAKE + 8)), (INVALID, dict(state_rows=-1)), (INVALID, dict(state_row=FAKE + 2)), (INVALID, dict(kv_len=FAKE + 1))]


@pytest.mark.parametrize("want,change", SIZES + [(INVALID, dict(out=None)), (INVALID, dict(out=FAKE)), (INVALID, dict(state_out=FAKE + 4)),
                                                 (OK, dict(sequences=0)), (OK, dict(tokens=0, state_out=None)), (OK, dict(max_q=0, state_out=None))])
def test_linear_attention_refusals(lib, want, change):
    assert lib.ttc_linear_attention(linear(**change), FAKE, 1 << 40, None) == want
    assert lib.ttc_linear_attention(None, FAKE, 1 << 40, None) == INVALID


def test_linear_attention_workspace(lib):
    a = linear()
    need = lib.ttc_linear_attention_workspace_bytes(a)
    assert need > 0
    for at, size in ((None, 0), (FAKE, need - 1), (FAKE + 8, need)):
        assert lib.ttc_linear_attention(a, at, size, None) == WORKSPACE
    assert lib.ttc_linear_attention_workspace_bytes(linear(max_q=1)) == 0
    assert lib.ttc_linear_attention_workspace_bytes(linear(heads=3)) == 0


def test_linear_attention_refuses_what_a_launch_does_not_count(lib):
    for change in (dict(tokens=1 << 28, max_q=1 << 28, heads=1, heads_qk=1), dict(tokens=1 << 26, max_q=1 << 25)):
        assert lib.ttc_linear_attention(linear(**change), None, 0, None) == WORKSPACE, change
    for change in (dict(tokens=1 << 30, max_q=1 << 30), dict(sequences=1 << 22), dict(heads=1 << 23), dict(sequences=1 << 20, dk=256, dv=256)):
        assert lib.ttc_linear_attention(linear(**change), FAKE, 1 << 62, None) == UNSUPPORTED, change
    # a gradient's results are contiguous, whatever the strides of what it is given
    assert lib.ttc_linear_attention_backward(backward(dict(heads=1 << 16, heads_qk=1 << 16)), FAKE, 1 << 62, None) == UNSUPPORTED


def backward(change_forward={}, **kw):
    return _fill(binding.LinearAttentionBackward(linear(**change_forward), FAKE, 512, 128, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE), kw)


def test_linear_attention_backward_refusals(lib):
    for want, change in SIZES:
        assert lib.ttc_linear_attention_backward(backward(change), FAKE, 1 << 40, None) == want, change
    for change in (dict(gout=None), dict(gout=FAKE + 1), dict(gq=None), dict(gk=None), dict(gv=FAKE + 1), dict(glog_decay=None), dict(gstate=FAKE + 8),
                   dict(gstate_out=FAKE + 4)):
        assert lib.ttc_linear_attention_backward(backward(**change), FAKE, 1 << 40, None) == INVALID, change
    assert lib.ttc_linear_attention_backward(None, FAKE, 1 << 40, None) == INVALID
    need = lib.ttc_linear_attention_backward_workspace_bytes(backward())
    assert need > 0
    for at, size in ((None, 0), (FAKE, need - 1), (FAKE + 8, need)):
        assert lib.ttc_linear_attention_backward(backward(), at, size, None) == WORKSPACE


def norm(**kw):
    s = binding.ResidualNorm(tokens=4, features=64, groups=1, dtype=1, post=1, pre=2, act=2, post_eps=1e-5, pre_eps=1e-5, scale=1.0, y=FAKE, gate=2 * FAKE,
                             residual=3 * FAKE, r=4 * FAKE, h=5 * FAKE, y_token=64, gate_token=64, residual_token=64, r_token=64, h_token=64)
    return _fill(s, kw)


NORM_SIZES = [(INVALID, dict(tokens=-1)), (INVALID, dict(features=0)), (INVALID, dict(groups=0)), (INVALID, dict(groups=3)), (UNSUPPORTED, dict(groups=16)),
              (UNSUPPORTED, dict(features=16392)), (INVALID, dict(dtype=2)), (INVALID, dict(post=3)), (INVALID, dict(pre=-1)), (INVALID, dict(act=3)),
              (INVALID, dict(post_eps=-1.0)), (INVALID, dict(pre_eps=float("nan"))), (INVALID, dict(scale=float("inf"))), (INVALID, dict(y=None)),
              (INVALID, dict(y=FAKE + 1)), (INVALID, dict(gate=FAKE + 1)), (INVALID, dict(residual=FAKE + 1)), (INVALID, dict(pre_gain=FAKE + 2))]


@pytest.mark.parametrize("want,change", NORM_SIZES + [
    (INVALID, dict(h=None)), (INVALID, dict(pre=0)), (INVALID, dict(r=4 * FAKE + 1)), (INVALID, dict(h=4 * FAKE)), (INVALID, dict(r=3 * FAKE, r_token=128)),
    (INVALID, dict(h=FAKE, h_token=128)), (INVALID, dict(r_token=0)), (INVALID, dict(h_token=63)), (INVALID, dict(r=None, h=None)), (OK, dict(tokens=0))])
def test_norm_refusals(lib, want, change):
    assert lib.ttc_residual_norm(norm(**change), None) == want
    assert lib.ttc_residual_norm(None, None) == INVALID


def test_norm_backward_refusals(lib):
    def call(change_forward={}, **kw):
        b = binding.ResidualNormBackward(forward=norm(**change_forward), gr=FAKE, gh=FAKE, gr_token=64, gh_token=64, gy=FAKE)
        return _fill(b, kw)

    for want, change in NORM_SIZES:
        assert lib.ttc_residual_norm_backward(call(change), FAKE, 1 << 40, None) == want, change
    for change in (dict(gh=None), dict(gr=FAKE + 1), dict(gy=FAKE + 1), dict(gpost_gain=FAKE), dict(gpre_offset=FAKE), dict(gresidual_gain=FAKE)):
        assert lib.ttc_residual_norm_backward(call(**change), FAKE, 1 << 40, None) == INVALID, change
    assert lib.ttc_residual_norm_backward(call(dict(gate=None), ggate=FAKE), FAKE, 1 << 40, None) == INVALID
    assert lib.ttc_residual_norm_backward(call(dict(residual=None), gresidual=FAKE), FAKE, 1 << 40, None) == INVALID
    summed = call(dict(pre_gain=FAKE), gpre_gain=FAKE)
    need = lib.ttc_residual_norm_backward_workspace_bytes(summed)
    assert need > 0 and lib.ttc_residual_norm_backward(summed, FAKE, need - 1, None) == WORKSPACE
    assert lib.ttc_residual_norm_backward_workspace_bytes(call()) == 0


def i32(*n):
    return torch.zeros(n, dtype=torch.int32)


def place_call(**change):
    a = dict(past=i32(3), new_tokens=i32(3), block_table=i32(3, 4), page=64, tokens=5, pages=16, free=i32(16), free_count=i32(1))
    return binding.ttc_kv_place(**{**a, **change})


def linear_args(**change):
    a = dict(q=torch.zeros(6, 2, 64), k=torch.zeros(6, 2, 64), v=torch.zeros(6, 4, 32), log_decay=torch.zeros(6, 4), cu_q=i32(3), max_q=6)
    return {**a, **change}


def test_place_wrapper_refuses():
    with pytest.raises(ValueError, match="on a GPU"):
        place_call()
    for change in (dict(past=i32(2)), dict(new_tokens=i32(3).long()), dict(block_table=i32(3, 4).long()), dict(block_table=i32(4, 3).T), dict(tokens=-1),
                   dict(page=0), dict(pages=1 << 31), dict(tokens=1 << 31), dict(free=i32(4, 4)), dict(free=None), dict(out={"slots": i32(5)}),
                   dict(out={"kv_len": i32(2)})):
        with pytest.raises(ValueError):
            place_call(**change)


def test_linear_attention_wrapper_refuses():
    for call, more in ((binding.ttc_linear_attention, {}), (binding.ttc_linear_attention_backward, dict(grad_out=torch.zeros(6, 4, 32)))):
        with pytest.raises(ValueError, match="on a GPU"):
            call(**linear_args(), **more)
        for change in (dict(q=torch.zeros(6, 2, 64).half()), dict(k=torch.zeros(6, 2, 32)), dict(k=torch.zeros(5, 2, 64)), dict(v=torch.zeros(6, 3, 32)),
                       dict(v=torch.zeros(5, 4, 32)), dict(v=torch.zeros(6, 4, 32).bfloat16()), dict(q=torch.zeros(6, 64, 2).transpose(1, 2)),
                       dict(log_decay=torch.zeros(6, 2)), dict(log_decay=torch.zeros(6, 4).double()), dict(max_q=None), dict(max_q=1 << 31),
                       dict(cu_q=torch.zeros(3)), dict(state=torch.zeros(3, 4, 64, 32)), dict(state=torch.zeros(2, 4, 64, 32).bfloat16()),
                       dict(state=torch.zeros(2, 4, 32, 64)), dict(state_row=i32(3)), dict(kv_len=i32(1)), dict(cu_q=i32(2, 2))):
            with pytest.raises(ValueError):
                call(**linear_args(**change), **more)
    for change in (dict(out={"out": torch.zeros(6, 4, 64)}), dict(out={"state": torch.zeros(1, 4, 64, 32)}), dict(want_state=True, state_row=i32(2))):
        with pytest.raises(ValueError):
            binding.ttc_linear_attention(**linear_args(), **change)
    for change in (dict(grad_out=torch.zeros(6, 4, 64)), dict(grad_out=torch.zeros(6, 4, 32).bfloat16()), dict(grad_state=torch.zeros(1, 4, 64, 32)),
                   dict(out={"gq": torch.zeros(6, 4, 64)}), dict(out={"glog_decay": torch.zeros(4)}), dict(log_decay=torch.zeros(4).expand(6, 4))):
        with pytest.raises(ValueError):
            binding.ttc_linear_attention_backward(**{**linear_args(), "grad_out": torch.zeros(6, 4, 32), **change})


def test_norm_wrapper_refuses():
    y, v = torch.zeros(3, 64), torch.zeros(64)
    for call, more in ((binding.ttc_residual_norm, {}), (binding.ttc_residual_norm_backward, dict(grad_h=y))):
        with pytest.raises(ValueError, match="on a GPU"):
            call(y, pre="rms", **more)
        for change in (dict(residual=y.bfloat16()), dict(gate=y[:2]), dict(gate=torch.zeros(64, 3).T), dict(activation="tanh", gate=y), dict(post="batch"),
                       dict(post_gain=v), dict(post="rms", post_gain=v.double()), dict(pre_gain=v[:3]), dict(residual_gain=y), dict(groups=1 << 31)):
            with pytest.raises(ValueError):
                call(y, pre="rms", **change, **more)
    with pytest.raises(ValueError):
        binding.ttc_residual_norm(y, out={"r": y.bfloat16()})
    for change in (dict(grad_h=y), dict(pre="rms"), dict(grad_r=y.bfloat16()), dict(out={"gy": y[:2]})):
        with pytest.raises(ValueError):
            binding.ttc_residual_norm_backward(y, **change)

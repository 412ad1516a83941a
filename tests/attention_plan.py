"""How ttc_attention shares a call out, asked of the host code that decides it (csrc/ttc_attention_plan.hpp), compiled by itself: tests ask which
kernel a case takes rather than repeat the rule."""
import ctypes
import functools
import os
import subprocess
import tempfile
from types import SimpleNamespace

from paper_2603_09221_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FIELDS = ("prompt", "shared", "workgroups", "entries", "items", "max_q", "max_kv", "workspace", "fits")
SOURCE = """
#include "ttc_attention_plan.hpp"
extern "C" void plan(const ttc_attention_t *a, int cus, long long *out) {
  ttc::AttentionArgs p;
  p.a = *a;
  const bool fits = ttc::plan_attention(p, cus);
  const long long no[] = {0, 0, 0, 0, 0, 0, 0, 0, 0},
                  v[] = {p.prompt, p.shared, p.workgroups, p.entries, p.items, p.a.max_q, p.a.max_kv, (long long)ttc::attention_workspace(p), 1};
  for (unsigned i = 0; i < sizeof v / sizeof *v; ++i) out[i] = fits ? v[i] : no[i];
}
"""


@functools.lru_cache(maxsize=None)
def _library():
    with tempfile.TemporaryDirectory() as folder:
        src, lib = os.path.join(folder, "plan.cpp"), os.path.join(folder, "plan.so")
        with open(src, "w") as f:
            f.write(SOURCE)
        subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2603_09221_amd", "csrc"), src, "-o", lib],
                       check=True)
        return ctypes.CDLL(lib)


def plan(attention, cus=256):
    """The plan of a binding.Attention on a device of `cus` compute units: a namespace of FIELDS."""
    out = (ctypes.c_longlong * len(FIELDS))()
    _library().plan(ctypes.byref(attention), cus, out)
    return SimpleNamespace(**dict(zip(FIELDS, out)))


def describe(sequences, tokens, heads_q, heads, d, page, bf16, max_q, max_kv, window=0, causal=True, pages=1, cu_q=True):
    """The descriptor of a call, without its tensors."""
    a = binding.Attention(cache=binding.KvCache(None, pages, heads, d, page), sequences=sequences, tokens=tokens, heads_q=heads_q,
                          dtype=1 if bf16 else 0, causal=int(causal), window=window, scale=1.0, max_q=max_q, max_kv=max_kv)
    a.cu_q = 1 << 12 if cu_q else None      # (never read)
    return a

"""What the host decides about a call of ttc_attention before it is launched (csrc/ttc_attention_plan.hpp).  No GPU."""
import pytest

from tests.attention_plan import describe, plan


@pytest.mark.parametrize("new", [1, 600])
@pytest.mark.parametrize("bf16", [True, False])
def test_a_cache_without_pages_is_not_read(new, bf16):
    """Whatever the lengths and the table say: kv_len is read as at most max_kv, and a row that sees nothing reads no page."""
    call = dict(sequences=2, tokens=2 * new, heads_q=64, heads=8, d=64, page=16, bf16=bf16, max_q=new, max_kv=100000)
    p = plan(describe(**call, pages=0))
    assert p.max_kv == 0 and not p.shared and p.workspace == 0 and bool(p.prompt) == (new > 1)
    assert plan(describe(**call, pages=1)).max_kv == 100000

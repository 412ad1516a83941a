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


@pytest.mark.parametrize("bf16,group", [(True, 64), (True, 128), (False, 100)])
def test_a_bound_wider_than_the_one_row_that_each_sequence_has(bf16, group):
    """Without cu_q: the same plan as with max_q = 1, and workgroups for every sequence's tiles."""
    call = dict(sequences=384, tokens=384, heads_q=group, heads=1, d=64, page=16, bf16=bf16, max_kv=80, cu_q=False)
    one = plan(describe(**call, max_q=1))
    for max_q in (2, 4, 1000):
        assert plan(describe(**call, max_q=max_q)) == one
    assert one.workgroups >= 384 and one.entries == 384 * -(-group // (128 if one.prompt else 16))
    assert plan(describe(**call, max_q=0)).max_q == 0


@pytest.mark.parametrize("bf16", [True, False])
def test_a_long_bound_on_new_tokens_is_no_reason_to_refuse(bf16):
    """256 sequences, one with 32768 new tokens beside single ones; a bound far above what there is; and what no launch holds."""
    call = dict(heads_q=32, heads=8, d=64, page=64, bf16=bf16)
    p = plan(describe(sequences=256, tokens=32768 + 255, max_q=32768, max_kv=40000, **call))
    assert p.fits and p.prompt and 8 * (32768 * 4 // 128 + 255) <= p.workgroups < 1 << 24
    p = plan(describe(sequences=40, tokens=2000, max_q=1 << 19, max_kv=1 << 19, **call))
    assert p.fits and p.prompt and p.workgroups == 8 * (2000 * 4 // 128 + 40)
    for sequences, tokens, max_q, max_kv in ((1 << 24, 1 << 24, 1, 64), (1 << 40, 1 << 40, 1, 64), (1, 1 << 29, 1 << 29, 64), (1, 1, 1, (1 << 30) + 1),
                                             (1 << 20, 1 << 20, 1 << 20, 64), ((1 << 63) - 1, (1 << 63) - 1, 0, 0)):
        assert not plan(describe(sequences=sequences, tokens=tokens, max_q=max_q, max_kv=max_kv, **call)).fits

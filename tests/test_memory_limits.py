"""How many tokens, sequences and heads one call of linear attention takes: both sides of what the header states, by sizes alone."""
import pytest

from tests.test_memory_boundary import UNSUPPORTED, WORKSPACE, backward, lib, linear  # noqa: F401  (lib is a fixture)

WIDE = dict(dk=256, dv=256)


def answers(lib, **sizes):  # noqa: F811
    """What forward and gradients say to addresses that nobody reads and no workspace; a forward call needs one only where a sequence is cut."""
    size = {**dict(heads_qk=sizes["heads"], g_token=0, q_token=8, k_token=8, v_token=8, out_token=8), **sizes}
    a = linear(**size)
    taken = lib.ttc_linear_attention_workspace_bytes(a) > 0 if size["max_q"] > 16 else None
    return taken, lib.ttc_linear_attention_backward(backward(size), None, 0, None)


@pytest.mark.parametrize("sizes", [WIDE, dict(dk=8, dv=8)])
@pytest.mark.parametrize("heads,sequences,tokens", [(1, 1, ((1 << 23) - 10) * 64), (1, 100, ((1 << 23) - 109) * 64), (32, 1, ((1 << 18) - 10) * 64),
                                                    (1, (1 << 20) - 9, 1 << 20), (64, (1 << 14) - 9, 1 << 14)])
def test_what_is_always_taken(lib, sizes, heads, sequences, tokens):  # noqa: F811
    assert (tokens / 64 + sequences + 8) * heads < 1 << 23 and (sequences + 8) * heads < 1 << 20
    taken, back = answers(lib, heads=heads, sequences=sequences, tokens=tokens, max_q=-(-tokens // sequences), **sizes)
    assert taken in (True, None) and back == WORKSPACE


@pytest.mark.parametrize("heads,sequences,tokens", [(1, 1, ((1 << 23) - 9) * 64), (1, 100, ((1 << 23) - 108) * 64), (32, 1, ((1 << 18) - 9) * 64)])
def test_one_chunk_more(lib, heads, sequences, tokens):  # noqa: F811
    """The first bound is the limit itself."""
    assert (tokens / 64 + sequences + 8) * heads == 1 << 23
    taken, back = answers(lib, heads=heads, sequences=sequences, tokens=tokens, max_q=tokens, **WIDE)
    assert taken is False and back == UNSUPPORTED


def test_the_eight_sequences_more_count(lib):  # noqa: F811
    """One sequence of 64 tokens with 2^19 heads: one sequence's heads are few, nine sequences' are not."""
    size = dict(heads=1 << 19, heads_qk=1 << 19, sequences=1, tokens=64, max_q=64, g_token=0, q_token=8, k_token=8, v_token=8, out_token=8, **WIDE)
    assert lib.ttc_linear_attention(linear(**size), None, 0, None) == UNSUPPORTED

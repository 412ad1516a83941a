"""The oracle of memory layers against closed forms and differences.  No GPU."""
import numpy as np
import pytest

from oracle import memory_oracle as oracle


def inputs(seed=0, n=7, heads=4, heads_qk=2, dk=3, dv=5):
    rng = np.random.default_rng(seed)
    return (rng.standard_normal((n, heads_qk, dk)), rng.standard_normal((n, heads_qk, dk)), rng.standard_normal((n, heads, dv)),
            -rng.exponential(0.5, (n, heads)))


def test_linear_attention_as_a_sum_over_pairs():
    q, k, v, g = inputs()
    cu, first = [0, 3, 3, 7], np.random.default_rng(1).standard_normal((3, 4, 3, 5))
    out, last = oracle.linear_attention(q, k, v, g, cu, 0.3, first)
    for s in range(3):
        for h in range(4):
            for i in range(cu[s], cu[s + 1]):
                want = np.exp(g[cu[s]:i + 1, h].sum()) * (q[i, h // 2] @ first[s, h])
                for j in range(cu[s], i + 1):
                    want = want + np.exp(g[j + 1:i + 1, h].sum()) * (q[i, h // 2] @ k[j, h // 2]) * v[j, h]
                assert np.allclose(out[i, h], 0.3 * want, rtol=1e-12)
    assert np.array_equal(last[1], first[1])


def test_linear_attention_without_decay_and_with_all_of_it():
    q, k, v, g = inputs()
    out, last = oracle.linear_attention(q, k, v, 0 * g, [0, 7], 1.0)
    assert np.allclose(last[0, 1], sum(np.outer(k[t, 0], v[t, 1]) for t in range(7)))
    out, last = oracle.linear_attention(q, k, v, np.full_like(g, -np.inf), [0, 7], 1.0)
    assert np.allclose(out[5, 3], (q[5, 1] @ k[5, 1]) * v[5, 3])


def differences(f, x, step=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        up, down = x.copy(), x.copy()
        up[i] += step
        down[i] -= step
        g[i] = (f(up) - f(down)) / (2 * step)
    return g


def test_linear_attention_gradients_against_differences():
    q, k, v, g = inputs(2)
    cu, rng = [0, 3, 3, 7], np.random.default_rng(3)
    first, glast, gout = rng.standard_normal((3, 4, 3, 5)), rng.standard_normal((3, 4, 3, 5)), rng.standard_normal(v.shape)

    def loss(q=q, k=k, v=v, g=g, first=first):
        out, last = oracle.linear_attention(q, k, v, g, cu, 0.7, first)
        return (out * gout).sum() + (last * glast).sum()

    got = oracle.linear_attention_gradients(q, k, v, g, cu, 0.7, gout, first, glast)
    for name, x, have in zip(("q", "k", "v", "g", "first"), (q, k, v, g, first), got):
        assert np.allclose(differences(lambda y: loss(**{name: y}), x), have, rtol=1e-6, atol=1e-7), name


@pytest.mark.parametrize("post,pre,groups,activation", [("rms", "layer", 1, "silu"), ("layer", "rms", 3, "sigmoid"), (None, "rms", 1, "identity"),
                                                        ("layer", None, 2, "silu")])
def test_norm_gradients_against_differences(post, pre, groups, activation):
    rng = np.random.default_rng(4)
    c = 6
    x = dict(y=rng.standard_normal((3, c)), residual=rng.standard_normal((3, c)), gate=rng.standard_normal((3, c)), residual_gain=rng.standard_normal(c))
    if post:
        x.update(post_gain=rng.standard_normal(c), post_offset=rng.standard_normal(c))
    if pre:
        x.update(pre_gain=rng.standard_normal(c), pre_offset=rng.standard_normal(c))
    kw = dict(activation=activation, post=post, groups=groups, scale=0.7, pre=pre)
    gr, gh = rng.standard_normal((3, c)), rng.standard_normal((3, c)) if pre else None

    def loss(**change):
        r, h = oracle.residual_norm(**{**x, **change}, **kw)
        return (r * gr).sum() + (0.0 if h is None else (h * gh).sum())

    got = oracle.residual_norm(**x, **kw, gr=gr, gh=gh)
    for name in x:
        assert np.allclose(differences(lambda t: loss(**{name: t}), x[name]), got["g" + name], rtol=1e-5, atol=1e-6), name


def test_norms_closed_forms():
    r, h = oracle.residual_norm(np.array([[3.0, 4.0]]), post="rms", pre="layer", eps=0.0)
    assert np.allclose(r, np.array([[3.0, 4.0]]) / np.sqrt(12.5)) and np.allclose(h, [[-1.0, 1.0]])
    r, h = oracle.residual_norm(np.array([[1.0, 3.0, 10.0, 30.0]]), post="layer", groups=2, eps=0.0, residual=np.ones((1, 4)), scale=2.0)
    assert np.allclose(r, [[-1.0, 3.0, -1.0, 3.0]]) and h is None


def test_places_by_hand():
    """Two pages of four tokens there, one needed by the first sequence, one given back by the second; the third lacks one."""
    table = np.array([[7, -1, -1], [5, 6, -1], [1, -1, -1]])
    got = oracle.place([3, 8, 4], [2, -1, 9], table, 4, 13, 10, free=[9, 0, 0, 0], count=1)
    assert list(got["cu_q"]) == [0, 2, 2, 11] and list(got["kv_len"]) == [5, 0, 13]
    assert list(got["sequence"]) == [0, 0] + [2] * 9 + [-1, -1]
    assert got["table"].tolist() == [[7, 6, -1], [5, 6, -1], [1, 5, 9]] and got["free_count"] == 0 and got["missing"] == 0
    assert list(got["slots"]) == [31, 24, 20, 21, 22, 23, 36, 37, 38, 39, -1, -1, -1]
    assert list(got["positions"]) == [3, 4, 4, 5, 6, 7, 8, 9, 10, 11, 12, 0, 0]

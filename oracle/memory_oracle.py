"""CPU float64 oracle of memory layers: linear attention with decays and its gradients, the norms around a block and theirs, the places of
new tokens in a paged cache.  Plain numpy from the definitions, token by token; shares no code with the GPU path."""
import numpy as np


def linear_attention(q, k, v, g, cu, scale, first=None):
    """out (n, heads, dv) and the sequences' last states; q, k (n, heads_qk, dk), v (n, heads, dv), g (n, heads), first (sequences, heads, dk, dv)."""
    heads, dk, dv = v.shape[1], q.shape[2], v.shape[2]
    group = heads // q.shape[1]
    q, k = np.repeat(q, group, 1), np.repeat(k, group, 1)
    out = np.zeros(v.shape)
    last = np.zeros((len(cu) - 1, heads, dk, dv))
    for s in range(len(cu) - 1):
        state = np.zeros((heads, dk, dv)) if first is None else np.array(first[s], dtype=np.float64)
        for t in range(cu[s], cu[s + 1]):
            state = np.exp(g[t])[:, None, None] * state + k[t][:, :, None] * v[t][:, None, :]
            out[t] = scale * np.einsum("hd,hde->he", q[t], state)
        last[s] = state
    return out, last


def linear_attention_gradients(q, k, v, g, cu, scale, gout, first=None, glast=None):
    """gq, gk (n, heads_qk, dk), gv, gg (n, heads), gfirst of the loss sum(gout * out) + sum(glast * last)."""
    heads_qk, heads, dk, dv = q.shape[1], v.shape[1], q.shape[2], v.shape[2]
    group = heads // heads_qk
    q, k = np.repeat(q, group, 1), np.repeat(k, group, 1)
    gq, gk, gv, gg = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape), np.zeros(g.shape)
    gfirst = np.zeros((len(cu) - 1, heads, dk, dv))
    for s in range(len(cu) - 1):
        states = [np.zeros((heads, dk, dv)) if first is None else np.array(first[s], dtype=np.float64)]
        for t in range(cu[s], cu[s + 1]):
            states.append(np.exp(g[t])[:, None, None] * states[-1] + k[t][:, :, None] * v[t][:, None, :])
        back = np.zeros((heads, dk, dv)) if glast is None else np.array(glast[s], dtype=np.float64)
        for t in reversed(range(cu[s], cu[s + 1])):
            now, before = states[t - cu[s] + 1], states[t - cu[s]]
            gq[t] = scale * np.einsum("hde,he->hd", now, gout[t])
            back = back + scale * q[t][:, :, None] * gout[t][:, None, :]
            gk[t] = np.einsum("hde,he->hd", back, v[t])
            gv[t] = np.einsum("hde,hd->he", back, k[t])
            back = np.exp(g[t])[:, None, None] * back
            gg[t] = (back * before).sum((1, 2))
        gfirst[s] = back
    n = len(q)
    return gq.reshape(n, heads_qk, group, dk).sum(2), gk.reshape(n, heads_qk, group, dk).sum(2), gv, gg, gfirst


def _unit(x, kind, eps, groups):
    """Normalised entries by groups of the last axis, and the factor that they were multiplied by."""
    y = x.reshape(*x.shape[:-1], groups, -1)
    if kind == "layer":
        y = y - y.mean(-1, keepdims=True)
    inverse = 1.0 / np.sqrt((y ** 2).mean(-1, keepdims=True) + eps)
    return (y * inverse).reshape(x.shape), np.broadcast_to(inverse, y.shape).reshape(x.shape)


def _unit_gradient(g, unit, inverse, kind, groups):
    shape = (*g.shape[:-1], groups, -1)
    g, unit, inverse = (x.reshape(shape) for x in (g, unit, inverse))
    mean = g.mean(-1, keepdims=True) if kind == "layer" else 0.0
    return (inverse * (g - mean - unit * (g * unit).mean(-1, keepdims=True))).reshape(*g.shape[:-2], -1)


def act(x, activation):
    """The gate's factor and its derivative."""
    s = 1.0 / (1.0 + np.exp(-x))
    return {"identity": (x, np.ones_like(x)), "sigmoid": (s, s * (1 - s)), "silu": (x * s, s + x * s * (1 - s))}[activation]


def residual_norm(y, residual=None, gate=None, activation="silu", post=None, post_gain=None, post_offset=None, groups=1, scale=1.0,
                  residual_gain=None, pre=None, pre_gain=None, pre_offset=None, eps=1e-5, gr=None, gh=None):
    """(r, h), or with a gradient gr (and gh) a dict of the gradients."""
    c = y.shape[1]
    one = np.ones(c)
    gain, by = one if post_gain is None else post_gain, scale * (one if residual_gain is None else residual_gain)
    unit, inverse = _unit(y, post, eps, groups) if post else (y, None)
    z = unit * gain + (0.0 if post_offset is None else post_offset)
    a, slope = act(gate, activation) if gate is not None else (np.ones_like(y), None)
    r = by * a * z + (0.0 if residual is None else residual)
    unit_r, inverse_r = _unit(r, pre, eps, 1) if pre else (None, None)
    pg = one if pre_gain is None else pre_gain
    if gr is None:
        return r, None if not pre else unit_r * pg + (0.0 if pre_offset is None else pre_offset)
    total, out = np.array(gr), {}
    if pre:
        total = total + _unit_gradient(gh * pg, unit_r, inverse_r, pre, 1)
        out.update(gpre_gain=(gh * unit_r).sum(0), gpre_offset=gh.sum(0))
    gz = total * by * a
    out.update(gresidual=total, gresidual_gain=(total * scale * a * z).sum(0), gpost_gain=(gz * unit).sum(0), gpost_offset=gz.sum(0))
    out["gy"] = _unit_gradient(gz * gain, unit, inverse, post, groups) if post else gz * gain
    if gate is not None:
        out["ggate"] = total * by * z * slope
    return out


def place(past, new, table, page, tokens, pages, free=None, count=0, capacity=None):
    """Token by token: a dict of what ttc_kv_place gives, the table and the list as they are afterwards among it."""
    table, width = np.array(table), table.shape[1]
    past = [min(max(int(p), 0), (1 << 30) - 1) for p in past]
    cu = [0]
    for n in new:
        cu.append(min(cu[-1] + max(int(n), 0), tokens))
    needed = lambda n: min(-(-n // page), width)
    out, lacking = {}, 0
    if free is not None:
        free, count = list(int(f) for f in free), min(max(count, 0), len(free))
        for s, n in enumerate(new):
            if n < 0:
                for c in range(needed(past[s])):
                    if 0 <= table[s, c] < pages and count < len(free):
                        free[count] = int(table[s, c])
                        count += 1
        for s, n in enumerate(new):
            if n >= 0:
                for c in range(needed(past[s]), needed(past[s] + cu[s + 1] - cu[s])):
                    if count:
                        count -= 1
                        table[s, c] = free[count]
                    else:
                        table[s, c] = -1
                        lacking += 1
        out.update(free=np.array(free), free_count=count, missing=lacking)
    positions, slots, sequence = np.zeros(tokens, dtype=np.int64), np.full(tokens, -1, dtype=np.int64), np.full(tokens, -1)
    for s in range(len(new)):
        for t in range(cu[s], cu[s + 1]):
            p = past[s] + t - cu[s]
            positions[t], sequence[t] = p, s
            if p // page < width and 0 <= table[s, p // page] < pages:
                slots[t] = int(table[s, p // page]) * page + p % page
    kv = [0 if n < 0 else p + cu[s + 1] - cu[s] for s, (p, n) in enumerate(zip(past, new))]
    return dict(out, cu_q=np.array(cu), kv_len=np.array(kv), positions=positions, slots=slots, sequence=sequence, table=table)

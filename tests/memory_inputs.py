"""Inputs of the tests of memory layers, made on the host from a seed, and the sizes that their tolerances count with."""
import numpy as np
import torch

DEV = "cuda:0"
U = 2.0 ** -24          # half a step of float32, of a number of 1
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}


def host(t):
    return t.detach().cpu().double().numpy()


def attention_inputs(lengths, heads, heads_qk, dk, dv, dtype, constant=False, seed=0, rate=None):
    """q, k, v, log_decay, cu_q on the GPU; keys of length about 1, decays from a head that remembers to one that forgets within a token."""
    gen = torch.Generator().manual_seed(seed)
    n = sum(lengths)
    q, v = torch.randn((n, heads_qk, dk), generator=gen), torch.randn((n, heads, dv), generator=gen)
    k = torch.randn((n, heads_qk, dk), generator=gen) * dk ** -0.5
    rates = torch.exp(-6.0 * torch.arange(heads) / max(1, heads - 1)) if rate is None else torch.full((heads,), rate)
    g = -rates if constant else -rates * 2.0 * torch.rand((n, heads), generator=gen)
    cu = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    return q.to(dtype).to(DEV), k.to(dtype).to(DEV), v.to(dtype).to(DEV), g.to(DEV), torch.from_numpy(cu).to(DEV)


def decays(g, n):
    """log decays as (n, heads) float64 on the host"""
    g = host(g)
    return np.broadcast_to(g, (n, g.shape[-1])) if g.ndim == 1 else g


def attention_roundings(dk, length):
    """Roundings to float32 that a result may pass: the sum over a key's entries, that over a chunk's tokens, the weight (an exponential, 4, of
    a difference, 2, and two factors), for each chunk the state's factor and sum; every one is half a step of a partial sum of magnitudes."""
    return dk + 64 + 8 + (length // 64 + 1) * (64 + 6)

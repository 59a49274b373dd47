"""The operators of a sequence model that learns from a larger one, in 64 bits on the CPU: scaled embedding, gated delta rule, loss against a teacher's top logits.

Written from the definitions, a step at a time, in differentiable torch operations: gradients are torch's."""
import math

import torch

EPS = 1e-6


def embedding(tokens, table, scale=1.0, pad=None):
    """Rows of tokens outside the table are NaN, those of the padding token zeros."""
    V = table.shape[0]
    inside = (tokens >= 0) & (tokens < V)
    out = scale * table[tokens.clamp(0, V - 1)]
    if pad is not None:
        out = torch.where((tokens == pad)[:, None], torch.zeros_like(out), out)
    return torch.where(inside[:, None], out, torch.full_like(out, math.nan))


def embedding_gradient(tokens, dout, V, scale=1.0, pad=None):
    out = torch.zeros((V, dout.shape[1]), dtype=torch.float64)
    for i, v in enumerate(tokens.tolist()):
        if 0 <= v < V and v != pad:
            out[v] += scale * dout[i]
    return out


def inverse_lengths(gi, heads):
    """1 / sqrt(D (|q|^2 + e)) and 1 / sqrt(|k|^2 + e) of rows gi [..,W]: two of [..,Hk,1]."""
    _, Hk, D, _ = heads
    q, k = (gi[..., i * Hk * D:(i + 1) * Hk * D].unflatten(-1, (Hk, D)) for i in (0, 1))
    return 1 / torch.sqrt(D * ((q * q).sum(-1, keepdim=True) + EPS)), 1 / torch.sqrt((k * k).sum(-1, keepdim=True) + EPS)


def _parts(gi, heads, normalised=False):
    H, Hk, D, Dv = heads
    q, k, v, a, b = gi.split([Hk * D, Hk * D, H * Dv, H, H], dim=-1)
    rows = lambda x, n: x.reshape(*x.shape[:-1], n, -1)
    q, k = rows(q, Hk), rows(k, Hk)
    if not normalised:
        iq, ik = inverse_lengths(gi, heads)
        q, k = q * iq, k * ik
    shared = lambda x: x.repeat_interleave(H // Hk, dim=-2)
    return shared(q), shared(k), rows(v, H), a, b


def delta_step(gi, S, heads, bias=None, normalised=False):
    """One step: gi [N,W], S [N,H,D,Dv] -> (o [N,H*Dv], S).  normalised: gi holds queries and keys as they are after that."""
    H = heads[0]
    q, k, v, a, b = _parts(gi, heads, normalised)
    if bias is not None:
        a, b = a + bias[:H], b + bias[H:]
    S = torch.sigmoid(a)[..., None, None] * S
    u = torch.sigmoid(b)[..., None] * (v - torch.einsum("nhdv,nhd->nhv", S, k))
    S = S + k[..., None] * u[..., None, :]
    return torch.einsum("nhdv,nhd->nhv", S, q).flatten(1), S


def delta(gi, heads, bias=None, h0=None, lengths=None, normalised=False):
    """gi [T,N,W] -> (o [T,N,H*Dv], the last state, the states in front of every 64th step).  Rows behind a sequence's end are not looked at."""
    T, N, _ = gi.shape
    H, _, D, Dv = heads
    S = torch.zeros((N, H, D, Dv), dtype=gi.dtype) if h0 is None else h0
    live = torch.ones((T, N), dtype=torch.bool) if lengths is None else torch.arange(T)[:, None] < lengths
    gi = torch.where(live[..., None], gi, torch.zeros_like(gi))
    out, saved = [], []
    for t in range(T):
        if t % 64 == 0:
            saved.append(S)
        o, after = delta_step(gi[t], S, heads, bias, normalised)
        S = torch.where(live[t][:, None, None, None], after, S)
        out.append(torch.where(live[t][:, None], o, torch.zeros_like(o)))
    return torch.stack(out), S, torch.stack(saved)


def distill_rows(logits, index, teacher, tau=1.0):
    """Each row's loss.  Places of a negative index are none; a row without any has none."""
    there = index >= 0
    some = there.any(1, keepdim=True)
    t = torch.where(there, teacher / tau, torch.full_like(teacher, -math.inf))
    p = torch.softmax(torch.where(some, t, torch.zeros_like(t)), 1)
    logq = torch.log_softmax(logits / tau, 1).gather(1, index.clamp(min=0).long())
    counts = there & (p > 0)
    q = torch.where(counts, logq, torch.zeros_like(logq))
    return tau * tau * torch.where(counts, p * (torch.where(counts, p, torch.ones_like(p)).log() - q), torch.zeros_like(p)).sum(1)


def distill(logits, index, teacher, tau=1.0, weights=None):
    """(loss, each row's): rows of weight 0 are not looked at."""
    if weights is None:
        weights = torch.ones(logits.shape[0], dtype=logits.dtype)
    used = (weights != 0) & (index >= 0).any(1)
    rows = torch.zeros(logits.shape[0], dtype=logits.dtype)
    if bool(used.any()):
        rows = rows.index_put((used.nonzero()[:, 0],), distill_rows(logits[used], index[used], teacher[used], tau))
    total = weights.sum()
    return (rows * weights).sum() / (total if float(total) else 1.0), rows

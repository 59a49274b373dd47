"""Oracle for the sequence models: layer norm with its residual add, the gated linear recurrence, AdamW with 8-bit moments.

TEST INFRASTRUCTURE ONLY (see the package docstring): plain numpy, one definition per function, steps in a Python loop, no fusion.  Layer
norm and the recurrence are float64; the optimizer step also exists in float32, operation by operation as include/nsk.h writes it, since
what a moment is rounded to depends on its last bit.
"""
from __future__ import annotations

import numpy as np

STRETCH, BLOCK = 16, 256


def _f64(a):
    return np.asarray(a, dtype=np.float64)


def sigmoid(a):
    """Of both signs without overflow."""
    e = np.exp(-np.abs(a))
    return np.where(a >= 0, 1, e) / (1 + e)


# ----------------------------------------------------------------------------- layer norm

def layernorm_fwd(s, gamma, beta, eps):
    """(y, mean, invstd) of rows s [rows, C]."""
    s = _f64(s)
    mean = s.mean(axis=1)
    invstd = 1 / np.sqrt(((s - mean[:, None]) ** 2).mean(axis=1) + eps)
    return (s - mean[:, None]) * invstd[:, None] * _f64(gamma) + _f64(beta), mean, invstd


def layernorm_bwd(dy, s, gamma, mean, invstd, dsum=None):
    """(dx, dgamma, dbeta)."""
    dy, s, mean, invstd = _f64(dy), _f64(s), _f64(mean)[:, None], _f64(invstd)[:, None]
    xh, gh = (s - mean) * invstd, dy * _f64(gamma)
    dx = invstd * (gh - gh.mean(axis=1, keepdims=True) - xh * (gh * xh).mean(axis=1, keepdims=True))
    return dx if dsum is None else dx + _f64(dsum), (dy * xh).sum(axis=0), dy.sum(axis=0)


# ----------------------------------------------------------------------------- gated linear recurrence

def glr_gates(gi, bias):
    """(f, 1 - f, c, o, 1 - o)."""
    H = gi.shape[-1] // 3
    a = _f64(gi) + (0 if bias is None else _f64(bias))
    f, c, o = a[..., :H], a[..., H:2 * H], a[..., 2 * H:]
    return sigmoid(f), sigmoid(-f), c, sigmoid(o), sigmoid(-o)


def glr_fwd(gi, bias, h0, lengths=None):
    """gi [T,N,3H] -> (y, states [T+1,N,H]): states[t] enters step t."""
    T, N, H = gi.shape[0], gi.shape[1], gi.shape[2] // 3
    h = np.zeros((N, H)) if h0 is None else _f64(h0)
    y, states = np.zeros((T, N, H)), [h]
    for t in range(T):
        live = np.ones(N, bool) if lengths is None else np.asarray(lengths) > t
        f, keep, c, o, _ = glr_gates(gi[t][live], bias)
        h = h.copy()
        h[live] = f * h[live] + keep * c
        y[t][live] = o * h[live]
        states.append(h)
    return y, np.stack(states)


def glr_bwd(gi, bias, states, dy, dh_last, lengths=None):
    """(dgi, dh0)."""
    T, N, H = gi.shape[0], gi.shape[1], gi.shape[2] // 3
    G = np.zeros((N, H)) if dh_last is None else _f64(dh_last).copy()
    dgi = np.zeros(gi.shape)
    for t in reversed(range(T)):
        live = np.ones(N, bool) if lengths is None else np.asarray(lengths) > t
        f, keep, c, o, shut = glr_gates(gi[t][live], bias)
        up = np.zeros_like(f) if dy is None else _f64(dy[t][live])
        g = G[live] + up * o
        dgi[t][live] = np.concatenate((g * (states[t][live] - c) * f * keep, g * keep, up * states[t + 1][live] * o * shut), axis=-1)
        G[live] = g * f
    return dgi, G


# ----------------------------------------------------------------------------- AdamW with 8-bit moments

def mix(x):
    x = np.asarray(x, dtype=np.uint64) & np.uint64(0xFFFFFFFF)
    low = np.uint64(0xFFFFFFFF)
    x = ((x ^ (x >> np.uint64(16))) * np.uint64(0x243F6A89)) & low
    x = ((x ^ (x >> np.uint64(15))) * np.uint64(0xB7E15163)) & low
    return x ^ (x >> np.uint64(16))


def random_bits(n, seed, index):
    """The 32 bits of each element of the index-th tensor."""
    i = np.arange(n, dtype=np.uint64)
    return mix(i * np.uint64(0x9E3779B9) + (i >> np.uint64(32)) * np.uint64(0x85A308D3) + mix((seed + index * 0x9E3779B9) & 0xFFFFFFFF))


def e4m3_values():
    """The value of each of the 256 codes."""
    code = np.arange(256)
    exponent, mantissa = (code >> 3) & 15, code & 7
    v = np.where(exponent == 0, mantissa * 2.0 ** -9, (1 + mantissa / 8) * 2.0 ** (exponent - 7.0))
    v[(code & 127) == 127] = np.nan
    return np.where(code >= 128, -v, v)


def block_scales(x):
    """The power of two of each block of 256 elements of x, by its largest finite magnitude."""
    x = np.where(np.isfinite(x), np.abs(x), 0)
    top = np.array([x[k:k + BLOCK].max() for k in range(0, x.size, BLOCK)], dtype=np.float64)
    mantissa, exponent = np.frexp(top)              # top = mantissa * 2^exponent, mantissa in [0.5, 1)
    return 2.0 ** np.maximum(np.where(top > 0, exponent - 9 + (mantissa > 0.875), -126), -126)


def held(x, scales, u16):
    """The e4m3 values (as numbers) for magnitudes x, float32: up where the part below the last place and u16 / 65536 of a place make a whole one."""
    y = np.abs(x).astype(np.float64) / np.repeat(scales, BLOCK)[:x.size]
    with np.errstate(invalid="ignore"):
        y32 = np.where(y < 2.0 ** -6, (y.astype(np.float32) + np.float32(2.0 ** -6)), y.astype(np.float32)).astype(np.float64)    # (rounded once, as a float)
        step = np.where(y < 2.0 ** -6, 2.0 ** -9, 2.0 ** (np.floor(np.log2(np.maximum(y, 2.0 ** -6))) - 3))
        q = np.floor(y32 / step + u16 / 65536.0) * step - np.where(y < 2.0 ** -6, 2.0 ** -6, 0)
    return np.where(np.isfinite(x), np.copysign(q, x), np.nan)


def adamw8_step(w, grad, m, r, scale_m, scale_r, step, seed, index, lr, beta1, beta2, eps, weight_decay, grad_scale=1.0, real=np.float32):
    """m, r: e4m3 values as numbers.  Returns (w, m, r, scale_m, scale_r, m and r before they are rounded), computed in `real`."""
    one, b1, b2 = np.float32(1), np.float32(beta1), np.float32(beta2)
    spread = lambda s: np.repeat(np.asarray(s, real), BLOCK)[:w.size]
    c1, c2 = real(1 / (1 - float(b1) ** step)), real(np.sqrt(1 / (1 - float(b2) ** step)))
    with np.errstate(all="ignore"):
        g = np.asarray(grad, real) * real(np.float32(grad_scale))
        mo, ro = np.asarray(m, real) * spread(scale_m), np.asarray(r, real) * spread(scale_r)
        mn = mo * real(b1) + g * real(one - b1)
        rn = np.sqrt(ro * ro * real(b2) + g * g * real(one - b2))
        wn = np.asarray(w, real) * real(one - np.float32(lr) * np.float32(weight_decay)) - real(np.float32(lr)) * (mn * c1 / (rn * c2 + real(np.float32(eps))))
    bits = random_bits(w.size, seed, index)
    sm, sr = block_scales(mn), block_scales(rn)
    qm, qr = held(mn, sm, (bits & np.uint64(0xFFFF)).astype(np.float64)), held(rn, sr, (bits >> np.uint64(16)).astype(np.float64))
    qr = np.where((rn > 0) & (qr < 2.0 ** -9), 2.0 ** -9, qr)
    return wn, qm, qr, sm, sr, mn, rn


# ----------------------------------------------------------------------------- the classifier made of them

def classifier_step(tokens, labels, p, lengths=None, eps=1e-5):
    """Loss, logits, final states of each block and gradients of the classifier in paper_2409_11600_amd/linear_recurrent.py, whose parameter names these are."""
    from . import gru, train
    T, N = tokens.shape
    L = sum(1 for k in p if k.startswith("w_in"))
    rows = lambda a: a.reshape(T * N, -1)
    s, u, gi, y, states, norms = [], [], [], [], [], []
    stream = gru.embedding_fwd(tokens.reshape(-1), p["table"])
    for k in range(L):
        s.append(stream)
        un, mean, invstd = layernorm_fwd(stream, p[f"gamma{k}"], p[f"beta{k}"], eps)
        u.append(un)
        norms.append((mean, invstd))
        gi.append((un @ _f64(p[f"w_in{k}"]).T).reshape(T, N, -1))
        yk, st = glr_fwd(gi[k], p[f"b_in{k}"], None, lengths)
        y.append(yk)
        states.append(st)
        if k < L - 1:
            stream = stream + rows(yk) @ _f64(p[f"w_out{k}"]).T
    z, zm, zi = layernorm_fwd(states[-1][-1], p["gamma"], p["beta"], eps)
    logits = train.linear_fwd(z, p["w_cls"], p["b_cls"])
    loss, _ = train.softmax_xent_fwd(logits, labels)
    dlogits = train.softmax_xent_bwd(logits, labels)
    g = {}
    g["w_cls"], g["b_cls"] = train.linear_wgrad(z, dlogits)
    dh, g["gamma"], g["beta"] = layernorm_bwd(train.linear_dgrad(dlogits, p["w_cls"]), states[-1][-1], p["gamma"], zm, zi)
    ds = None
    for k in reversed(range(L)):
        dy = None
        if k < L - 1:
            g[f"w_out{k}"] = ds.T @ rows(y[k])
            dy = (ds @ _f64(p[f"w_out{k}"])).reshape(T, N, -1)
        dgi, _ = glr_bwd(gi[k], p[f"b_in{k}"], states[k], dy, dh if k == L - 1 else None, lengths)
        g[f"w_in{k}"], g[f"b_in{k}"] = rows(dgi).T @ u[k], dgi.sum(axis=(0, 1))
        ds, g[f"gamma{k}"], g[f"beta{k}"] = layernorm_bwd(rows(dgi) @ _f64(p[f"w_in{k}"]), s[k], p[f"gamma{k}"], *norms[k], dsum=ds)
    g["table"] = gru.embedding_bwd(tokens.reshape(-1), ds, p["table"].shape[0])
    return loss, logits, [st[-1] for st in states], g

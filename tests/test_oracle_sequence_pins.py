"""Pins of the oracle for the sequence models (CPU): torch's float64 arithmetic with autograd, central differences, closed forms."""
import numpy as np
import pytest
import torch

from oracle import sequence as S


def rng(seed):
    return np.random.default_rng(seed)


def differences(f, x, h=1e-6):
    """Central differences of the number f(x)."""
    g = np.zeros(x.shape)
    for i in np.ndindex(*x.shape):
        up, down = x.copy(), x.copy()
        up[i] += h
        down[i] -= h
        g[i] = (f(up) - f(down)) / (2 * h)
    return g


@pytest.mark.parametrize("rows,C", [(1, 1), (1, 7), (5, 2), (4, 33)])
def test_layer_norm_against_torch_and_differences(rows, C):
    r = rng(rows * 100 + C)
    s, gamma, beta, dy = r.normal(size=(rows, C)), r.normal(size=C), r.normal(size=C), r.normal(size=(rows, C))
    y, mean, invstd = S.layernorm_fwd(s, gamma, beta, 1e-5)
    ts, tg, tb = (torch.tensor(a, requires_grad=True) for a in (s, gamma, beta))
    ty = torch.nn.functional.layer_norm(ts, (C,), tg, tb, 1e-5)
    ty.backward(torch.tensor(dy))
    dx, dgamma, dbeta = S.layernorm_bwd(dy, s, gamma, mean, invstd)
    for got, want in ((y, ty.detach()), (dx, ts.grad), (dgamma, tg.grad), (dbeta, tb.grad)):
        assert np.abs(got - want.numpy()).max() <= 1e-9 * (1 + np.abs(want.numpy()).max())
    loss = lambda a: float((S.layernorm_fwd(a, gamma, beta, 1e-5)[0] * dy).sum())
    if C > 1:       # (one column: y is beta whatever s holds)
        assert np.abs(differences(loss, s) - dx).max() <= 1e-6 * (1 + np.abs(dx).max()) * max(1, invstd.max() ** 2)
    assert np.array_equal(S.layernorm_bwd(dy, s, gamma, mean, invstd, dsum=s)[0], dx + s)


@pytest.mark.parametrize("T,N,H,ragged", [(1, 1, 1, False), (5, 2, 3, False), (7, 4, 2, True)])
def test_recurrence_against_torch_and_differences(T, N, H, ragged):
    r = rng(T)
    gi, bias, h0, dy, dl = (r.normal(size=s) for s in ((T, N, 3 * H), (3 * H,), (N, H), (T, N, H), (N, H)))
    lengths = np.array([T, 0, 1, T // 2][:N]) if ragged else None
    y, states = S.glr_fwd(gi, bias, h0, lengths)
    tgi, tb, th = (torch.tensor(a, requires_grad=True) for a in (gi, bias, h0))
    h, out = th, []
    for t in range(T):
        a = tgi[t] + tb
        f, c, o = torch.sigmoid(a[:, :H]), a[:, H:2 * H], torch.sigmoid(a[:, 2 * H:])
        live = torch.tensor(np.ones(N, bool) if lengths is None else lengths > t)[:, None]
        h = torch.where(live, f * h + (1 - f) * c, h)
        out.append(torch.where(live, o * h, torch.zeros_like(h)))
    (torch.stack(out) * torch.tensor(dy)).sum().add((h * torch.tensor(dl)).sum()).backward()
    dgi, dh0 = S.glr_bwd(gi, bias, states, dy, dl, lengths)
    for got, want in ((y, torch.stack(out).detach()), (states[-1], h.detach()), (dgi, tgi.grad), (dh0, th.grad), (dgi.sum((0, 1)), tb.grad)):
        assert np.abs(got - want.numpy()).max() <= 1e-12

    def loss(g, b, s):
        yy, st = S.glr_fwd(g, b, s, lengths)
        return float((yy * dy).sum() + (st[-1] * dl).sum())
    assert np.abs(differences(lambda a: loss(a, bias, h0), gi) - dgi).max() <= 1e-8
    assert np.abs(differences(lambda a: loss(gi, bias, a), h0) - dh0).max() <= 1e-8


def test_recurrence_of_steps_that_are_not_there():
    """What lies behind a sequence's end is not used, whatever it holds."""
    gi = rng(3).normal(size=(6, 3, 6))
    lengths = np.array([6, 0, 2])
    y, states = S.glr_fwd(gi, None, None, lengths)
    bad = gi.copy()
    bad[2:, 2] = np.nan
    bad[:, 1] = np.inf
    y2, states2 = S.glr_fwd(bad, None, None, lengths)
    assert np.array_equal(y, y2) and np.array_equal(states, states2) and not y[2:, 2].any() and not y[:, 1].any()
    assert np.array_equal(S.glr_bwd(gi, None, states, y, None, lengths)[0], S.glr_bwd(bad, None, states, y, None, lengths)[0])


def test_e4m3_values_are_torchs():
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(S.e4m3_values(), want, equal_nan=True)


def test_scales():
    for top, want in ((448.0, 1.0), (np.nextafter(np.float32(448), np.float32(500)), 2.0), (224.0, 0.5), (225.0, 1.0), (0.0, 2.0 ** -126), (1e-40, 2.0 ** -126)):
        assert S.block_scales(np.array([0, top, -top / 2], np.float32)) == want
    assert S.block_scales(np.array([np.inf, np.nan, 300], np.float32)) == 1.0


def test_held_values_are_neighbours_with_the_right_mean():
    values = np.sort(S.e4m3_values()[:127])
    x = np.concatenate((rng(1).uniform(0, 448, 200), 10.0 ** rng(2).uniform(-4, 2.6, 200), [0, 448, 2.0 ** -6, 2.0 ** -9])).astype(np.float32)
    scales = np.ones(-(-x.size // S.BLOCK))
    below = values[np.searchsorted(values, x, side="right") - 1]
    above = values[np.minimum(np.searchsorted(values, x, side="left"), values.size - 1)]
    every = [S.held(x, scales, u) for u in range(0, 65536, 64)]
    for q in every:
        assert ((q == below) | (q == above)).all()
    mean, place = np.mean(every, axis=0), np.maximum(above - below, 1e-30)
    assert (np.abs(mean - x) <= (1 / 1024 + 2.0 ** -12) * place + 1e-9).all()


def test_random_bits_are_even_and_independent():
    n = 1 << 18
    u = S.random_bits(n, 77, 0)
    for shift in (0, 16):
        counts = np.bincount(((u >> np.uint64(shift)) & np.uint64(0xFF)).astype(int), minlength=256)
        chi = ((counts - n / 256) ** 2 / (n / 256)).sum()
        assert abs(chi - 255) <= 6 * np.sqrt(2 * 255)
    bound = 6 / np.sqrt(n)
    low, high = (u & np.uint64(0xFFFF)).astype(float), (u >> np.uint64(16)).astype(float)
    others = [high, np.roll(low, 1), np.roll(low, 256)] + [(S.random_bits(n, s, k) & np.uint64(0xFFFF)).astype(float) for s, k in ((78, 0), (77, 1))]
    assert all(abs(np.corrcoef(low, o)[0, 1]) <= bound for o in others)


def test_optimizer_step_of_both_precisions():
    """The float32 step against 64 bits, and a first step in closed form: every weight moves by lr * sign(g)."""
    r = rng(5)
    n = 700
    w, g = r.normal(size=n).astype(np.float32), r.normal(size=n).astype(np.float32)
    zero, scales = np.zeros(n), np.zeros(3)
    first = S.adamw8_step(w, g, zero, zero, scales, scales, 1, 9, 0, 1e-3, 0.9, 0.999, 1e-8, 0.0)
    assert np.abs(first[0] - (w - np.float32(1e-3) * np.sign(g))).max() <= 1e-6
    a = S.adamw8_step(w, g, first[1], first[2], first[3], first[4], 2, 10, 0, 1e-3, 0.9, 0.999, 1e-8, 1e-2, 0.5)
    b = S.adamw8_step(w, g, first[1], first[2], first[3], first[4], 2, 10, 0, 1e-3, 0.9, 0.999, 1e-8, 1e-2, 0.5, real=np.float64)
    assert np.abs(a[0] - b[0]).max() <= 1e-6 and np.array_equal(a[3], b[3]) and np.array_equal(a[4], b[4])
    assert np.mean(a[1] != b[1]) <= 0.01 and np.mean(a[2] != b[2]) <= 0.01


def test_classifier_gradients_against_differences():
    T, N, E, H, V, K, L = 4, 3, 5, 4, 7, 2, 2
    r = rng(31)
    tokens, labels, lengths = r.integers(0, V, (T, N)), r.integers(0, K, N), np.array([4, 1, 3])
    p = {"table": r.normal(size=(V, E)), "gamma": 1 + 0.1 * r.normal(size=H), "beta": 0.1 * r.normal(size=H), "w_cls": r.normal(size=(K, H)), "b_cls": r.normal(size=K)}
    for k in range(L):
        p |= {f"gamma{k}": 1 + 0.1 * r.normal(size=E), f"beta{k}": 0.1 * r.normal(size=E), f"w_in{k}": r.normal(size=(3 * H, E)), f"b_in{k}": r.normal(size=3 * H)}
    p["w_out0"] = r.normal(size=(E, H))
    _, _, _, g = S.classifier_step(tokens, labels, p, lengths)
    assert set(g) == set(p)
    for name in p:
        d = differences(lambda a: float(S.classifier_step(tokens, labels, {**p, name: a}, lengths)[0]), p[name], 1e-5)
        assert np.abs(d - g[name]).max() <= 1e-6 * (1 + np.abs(g[name]).max()), name

"""What the 64-bit forms of oracle/learning.py are held to: closed forms, and differences for the gradients that torch makes of them."""
import math

import pytest
import torch

from oracle import learning as O


def _draw(*shape, seed=0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


def _differences(f, x, g, count=24, h=1e-6):
    """g against central differences of f, at `count` places of x: their error is h^2 / 6 of the third derivative and 2^-53 / h of the value, both far below 1e-6 of values of one."""
    flat, places = x.reshape(-1), torch.randperm(x.numel(), generator=torch.Generator().manual_seed(1))[:count]
    for i in places.tolist():
        at = flat[i].item()
        flat[i] = at + h
        up = f().item()
        flat[i] = at - h
        down = f().item()
        flat[i] = at
        assert abs((up - down) / (2 * h) - g.reshape(-1)[i].item()) < 1e-6


def test_embedding():
    tokens, table = torch.tensor([2, 0, 5, -1, 1, 2]), _draw(3, 4)
    out = O.embedding(tokens, table, 3.0, pad=1)
    assert torch.equal(out[0], 3 * table[2]) and torch.equal(out[1], 3 * table[0]) and out[2:4].isnan().all() and not out[4].any()
    w = _draw(6, 4)
    grad = O.embedding_gradient(tokens, w, 3, 3.0, pad=1)
    assert torch.allclose(grad, torch.stack((3 * w[1], 0 * w[0], 3 * (w[0] + w[5]))))


def test_delta_rule_recalls():
    """Unit keys at right angles, open gates: what was written under a key is read back with it; written again, it is replaced."""
    D, Dv, T = 4, 3, 5
    heads, v = (1, 1, D, Dv), _draw(T, Dv)
    key = [0, 1, 2, 0, 3]
    gi = torch.zeros((T, 1, 2 * D + Dv + 2), dtype=torch.float64)
    for t in range(T):
        gi[t, 0, key[t]] = gi[t, 0, D + key[t]] = 1e6
        gi[t, 0, 2 * D:2 * D + Dv] = v[t]
    gi[..., -2:] = 60.0                     # alpha = beta = 1 to 1e-26
    o, S, saved = O.delta(gi, heads)
    assert torch.allclose(o[:, 0] * math.sqrt(D), v, atol=1e-9)
    assert torch.allclose(S[0, 0], torch.stack((v[3], v[1], v[2], v[4])), atol=1e-9) and not saved[0].any()
    # half a step towards it, after half of what was there
    gi[..., -2:] = 0.0
    _, S, _ = O.delta(gi[:1], heads, h0=torch.ones((1, 1, D, Dv), dtype=torch.float64))
    assert torch.allclose(S[0, 0, 0], 0.5 + 0.5 * (v[0] - 0.5), atol=1e-9) and torch.allclose(S[0, 0, 1:], torch.tensor(0.5, dtype=torch.float64))


def test_delta_rule_lengths():
    heads, T, N = (2, 1, 3, 2), 70, 4
    gi, h0, lengths = _draw(T, N, 14), _draw(N, 2, 3, 2, seed=3), torch.tensor([0, 1, 66, 99])
    o, S, saved = O.delta(gi, heads, h0=h0, lengths=lengths)
    assert torch.equal(S[0], h0[0]) and not o[:, 0].any() and not o[1:, 1].any() and torch.equal(saved[1, 0], h0[0])
    for n, l in ((1, 1), (2, 66), (3, 70)):
        alone = O.delta(gi[:l, n:n + 1], heads, h0=h0[n:n + 1])
        assert torch.allclose(S[n], alone[1][0]) and torch.allclose(o[:l, n], alone[0][:, 0])
    gi[66:, 2] = math.nan
    assert torch.equal(O.delta(gi, heads, h0=h0, lengths=lengths)[1], S)


@pytest.mark.parametrize("which", ["gi", "h0", "bias"])
def test_delta_rule_differences(which):
    heads, T, N = (4, 2, 3, 2), 6, 2
    x = {"gi": _draw(T, N, 28), "h0": _draw(N, 4, 3, 2, seed=5), "bias": _draw(8, seed=6)}
    w, ws = _draw(T, N, 8, seed=7), _draw(N, 4, 3, 2, seed=8)

    def f():
        o, S, _ = O.delta(x["gi"], heads, x["bias"], x["h0"], torch.tensor([6, 4]))
        return (o * w).sum() + (S * ws).sum()

    x[which].requires_grad_(True)
    (g,) = torch.autograd.grad(f(), x[which])
    x[which] = x[which].detach()
    _differences(f, x[which], g)


def test_distill():
    z, t = _draw(4, 7), _draw(4, 3, seed=2)
    index = torch.tensor([[0, 3, 6], [1, -1, 4], [-1, -1, -1], [2, 2, 5]])
    tau = 2.0
    rows = O.distill_rows(z, index, t, tau)
    q = torch.softmax(z / tau, 1)
    p = torch.softmax(t[0] / tau, 0)
    assert torch.allclose(rows[0], 4 * (p * (p / q[0, [0, 3, 6]]).log()).sum())
    p = torch.softmax(t[1, [0, 2]] / tau, 0)
    assert torch.allclose(rows[1], 4 * (p * (p / q[1, [1, 4]]).log()).sum()) and rows[2] == 0
    # a teacher whose places are all and who says the same: nothing to learn
    whole = torch.arange(7).expand(4, 7)
    assert torch.allclose(O.distill_rows(z, whole, z, tau), torch.zeros(4, dtype=torch.float64), atol=1e-14)
    weights = torch.tensor([0.0, 2.0, 1.0, 1.0], dtype=torch.float64)
    bad = z.clone()
    bad[0] = math.nan
    assert torch.allclose(O.distill(bad, index, t, tau, weights)[0], (2 * rows[1] + rows[3]) / 4)
    assert O.distill(z, index, t, tau, 0 * weights)[0] == 0


def test_distill_differences():
    z, t, index, weights = _draw(3, 6), _draw(3, 4, seed=2), torch.tensor([[0, 3, 3, 5], [1, -1, 4, -1], [2, 1, 0, 5]]), torch.tensor([0.5, 2.0, 0.0], dtype=torch.float64)
    f = lambda: O.distill(z, index, t, 1.7, weights)[0]
    z.requires_grad_(True)
    (g,) = torch.autograd.grad(f(), z)
    z = z.detach()
    _differences(f, z, g)
    # tau (q - p), by hand
    q, p = torch.softmax(z / 1.7, 1), torch.zeros(6, dtype=torch.float64).index_add(0, index[0], torch.softmax(t[0] / 1.7, 0))
    assert torch.allclose(g[0], 0.2 * 1.7 * (q[0] - p)) and not g[2].any()

"""The gated linear recurrence on the GPU against the 64-bit oracle, on the values as stored.

Bounds, element by element, with u = 2^-24.  A gate's argument is rounded once (u of it), its exponential to 2 ulp more than its argument's error,
and two operations follow: each of f, 1 - f, o, 1 - o is off by at most (8 + 2|a|) u of itself.  A state is a sum of products of gates; with errors of K u in
each factor and operation, h_t = f h + (1 - f) c is off by err_t = f err_{t-1} + K u mag_t, mag the same recurrence of magnitudes, however the steps are
grouped (a product of n gates times a state has n of these errors, the recurrence counts them one by one).  Backwards likewise."""
import numpy as np
import pytest
import torch

from oracle import sequence as S
from paper_2409_11600_amd import binding as B
from parity import guarded, torch_dtype

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
# one step to many stretches, and channels that fill no wavefront, one, and several
SHAPES = [(1, 1, 1), (1, 3, 64), (2, 5, 7), (15, 2, 65), (16, 1, 130), (17, 4, 33), (33, 3, 128), (64, 2, 256), (100, 3, 201), (200, 5, 64), (257, 2, 96), (300, 1, 1),
          (513, 1, 40), (1000, 2, 24), (2049, 1, 66), (5000, 1, 32)]


def half(dtype):
    return torch.finfo(torch_dtype(dtype)).eps / 2


def host(t):
    return t.detach().double().cpu().numpy()


def make(seed, T, N, H, dtype, ragged):
    g = torch.Generator().manual_seed(seed)
    f = lambda *s: torch.randn(s, generator=g)
    gi, dy = f(T, N, 3 * H).to(torch_dtype(dtype)).cuda(), f(T, N, H).to(torch_dtype(dtype)).cuda()
    bias = torch.cat((1 + 2 * f(H), 0.3 * f(2 * H))).cuda()
    lengths = None
    if ragged:
        lengths = torch.randint(0, T + 1, (N,), generator=g, dtype=torch.int32)
        lengths[:3] = torch.tensor([T // 2, 0, 1][:N], dtype=torch.int32)
        lengths = lengths.cuda()
    return gi, dy, bias, f(N, H).cuda(), f(N, H).cuda(), lengths


def bounds(gi, bias, h0, lengths, dy, dh_last):
    """(states, y, dgi, dh0 wanted, and the error of each without the final rounding)."""
    T, N, H = gi.shape[0], gi.shape[1], gi.shape[2] // 3
    y, states = S.glr_fwd(gi, bias, h0, lengths)
    dgi, dh0 = S.glr_bwd(gi, bias, states, dy, dh_last, lengths)
    err, mag = [np.zeros((N, H))], [np.abs(h0)]
    err_y, f_, keep_, c_, o_, shut_, k_ = np.zeros((T, N, H)), *(np.zeros((T, N, H)) for _ in range(6))
    for t in range(T):
        live = (np.ones(N, bool) if lengths is None else lengths > t)[:, None]
        f, keep, c, o, shut = S.glr_gates(gi[t], bias)
        a = np.abs(gi[t] + bias)
        k = 16 + 2 * (a[:, :H] + a[:, 2 * H:])
        mag_c = np.abs(gi[t][:, H:2 * H]) + np.abs(bias[H:2 * H])
        m = np.where(live, f * mag[-1] + keep * mag_c, mag[-1])
        err.append(np.where(live, f * err[-1] + k * U * m, err[-1]))
        mag.append(m)
        err_y[t] = np.where(live, o * err[-1] + k * U * o * m, 0)
        f_[t], keep_[t], c_[t], o_[t], shut_[t], k_[t] = np.where(live, f, 1), np.where(live, keep, 0), np.where(live, mag_c, 0), np.where(live, o, 0), shut, k
    G, eG = np.abs(dh_last), np.zeros((N, H))
    err_g = np.zeros(gi.shape)
    up = np.abs(dy)
    for t in reversed(range(T)):
        G = G + up[t] * o_[t]
        eG = eG + k_[t] * U * G
        fac = keep_[t] * f_[t]
        around = mag[t] + c_[t]
        err_g[t] = np.concatenate((fac * (eG * around + G * err[t] + 3 * k_[t] * U * G * around), keep_[t] * (eG + 2 * k_[t] * U * G),
                                   up[t] * o_[t] * shut_[t] * (err[t + 1] + 4 * k_[t] * U * mag[t + 1])), axis=-1)
        G, eG = f_[t] * G, f_[t] * (eG + 2 * k_[t] * U * G)
    return (states, y, dgi, dh0), (np.stack(err), err_y, err_g, eG + 4 * U * np.abs(dh0))


def in_bound(got, want, bound, what):
    bad = ~(np.abs(got - want) <= bound + 1e-37)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:3].tolist(), float(np.max(np.abs(got - want)[bad])), float(np.max((np.abs(got - want) / (bound + 1e-37))[bad])))


def check(gi, dy, bias, h0, dh_last, lengths, dtype):
    T, N, H = dy.shape
    n64 = lambda t: None if t is None else host(t)
    hl = None if lengths is None else lengths.cpu().numpy()
    zero = np.zeros((N, H))
    (states, wy, wg, w0), (es, ey, eg, e0) = bounds(host(gi), np.zeros(3 * H) if bias is None else host(bias), zero if h0 is None else host(h0), hl, host(dy), zero if dh_last is None else host(dh_last))
    r = half(dtype)
    y, y_ok = guarded((T, N, H), gi.dtype)
    h_last, h_ok = guarded((N, H), torch.float32)
    saved, s_ok = guarded((-(-T // 16), N, H), torch.float32)
    B.glr_fwd(gi, bias, h0=h0, lengths=lengths, y=y, h_last=h_last, saved=saved)
    y_ok(), h_ok(), s_ok()
    in_bound(host(h_last), states[-1], es[-1], "h_last")
    in_bound(host(saved), states[:-1][::16], es[:-1][::16], "saved")
    in_bound(host(y), wy, ey * (1 + r) + r * np.abs(wy), "y")
    dgi, g_ok = guarded((T, N, 3 * H), gi.dtype)
    dh0, d_ok = guarded((N, H), torch.float32)
    B.glr_bwd(gi, saved, bias, dy=dy, dh_last=dh_last, lengths=lengths, dgi=dgi, dh0=dh0)
    g_ok(), d_ok()
    in_bound(host(dgi), wg, eg * (1 + r) + r * np.abs(wg), "dgi")
    in_bound(host(dh0), w0, e0, "dh0")
    return y, h_last, saved, dgi, dh0


@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,H", SHAPES)
def test_sequences(T, N, H, dtype, ragged):
    print(f"recurrence T={T} N={N} H={H} {dtype} ragged={ragged}", flush=True)
    gi, dy, bias, h0, dh_last, lengths = make(T + H, T, N, H, dtype, ragged)
    y, h_last, saved, dgi, dh0 = check(gi, dy, bias, h0, dh_last, lengths, dtype)
    # without what may be left out: the same values
    y2, h2, none = B.glr_fwd(gi, bias, h0=h0, lengths=lengths, save=False)
    assert none is None and torch.equal(y2, y) and torch.equal(h2, h_last)
    none, h3, s3 = B.glr_fwd(gi, bias, h0=h0, lengths=lengths, want_y=False)
    assert none is None and torch.equal(h3, h_last) and torch.equal(s3, saved)
    g2, none = B.glr_bwd(gi, saved, bias, dy=dy, dh_last=dh_last, lengths=lengths, want_dh0=False)
    assert none is None and torch.equal(g2, dgi)
    zero = torch.zeros_like(dh_last)
    assert all(torch.equal(a, b) for a, b in zip(B.glr_bwd(gi, saved, bias, dy=dy, lengths=lengths), B.glr_bwd(gi, saved, bias, dy=dy, dh_last=zero, lengths=lengths)))
    assert all(torch.equal(a, b) for a, b in zip(B.glr_bwd(gi, saved, bias, dh_last=dh_last, lengths=lengths), B.glr_bwd(gi, saved, bias, dy=torch.zeros_like(dy), dh_last=dh_last, lengths=lengths)))


def test_without_bias_or_initial_state():
    gi, dy, _, _, dh_last, _ = make(4, 40, 3, 70, "f32", False)
    check(gi, dy, None, None, dh_last, None, "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,H", [(5, 3, 24), (100, 4, 65), (700, 2, 64)])
def test_strides(T, N, H, dtype):
    """Batch-major tensors, and tensors that are columns of wider ones, give what dense time-major ones give, bit by bit, and touch nothing else."""
    gi, dy, bias, h0, dh_last, lengths = make(9, T, N, H, dtype, True)
    y, h_last, saved = B.glr_fwd(gi, bias, h0=h0, lengths=lengths)
    dgi, dh0 = B.glr_bwd(gi, saved, bias, dy=dy, dh_last=dh_last, lengths=lengths)
    batch = lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)
    y2, h2, s2 = B.glr_fwd(batch(gi), bias, h0=h0, lengths=lengths)
    assert y2.stride(1) > y2.stride(0) or N == 1
    g2, d2 = B.glr_bwd(batch(gi), s2, bias, dy=batch(dy), dh_last=dh_last, lengths=lengths)
    assert torch.equal(y2, y) and torch.equal(h2, h_last) and torch.equal(s2, saved) and torch.equal(g2, dgi) and torch.equal(d2, dh0)
    for pad in (1, 8):
        wide = lambda t: torch.full((T, N, t.shape[2] + pad), float("nan"), dtype=t.dtype, device="cuda:0")
        wgi, wy, wdy, wg = wide(gi), wide(dy), wide(dy), wide(gi)
        wgi[..., :3 * H], wdy[..., :H] = gi, dy
        y3, h3, s3 = B.glr_fwd(wgi[..., :3 * H], bias, h0=h0, lengths=lengths, y=wy[..., :H])
        g3, d3 = B.glr_bwd(wgi[..., :3 * H], s3, bias, dy=wdy[..., :H], dh_last=dh_last, lengths=lengths, dgi=wg[..., :3 * H])
        assert torch.equal(y3, y) and torch.equal(h3, h_last) and torch.equal(s3, saved) and torch.equal(g3, dgi) and torch.equal(d3, dh0)
        assert wy[..., H:].isnan().all() and wg[..., 3 * H:].isnan().all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,H", [(50, 30), (600, 64), (3000, 16)])
def test_what_lies_behind_a_sequence_is_not_used(T, H, dtype):
    gi, dy, bias, h0, dh_last, _ = make(13, T, 5, H, dtype, False)
    lengths = torch.tensor([T, 0, 1, T // 3, T - 1], dtype=torch.int32, device="cuda:0")
    want = B.glr_fwd(gi, bias, h0=h0, lengths=lengths)
    want += B.glr_bwd(gi, want[2], bias, dy=dy, dh_last=dh_last, lengths=lengths)
    for junk in (float("nan"), float("inf"), torch.finfo(gi.dtype).min):
        g, d = gi.clone(), dy.clone()
        for n, length in enumerate(lengths.tolist()):
            g[length:, n] = junk
            d[length:, n] = junk
        got = B.glr_fwd(g, bias, h0=h0, lengths=lengths)
        got += B.glr_bwd(g, got[2], bias, dy=d, dh_last=dh_last, lengths=lengths)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), junk
    # a length that says less than nothing, or more than there is
    odd = torch.tensor([T + 5, -3, 1, T // 3, T - 1], dtype=torch.int32, device="cuda:0")
    assert all(torch.equal(a, b) for a, b in zip(B.glr_fwd(gi, bias, h0=h0, lengths=odd), want))
    assert torch.equal(want[0][:, 1], torch.zeros_like(want[0][:, 1])) and torch.equal(want[1][1], h0[1]) and torch.equal(want[4][1], dh_last[1])


def test_gates_at_their_ends():
    """Arguments far beyond where a gate is 0 or 1 to all places: states kept for ever, and states that are the last candidate."""
    T, N, H = 70, 2, 64
    gi, dy, _, h0, dh_last, _ = make(17, T, N, H, "f32", False)
    for a in (1e4, -1e4, float("inf"), float("-inf")):
        g = gi.clone()
        g[..., :H] = a
        y, h, saved = B.glr_fwd(g, None, h0=h0)
        o = torch.sigmoid(gi[..., 2 * H:].double())
        want = h0 if a > 0 else gi[-1, :, H:2 * H]
        assert torch.equal(h, want)
        dgi, dh0 = B.glr_bwd(g, saved, None, dy=dy, dh_last=dh_last)
        assert torch.isfinite(dgi).all() and not dgi[..., :H].any()
        if a < 0:
            assert not dh0.any()
        else:
            in_bound(host(dh0), host((dy.double() * o).sum(0) + dh_last.double()), (T + 12) * U * host((dy.double() * o).abs().sum(0) + dh_last.abs()), "dh0")


@pytest.mark.parametrize("low,high", [(0.0, 4.0), (4.0, 8.0), (8.0, 12.0), (12.0, 16.0), (16.0, 24.0), (24.0, 80.0)])
def test_a_gate_that_is_nearly_closed(low, high):
    """Gates whose arguments are exact (no bias) to within a few units, whatever the argument.  With u = 2^-24: the exponential is good to 1 ulp = 2 u and
    rounded once more when its argument's rounding is put back, 3 u; 1 + e, its reciprocal and the product of the two add u each: 6 u.  ln(2) in one word is off by 2.7e-9 of itself:
    0.05 u for a unit of the argument, 1.2 u at 24 and 4 u at 80: 8 u and 10 u.  h = f * 1 + (1 - f) * 0 and 0 + (1 - f) * 1 are the gates themselves (one product by 1,
    one sum with 0: exact), y = o * 1.  A product of two gates has both errors and u, each further product u.  All steps at once and one token take the same gates."""
    H, n = 4096, 8 if high <= 24 else 10
    a = torch.linspace(low, high, H, device="cuda:0")
    a[0], a[-1] = low, high
    gate = lambda x: (S.sigmoid(host(x)), S.sigmoid(-host(x)))
    one, far = torch.ones(H, device="cuda:0"), torch.full((H,), float("inf"), device="cuda:0")
    rel = lambda got, want, units, what: in_bound(host(got), want, units * U * np.abs(want), (what, low))

    def both(f, c, o, h0):
        """(y, h, saved) of one step, and the same for a token."""
        gi = torch.cat((f, c, o))[None, None]
        y, h, saved = B.glr_fwd(gi, None, h0=h0[None])
        state = h0[None].clone()
        y2 = B.glr_step(gi[0], state, None)
        in_bound(host(state), host(h), 2 * U * np.abs(host(h)), "token state")
        in_bound(host(y2), host(y[0]), 3 * U * np.abs(host(y[0])), "token y")
        return gi, y, h, saved

    for x in (a, -a):
        f, keep = gate(x)
        _, _, h, _ = both(x, 0 * one, 0 * one, one)
        rel(h[0], f, n, "f")
        gi, _, h, saved = both(x, one, 0 * one, 0 * one)
        rel(h[0], keep, n, "1 - f")
        dgi, dh0 = B.glr_bwd(gi, saved, None, dh_last=one[None])
        rel(dh0[0], f, n, "dh0")
        rel(dgi[0, 0, H:2 * H], keep, n, "dc")
        rel(dgi[0, 0, :H], -f * keep, 2 * n + 1, "df")
        gi, y, _, saved = both(-far, one, x, one)              # f = 0: h = c = 1
        rel(y[0, 0], f, n, "o")
        dgi, _ = B.glr_bwd(gi, saved, None, dy=one[None, None])
        rel(dgi[0, 0, 2 * H:], f * keep, 2 * n + 2, "do")


def test_a_nan_stays_in_its_channel():
    gi, dy, bias, h0, _, _ = make(19, 300, 2, 70, "f32", False)
    want = B.glr_fwd(gi, bias, h0=h0)
    gi[100, 1, 5] = float("nan")
    got = B.glr_fwd(gi, bias, h0=h0)
    assert got[0][100:, 1, 5].isnan().all() and got[1][1, 5].isnan()
    got[0][100:, 1, 5] = want[0][100:, 1, 5]
    assert torch.equal(got[0], want[0])


@pytest.mark.parametrize("T,N,H", [(3, 1, 2), (40, 2, 3)])
def test_gradient_against_differences(T, N, H):
    """The kernel's gradients against differences of its own forward pass: the loss is summed in 64 bits; steps of 2^-8; the third derivative of the loss along one
    gate's argument is below the sum of |dy| that it reaches times the candidates' size, and the rounding 64 u of the same over 2h."""
    gi, dy, bias, h0, dh_last, _ = make(23, T, N, H, "f32", False)
    saved = B.glr_fwd(gi, bias, h0=h0)[2]
    dgi, dh0 = B.glr_bwd(gi, saved, bias, dy=dy, dh_last=dh_last)
    h = 2.0 ** -8

    def loss(g, s):
        y, last, _ = B.glr_fwd(g, bias, h0=s)
        return float((y.double() * dy.double()).sum() + (last.double() * dh_last.double()).sum())

    size = float(dy.abs().double().sum() + dh_last.abs().double().sum()) * float(gi.abs().max() + bias.abs().max() + h0.abs().max())
    limit = h * h / 6 * float(dy.abs().sum(0).max() + dh_last.abs().max()) * float(gi.abs().max() + bias.abs().max() + h0.abs().max()) + 64 * U * size / (2 * h)
    for i in np.ndindex(*gi.shape):
        e = torch.zeros_like(gi)
        e[i] = h
        assert abs((loss(gi + e, h0) - loss(gi - e, h0)) / (2 * h) - float(dgi[i])) <= limit, i
    for i in np.ndindex(N, H):
        e = torch.zeros_like(h0)
        e[i] = h
        assert abs((loss(gi, h0 + e) - loss(gi, h0 - e)) / (2 * h) - float(dh0[i])) <= limit, i


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,H", [(1, 1), (3, 8), (50, 256), (7, 65), (300, 40), (2, 4100)])
def test_single_tokens(N, H, dtype):
    print(f"token N={N} H={H} {dtype}", flush=True)
    gi, _, bias, h0, _, _ = make(N + H, 1, N, H, dtype, False)
    (states, wy, _, _), (es, ey, _, _) = bounds(host(gi), host(bias), host(h0), None, np.zeros((1, N, H)), np.zeros((N, H)))
    r = half(dtype)
    state, s_ok = guarded((N, H), torch.float32)
    y, y_ok = guarded((N, H), gi.dtype)
    state.copy_(h0)
    B.glr_step(gi[0], state, bias, y=y)
    s_ok(), y_ok()
    in_bound(host(state), states[1], es[1], "state")
    in_bound(host(y), wy[0], ey[0] * (1 + r) + r * np.abs(wy[0]), "y")
    # the states in a larger table, in another order; idle places change nothing
    S_ = N + 9
    slots = torch.randperm(S_)[:N].to(torch.int32).cuda()
    table = torch.randn(S_, H, device="cuda:0")
    table[slots.long()] = h0
    idle = torch.zeros(N, dtype=torch.bool, device="cuda:0")
    idle[1::3] = True
    slots[1::3] = torch.where(torch.arange(slots[1::3].numel(), device="cuda:0") % 2 == 0, -1, S_).to(torch.int32)
    want_t = table.clone()
    want_t[slots[~idle].long()] = state[~idle]
    got = B.glr_step(gi[0], table, bias, slots=slots)
    assert torch.equal(table, want_t) and torch.equal(got[~idle], y[~idle]) and not got[idle].any()
    none = B.glr_step(gi[0], table.clone(), bias, slots=slots, want_y=False)
    assert none is None


def test_tokens_one_by_one_are_the_sequence():
    T, N, H = 40, 3, 72
    gi, _, bias, h0, _, _ = make(29, T, N, H, "f32", False)
    y, h_last, _ = B.glr_fwd(gi, bias, h0=h0)
    (_, wy, _, _), (_, ey, _, _) = bounds(host(gi), host(bias), host(h0), None, np.zeros((T, N, H)), np.zeros((N, H)))
    state = h0.clone()
    ys = torch.stack([B.glr_step(gi[t], state, bias) for t in range(T)])
    in_bound(host(ys), wy, ey + U * np.abs(wy), "y")
    in_bound(host(y), wy, ey + U * np.abs(wy), "y")


LONG = [(300, 1, 64), (2100, 3, 24), (4000, 20, 40), (20000, 1, 1), (700, 90, 200), (90, 2100, 64)]      # several segments: one tile, two, 13, one, 282, 2100


@pytest.mark.parametrize("T,N,H", LONG)
def test_long_sequences_give_the_same_bits_every_time(T, N, H):
    """Whatever the blocks find of each other's values, and whatever runs beside them: two streams at once, each with scratch of its own."""
    gi, dy, bias, h0, dh_last, lengths = make(37, T, N, H, "bf16", True)

    def run(ws):
        y, h, saved = B.glr_fwd(gi, bias, h0=h0, lengths=lengths, ws=ws)
        return (y, h, saved, *B.glr_bwd(gi, saved, bias, dy=dy, dh_last=dh_last, lengths=lengths, ws=ws))

    want = run(B.Workspace("cuda:0"))
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    spaces = [B.Workspace("cuda:0") for _ in streams]
    for _ in range(6):
        for stream, ws in zip(streams, spaces):
            with torch.cuda.stream(stream):
                got.append(run(ws))
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, want))


@pytest.mark.parametrize("T,N,H", LONG)
def test_long_sequences_that_hold_the_mark_of_nothing(T, N, H):
    """Values whose bits are all ones, a NaN, which is also what the scratch memory holds where no block has left anything yet: the NaN goes on, in its channel alone."""
    gi, dy, bias, h0, dh_last, _ = make(41, T, N, H, "f32", False)
    want = B.glr_fwd(gi, bias, h0=h0)
    want += B.glr_bwd(gi, want[2], bias, dy=dy, dh_last=dh_last)
    for where in (slice(0, H), slice(H, 2 * H), slice(2 * H, 3 * H)):
        bad, bad_dy = gi.clone(), dy.clone()
        at = T // 2
        bad[at, 0, where][0:1].view(torch.int32).fill_(-1)
        bad_dy[at, 0, 0:1].view(torch.int32).fill_(-1)
        y, h, saved = B.glr_fwd(bad, bias, h0=h0)
        dgi, dh0 = B.glr_bwd(bad, saved, bias, dy=bad_dy, dh_last=dh_last)
        torch.cuda.synchronize()
        assert dh0[0, 0].isnan() and y[at, 0, 0].isnan()
        keep = torch.ones((N, H), dtype=torch.bool, device="cuda:0")
        keep[0, 0] = False
        assert torch.equal(y[:, keep], want[0][:, keep]) and torch.equal(h[keep], want[1][keep]) and torch.equal(dh0[keep], want[4][keep])
        assert torch.equal(dgi[..., :H][:, keep], want[3][..., :H][:, keep]) and torch.equal(dgi[..., 2 * H:][:, keep], want[3][..., 2 * H:][:, keep])


@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,H", LONG)
def test_blocks_that_wait_for_nobody(nsk_env, T, N, H, dtype, ragged):
    """Blocks that look once for the state in front of their segment and make it themselves if it is not there: the same values to rounding."""
    nsk_env("NSK_GLR_POLLS", "0")
    print(f"recurrence, no waiting, T={T} N={N} H={H} {dtype} ragged={ragged}", flush=True)
    gi, dy, bias, h0, dh_last, lengths = make(T + H + 1, T, N, H, dtype, ragged)
    check(gi, dy, bias, h0, dh_last, lengths, dtype)


def test_offsets_beyond_32_bits():
    """Rows whose offsets, in elements and in bytes, pass 2^31 and 2^32: the last sequences of a batch-major tensor of 2^31 + elements against the same alone."""
    H, T = 128, 700
    N = (1 << 31) // (3 * H * T) + 20
    gi = torch.empty((N, T, 3 * H), dtype=torch.bfloat16, device="cuda:0")
    gi[:8].normal_()
    gi[-8:].normal_()
    gi[8:-8] = 0
    bias = torch.randn(3 * H, device="cuda:0")
    y, h_last, saved = B.glr_fwd(gi.transpose(0, 1), bias)
    dgi, _ = B.glr_bwd(gi.transpose(0, 1), saved, bias, dy=y)
    for part in (slice(0, 8), slice(N - 8, N)):
        y2, h2, s2 = B.glr_fwd(gi[part].transpose(0, 1), bias)
        g2, _ = B.glr_bwd(gi[part].transpose(0, 1), s2, bias, dy=y2)
        for a, b in ((y[:, part], y2), (h_last[part], h2), (dgi[:, part], g2)):
            in_bound(host(a.float()), host(b.float()), 2.0 ** -6 * np.abs(host(b.float())) + 1e-4, "part")


def sequences_in_bound(at, inputs, outputs, dtype):
    """The outputs (y, h_last, saved, dgi, dh0) of the sequences `at` against the oracle."""
    gi, dy, bias, h0, dh_last, lengths = inputs
    part = lambda t: host(t[:, at] if t.dim() == 3 else t[at])
    (states, wy, wg, w0), (es, ey, eg, e0) = bounds(part(gi), host(bias), part(h0), None if lengths is None else lengths[at].cpu().numpy(), part(dy), part(dh_last))
    y, h_last, saved, dgi, dh0 = (part(t) for t in outputs)
    r = half(dtype)
    in_bound(h_last, states[-1], es[-1], "h_last")
    in_bound(saved, states[:-1][::16], es[:-1][::16], "saved")
    in_bound(y, wy, ey * (1 + r) + r * np.abs(wy), "y")
    in_bound(dgi, wg, eg * (1 + r) + r * np.abs(wg), "dgi")
    in_bound(dh0, w0, e0, "dh0")


@pytest.mark.parametrize("dtype,T,N,H,stride", [("bf16", 300, 3, 65, (1 << 29) + 24), ("f32", 300, 3, 65, (1 << 28) + 20), ("bf16", 40, 2, 7, (1 << 31) + 8), ("f32", 700, 2, 130, (1 << 30) + 4),
                                                ("bf16", 300, 9, 7, 54_000_000)])
def test_sequences_far_from_each_other(dtype, T, N, H, stride):
    """Sequences that begin so far from each other that a tile cannot go on from one to the next (a lane's offset has 30 bits), against the oracle; nothing else is written.
    In the last case it is a tile's ten sequences that are too far for the bits, not two of them.  Where dense tensors have as few tiles, and so blocks of the same size, their bits."""
    print(f"recurrence, far apart, T={T} N={N} H={H} {dtype} stride={stride}", flush=True)
    gi, dy, bias, h0, dh_last, lengths = make(T + H, T, N, H, dtype, True)
    dense = check(gi, dy, bias, h0, dh_last, lengths, dtype)

    def far(width, fill):
        buf = torch.full(((N - 1) * stride + T * width,), fill, dtype=gi.dtype, device="cuda:0")
        return buf, buf.as_strided((T, N, width), (width, stride, 1))

    (_, fgi), (_, fdy), (by, fy), (bg, fg) = far(3 * H, 0.0), far(H, 0.0), far(H, float("nan")), far(3 * H, float("nan"))
    fgi.copy_(gi), fdy.copy_(dy)
    _, h2, s2 = B.glr_fwd(fgi, bias, h0=h0, lengths=lengths, y=fy)
    _, d2 = B.glr_bwd(fgi, s2, bias, dy=fdy, dh_last=dh_last, lengths=lengths, dgi=fg)
    torch.cuda.synchronize()
    sequences_in_bound(list(range(N)), (gi, dy, bias, h0, dh_last, lengths), (fy, h2, s2, fg, d2), dtype)
    if N * -(-H // 64) < 8:
        assert all(torch.equal(a, b) for a, b in zip((fy, h2, s2, fg, d2), dense))
    for buf, part in ((by, fy), (bg, fg)):
        part.fill_(float("nan"))
        assert all(bool(buf[k:k + (1 << 28)].isnan().all()) for k in range(0, buf.numel(), 1 << 28))


@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,H", [(140, 1024, 64), (230, 700, 96), (170, 1024, 64), (330, 520, 128)])
def test_small_blocks_where_tiles_are_many(T, N, H, dtype, ragged):
    """Blocks of three stretches (9, 15 and 21 of them) and of two (11), in both directions: sequences here and there against the oracle, and all the same bits twice."""
    print(f"recurrence, small blocks, T={T} N={N} H={H} {dtype} ragged={ragged}", flush=True)
    gi, dy, bias, h0, dh_last, lengths = make(T + N, T, N, H, dtype, ragged)
    ws = B.Workspace("cuda:0")

    def run():
        y, h_last, saved = B.glr_fwd(gi, bias, h0=h0, lengths=lengths, ws=ws)
        return (y, h_last, saved, *B.glr_bwd(gi, saved, bias, dy=dy, dh_last=dh_last, lengths=lengths, ws=ws))

    got = run()
    assert all(torch.equal(a, b) for a, b in zip(run(), got))
    sequences_in_bound([0, 1, 2, 3, 63, 64, N // 2, N - 65, N - 2, N - 1], (gi, dy, bias, h0, dh_last, lengths), got, dtype)


def test_a_launch_of_nearly_all_threads_that_there_are():
    """Nine tiles of 70 million steps: with as many blocks for each of eight groups of tiles the launch would have more than 2^32 threads.  The same steps in seven calls, each of which
    begins with the state that the one before left, take the same stretches and segments: the same bits."""
    N, T, parts = 9, 70_000_000, 7
    each = T // parts
    g = torch.Generator(device="cuda").manual_seed(43)
    gi = torch.randn((N, T, 3), generator=g, device="cuda:0", dtype=torch.bfloat16).transpose(0, 1)
    dy = torch.randn((N, T, 1), generator=g, device="cuda:0", dtype=torch.bfloat16).transpose(0, 1)
    bias, h0, dh_last = torch.tensor([1.0, 0.2, -0.1], device="cuda:0"), torch.randn((N, 1), generator=g, device="cuda:0"), torch.randn((N, 1), generator=g, device="cuda:0")
    ws = B.Workspace("cuda:0")
    print("recurrence T=70000000 N=9 H=1 bf16 forward", flush=True)
    y, h_last, saved = B.glr_fwd(gi, bias, h0=h0, ws=ws)
    torch.cuda.synchronize()
    print("backward", flush=True)
    dgi, dh0 = B.glr_bwd(gi, saved, bias, dy=dy, dh_last=dh_last, ws=ws)
    torch.cuda.synchronize()
    cut = lambda t, k: t[k * each:(k + 1) * each]
    h = h0
    for k in range(parts):
        y2, h, s2 = B.glr_fwd(cut(gi, k), bias, h0=h, ws=ws)
        assert torch.equal(y2, cut(y, k)) and torch.equal(s2, saved[k * each // 16:(k + 1) * each // 16])
    assert torch.equal(h, h_last)
    d = dh_last
    for k in reversed(range(parts)):
        g2, d = B.glr_bwd(cut(gi, k), saved[k * each // 16:(k + 1) * each // 16], bias, dy=cut(dy, k), dh_last=d, ws=ws)
        assert torch.equal(g2, cut(dgi, k))
    assert torch.equal(d, dh0)


@pytest.mark.parametrize("T,N,H", [(90, 4, 72), (3000, 1, 64)])
def test_on_a_stream_and_in_a_graph(T, N, H):
    gi, dy, bias, h0, dh_last, lengths = make(31, T, N, H, "bf16", True)
    ws = B.Workspace("cuda:0")
    y, dgi = torch.empty_like(dy), torch.empty_like(gi)
    h_last, dh0, saved = torch.empty_like(h0), torch.empty_like(h0), torch.empty((-(-T // 16), N, H), device="cuda:0")

    def step():
        B.glr_fwd(gi, bias, h0=h0, lengths=lengths, y=y, h_last=h_last, saved=saved, ws=ws)
        B.glr_bwd(gi, saved, bias, dy=dy, dh_last=dh_last, lengths=lengths, dgi=dgi, dh0=dh0, ws=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        gi.copy_(torch.randn(gi.shape, device="cuda:0").to(gi.dtype))
        graph.replay()
        torch.cuda.synchronize()
        got = [b.clone() for b in (y, dgi, h_last, dh0, saved)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (y, dgi, h_last, dh0, saved))), k

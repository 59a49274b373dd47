"""Gated delta rule against the step-by-step form in 64 bits (oracle/learning.py), its gradients against torch's of that form.

Tolerances.  fp32: a value is reached through at most eight products one after the other (A, the inverse of a block, the solution, the state, and back), each a sum of at most 192 terms
whose roundings, 2^-24 of the partial sum each, add up like sqrt(192); the state adds one such error a chunk, of which the gates leave a geometric sum (at most 8 here): 8 * sqrt(192) * 8 *
2^-24 = 5.3e-5 of the largest value at the very worst, and of the norm by a sqrt of the eight products and chunks less, 8 * sqrt(192) * 2^-24 = 6.6e-6.  Values in bf16 are rounded once more: half a step,
2^-8 of the value.  Of the gradient y of a normalised query or key what lies along it is taken out, r (y - x^ (x^.y)) with r = 1 / length: both terms are rounded at their size, so F32 * r * |y| stays,
also where little is left of them (all of it where D = 1)."""
import math

import pytest
import torch

from oracle import learning as O
from paper_2409_11600_amd import binding as B

pytestmark = pytest.mark.gpu
F32 = 8 * math.sqrt(192) * 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def close(got, want, name="", slack=None):
    assert got.shape == want.shape
    bf16 = got.dtype == torch.bfloat16
    got, want = got.detach().double().cpu(), want.detach().double()
    assert bool(torch.isfinite(got).all()), name
    top = want.abs().max().item()
    slack = torch.zeros(()) if slack is None else slack
    tol, half = F32 + (2.0 ** -8 if bf16 else 0), 2.0 ** -8 if bf16 else 0
    assert bool((got - want).norm() <= tol * want.norm() + slack.norm() + 1e-30), (name, ((got - want).norm() / want.norm()).item())
    assert bool(((got - want).abs() <= 8 * F32 * top + half * want.abs() + slack + 1e-30).all()), (name, (got - want).abs().max().item(), top)


def case(T, N, heads, dtype="f32", lengths=None, seed=0, bias=True, h0=True):
    H, Hk, D, Dv = heads
    gen = torch.Generator().manual_seed(seed)
    normal = lambda *s: torch.randn(s, generator=gen)
    dt = TYPES[dtype]
    c = {"gi": normal(T, N, 2 * Hk * D + H * (Dv + 2)).to(dt), "do": normal(T, N, H * Dv).to(dt), "dh_last": normal(N, H, D, Dv), "lengths": None}
    c["bias"] = torch.cat((1 + 4 * torch.rand(H, generator=gen), 0.5 * normal(H))) if bias else None
    c["h0"] = normal(N, H, D, Dv) if h0 else None
    if lengths is not None:
        c["lengths"] = torch.tensor(lengths, dtype=torch.int32)
    return c


def along(c, heads):
    """F32 * r * |y| of each query and key row, over its elements; zeros elsewhere."""
    H, Hk, D, _ = heads
    gi = torch.nan_to_num(c["gi"].double(), nan=0.0, posinf=0.0, neginf=0.0)
    iq, ik = O.inverse_lengths(gi, heads)
    x = gi.clone()
    for i, r in enumerate((iq, ik)):
        x[..., i * Hk * D:(i + 1) * Hk * D] = (gi[..., i * Hk * D:(i + 1) * Hk * D].unflatten(-1, (Hk, D)) * r).flatten(-2)
    y = wanted(dict(c, gi=x), heads, normalised=True)[3]
    slack = torch.zeros_like(y)
    for i, r in enumerate((iq, ik)):
        rows = y[..., i * Hk * D:(i + 1) * Hk * D].unflatten(-1, (Hk, D))
        slack[..., i * Hk * D:(i + 1) * Hk * D] = (F32 * r * rows.norm(dim=-1, keepdim=True)).expand_as(rows).flatten(-2)
    return slack


def wanted(c, heads, normalised=False):
    """(o, h_last, saved, dgi, dh0) in 64 bits."""
    x = {k: v.double().requires_grad_(k in ("gi", "h0")) for k, v in c.items() if v is not None and v.is_floating_point()}
    N, (H, _, D, Dv) = c["gi"].shape[1], heads
    h0 = x.get("h0", torch.zeros((N, H, D, Dv), dtype=torch.float64, requires_grad=True))
    o, S, saved = O.delta(x["gi"], heads, x.get("bias"), h0, None if c["lengths"] is None else c["lengths"].clamp(0, c["gi"].shape[0]), normalised)
    loss = (o * x["do"]).sum() if "do" in x else 0.0
    loss = loss + (S * x["dh_last"]).sum() if "dh_last" in x else loss
    dgi, dh0 = torch.autograd.grad(loss, (x["gi"], h0))
    return o, S, saved, dgi, dh0


def gpu(c):
    return {k: None if v is None else v.cuda() for k, v in c.items()}


def both(g, heads, **kw):
    o, last, saved = B.delta_fwd(g["gi"], heads, g["bias"], h0=g["h0"], lengths=g["lengths"], **kw)
    dgi, dh0 = B.delta_bwd(g["gi"], saved, heads, g["bias"], do=g.get("do"), dh_last=g.get("dh_last"), lengths=g["lengths"], **kw)
    return o, last, saved, dgi, dh0


def check(c, heads):
    want, got, slack = wanted(c, heads), both(gpu(c), heads), along(c, heads)
    for name, a, b in zip(("o", "h_last", "saved", "dgi", "dh0"), got, want):
        close(a, b, name, slack if name == "dgi" else None)
    # the parts of a row by themselves: small ones must not hide behind large
    H, Hk, D, Dv = heads
    parts = [Hk * D, Hk * D, H * Dv, H, H]
    for name, a, b, more in zip("qkvab", got[3].split(parts, -1), want[3].split(parts, -1), slack.split(parts, -1)):
        close(a, b, "d" + name, more)


# (heads, rows): one chunk and several, ends of chunks and of tiles, one key head for several, widths below, at and above the tiles'
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,heads", [(1, 2, (2, 2, 16, 16)), (15, 1, (1, 1, 1, 1)), (16, 3, (2, 1, 8, 24)), (63, 2, (3, 3, 33, 17)), (64, 1, (4, 2, 64, 64)), (65, 2, (2, 2, 64, 128)),
                                       (128, 1, (2, 1, 128, 64)), (130, 2, (6, 2, 13, 100)), (200, 2, (2, 2, 128, 128)), (257, 1, (3, 1, 40, 72))])
def test_sizes(T, N, heads, dtype):
    check(case(T, N, heads, dtype, seed=T), heads)


# many heads: a block takes all chunks of one, or two do, or eight wavefronts; few heads and many chunks: cut into segments, the last of one chunk
@pytest.mark.parametrize("T,N,heads,dtype", [(140, 66, (3, 1, 20, 36), "f32"), (135, 50, (4, 4, 32, 48), "bf16"), (70, 100, (2, 2, 72, 80), "f32"), (3137, 1, (2, 1, 24, 40), "f32"),
                                             (3100, 2, (1, 1, 16, 8), "bf16"), (330, 40, (3, 1, 64, 100), "bf16"), (200, 60, (2, 2, 40, 128), "f32"), (150, 70, (2, 1, 24, 72), "bf16"),
                                             (200, 36, (2, 2, 100, 120), "bf16")])
def test_ways_of_going_through(T, N, heads, dtype):
    lengths = [(37 * n + T // 2) % (T + 1) for n in range(N)]
    lengths[0] = T
    check(case(T, N, heads, dtype, lengths=lengths, seed=T), heads)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,heads", [(70, (2, 2, 16, 24)), (200, (2, 1, 48, 40))])
def test_lengths(T, heads, dtype):
    """No step, one, the ends of chunks, more than there are and fewer than none; what lies behind an end is not used, whatever it is."""
    c = case(T, 9, heads, dtype, lengths=[T, 0, 1, 63, 64, 65, -5, T + 9, 2])
    for n, l in enumerate(c["lengths"].clamp(0, T).tolist()):
        for k in ("gi", "do"):
            c[k][l:, n] = 0
    want = wanted(c, heads)
    for n, l in enumerate(c["lengths"].clamp(0, T).tolist()):
        for i, k in enumerate(("gi", "do")):
            c[k][l:, n] = (math.nan, math.inf)[(n + i) % 2]
    for name, a, b in zip(("o", "h_last", "saved", "dgi", "dh0"), both(gpu(c), heads), want):
        close(a, b, name)


def test_all_empty():
    heads = (2, 1, 16, 16)
    for T in (30, 300, 4000):
        c = case(T, 2, heads, lengths=[0, 0])
        o, last, saved, dgi, dh0 = both(gpu(c), heads)
        assert not o.any() and not dgi.any() and torch.equal(last.cpu(), c["h0"]) and torch.equal(dh0.cpu(), c["dh_last"])
        assert all(torch.equal(s.cpu(), c["h0"]) for s in saved)


@pytest.mark.parametrize("T", [40, 300])
def test_left_out(T):
    """No bias, no initial state, only one of the outputs, only one of the gradients."""
    heads = (2, 2, 24, 16)
    c = case(T, 2, heads, bias=False, h0=False)
    want, g = wanted(c, heads), gpu(c)
    o, last, saved = B.delta_fwd(g["gi"], heads)
    close(o, want[0]), close(last, want[1])
    none, last2, no_saved = B.delta_fwd(g["gi"], heads, want_o=False, save=False)
    assert none is None and no_saved is None and torch.equal(last, last2)
    for gone in ("do", "dh_last"):
        part = {k: v for k, v in c.items() if k != gone}
        want = wanted(part, heads)
        dgi, dh0 = B.delta_bwd(g["gi"], saved, heads, do=None if gone == "do" else g["do"], dh_last=None if gone == "dh_last" else g["dh_last"])
        close(dgi, want[3]), close(dh0, want[4])
        dgi2, no = B.delta_bwd(g["gi"], saved, heads, do=None if gone == "do" else g["do"], dh_last=None if gone == "dh_last" else g["dh_last"], want_dh0=False)
        assert no is None and torch.equal(dgi, dgi2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lay", ["batch", "wide", "odd"])
def test_strides(lay, dtype):
    """Batch-major rows, rows with room between them (which stays as it is), rows that begin on no vector's boundary: the same bits as dense."""
    T, N, heads = 150, 3, (2, 1, 24, 16)
    g = gpu(case(T, N, heads, dtype, lengths=[150, 70, 3]))
    ws = B.Workspace()
    want = both(g, heads, ws=ws)

    def laid(x):
        width = x.shape[-1]
        if lay == "batch":
            buf = torch.full((N, T, width), 7.0, dtype=x.dtype, device="cuda")
            view = buf.transpose(0, 1)
        else:
            buf = torch.full((T, N, width + (16 if lay == "wide" else 1)), 7.0, dtype=x.dtype, device="cuda")
            view = buf[..., :width]
        view.copy_(x)
        return buf, view

    (_, gi), (_, do) = laid(g["gi"]), laid(g["do"])
    bo, o = laid(torch.zeros_like(g["do"]))
    bg, dgi = laid(torch.zeros_like(g["gi"]))
    _, last, saved = B.delta_fwd(gi, heads, g["bias"], h0=g["h0"], lengths=g["lengths"], o=o, ws=ws)
    _, dh0 = B.delta_bwd(gi, saved, heads, g["bias"], do=do, dh_last=g["dh_last"], lengths=g["lengths"], dgi=dgi, ws=ws)
    # (the vector and the scalar loads take the sums of squares in another order: not the same bits, but the same values)
    for a, b in zip((o, last, saved, dgi, dh0), want):
        if lay == "odd":
            close(a, b.double().cpu())
        else:
            assert torch.equal(a, b)
    if lay != "batch":
        assert bool((bo[..., g["do"].shape[-1]:] == 7).all()) and bool((bg[..., g["gi"].shape[-1]:] == 7).all())


def test_closed_and_open_gates():
    """Memory that ends at once, lasts for ever, or ends in the middle of a chunk; nothing and everything written."""
    T, N, heads = 130, 4, (3, 3, 16, 16)
    c = case(T, N, heads, bias=False)
    a, b = c["gi"][..., -6:-3], c["gi"][..., -3:]
    a[..., 0], a[..., 1] = -math.inf, 200.0
    a[40:45, :, 2], a[70, :, 2] = -2000.0, -88.0
    b[..., 0], b[:, 0, 1], b[:, 1, 1] = 90.0, -math.inf, math.inf
    x = {k: v for k, v in c.items()}
    want, got = wanted(x, heads), both(gpu(c), heads)
    for name, p, q in zip(("o", "h_last", "saved"), got, want):
        close(p, q, name)
    # (the 64-bit gradient of a gate at infinity is 0 * infinity in torch; the formula's is 0)
    close(got[3], torch.nan_to_num(want[3], nan=0.0), "dgi")
    close(got[4], want[4], "dh0")


def test_keys_of_no_length_and_the_same_key():
    """Queries and keys of zeros; one key in all steps, written in full and kept, where the powers of A are largest."""
    T, N, heads = 200, 2, (2, 2, 16, 24)
    c = case(T, N, heads, bias=False)
    c["gi"][50:60, :, :64] = 0
    check(c, heads)
    c["gi"][..., 32:64] = c["gi"][:1, :1, 32:64]
    c["gi"][..., -4:] = 12.0
    # here a step takes out what the one before wrote: U is a difference of values next to each other, sums of 64 steps of +-1 before it; their roundings count up to 64 times
    want, got = wanted(c, heads), both(gpu(c), heads)
    for name, p, q in zip(("o", "h_last", "saved"), got, want):
        d = (p.double().cpu() - q).norm() / q.norm()
        assert d <= 64 * F32, (name, d)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads", [(2, 1, 16, 16), (1, 1, 64, 64), (3, 1, 13, 7), (2, 2, 128, 100), (2, 2, 100, 128)])
def test_steps_are_the_sequence(heads, dtype):
    """Token by token in a table of states, some places idle, against the whole sequence."""
    T, N, S = 20, 5, 9
    c = case(T, N, heads, dtype, h0=False)
    g, (H, _, D, Dv) = gpu(c), heads
    want = wanted(c, heads)
    table = torch.full((S, H, D, Dv), 3.0, device="cuda")
    slots = torch.tensor([7, 2, -1, 0, 9], dtype=torch.int32, device="cuda")       # the third and the last are idle
    for s in (7, 2, 0):
        table[s] = 0
    for t in range(T):
        o = B.delta_step(g["gi"][t].clone(), table, heads, g["bias"], slots=slots)
        for n, s in enumerate(slots.tolist()):
            if 0 <= s < S:
                close(o[n], want[0][t, n], f"step {t}")
            else:
                assert not o[n].any()
    for n, s in enumerate(slots.tolist()):
        if 0 <= s < S:
            close(table[s], want[1][n])
    assert bool((table[[1, 3, 4, 5, 6, 8]] == 3).all())
    first = torch.zeros(N + 2, H, D, Dv, device="cuda")
    assert B.delta_step(g["gi"][0].clone(), first, heads, g["bias"], want_o=False) is None
    close(first[:N].reshape(N, -1), O.delta_step(c["gi"][0].double(), torch.zeros(N, H, D, Dv, dtype=torch.float64), heads, c["bias"].double())[1].reshape(N, -1))
    assert not first[N:].any()


def test_same_bits_and_beside_each_other():
    """Twice the same call, and two streams at once with a workspace each."""
    kinds = [((2, 1, 64, 64), 500, 3), ((2, 2, 24, 72), 3200, 1), ((4, 4, 32, 32), 130, 60)]
    data = [(gpu(case(T, N, heads, "bf16", seed=i)), heads) for i, (heads, T, N) in enumerate(kinds)]
    want = [both(g, heads) for g, heads in data]
    torch.cuda.synchronize()
    streams, spaces, got = [torch.cuda.Stream() for _ in data], [B.Workspace() for _ in data], []
    for _ in range(4):
        for s, ws, (g, heads) in zip(streams, spaces, data):
            with torch.cuda.stream(s):
                got.append(both(g, heads, ws=ws))
    torch.cuda.synchronize()
    for i, r in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(r, want[i % len(want)]))


@pytest.mark.parametrize("T,N,heads", [(150, 2, (2, 1, 32, 32)), (3100, 1, (2, 2, 16, 16)), (70, 100, (2, 2, 16, 16)), (70, 2, (2, 2, 16, 72))])
def test_states_in_place(T, N, heads):
    """The last state into the buffer of the first, and the gradient of the first into that of the last: what a sequence in parts does."""
    c = case(T, N, heads)
    g = gpu(c)
    o, last, saved, dgi, dh0 = both(g, heads)
    h, dh = g["h0"].clone(), g["dh_last"].clone()
    again, _, _ = B.delta_fwd(g["gi"], heads, g["bias"], h0=h, h_last=h)
    assert torch.equal(again, o) and torch.equal(h, last)
    dgi2, _ = B.delta_bwd(g["gi"], saved, heads, g["bias"], do=g["do"], dh_last=dh, dh0=dh)
    assert torch.equal(dgi2, dgi) and torch.equal(dh, dh0)


def test_very_long():
    """Two million chunks, offsets beyond 2^31 bytes.  Where alpha is 0.3 a step, what was 128 steps ago is 1e-67 of itself: windows of steps say what the outputs are."""
    T, heads = (1 << 27) + 77, (1, 1, 1, 1)
    gen = torch.Generator("cuda").manual_seed(5)
    gi = torch.randn(T, 1, 5, device="cuda", dtype=torch.bfloat16, generator=gen)
    bias = torch.tensor([-1.0, 0.0], device="cuda")
    gi[..., 3].clamp_(-1, 0.15)
    o, last, _ = B.delta_fwd(gi, heads, bias, save=False)
    for at in (0, 128 * 64, 2048 * 64 - 20, (1 << 25) + 5, 3 * (1 << 25), (1 << 27) - 60, T - 64):
        begin = max(at - 128, 0)
        want, S, _ = O.delta(gi[begin:at + 64].double().cpu(), heads, bias.double().cpu())
        close(o[at:at + 64], want[at - begin:])
    close(last, S)


@pytest.mark.parametrize("T,N,heads", [(150, 2, (2, 1, 32, 32)), (3100, 1, (2, 2, 16, 16)), (70, 100, (2, 2, 16, 16))])
def test_captured(T, N, heads):
    """Both passes in a graph, replayed with other inputs, eager work between the replays."""
    g = gpu(case(T, N, heads))
    ws = B.Workspace()
    bufs = both(g, heads, ws=ws)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    o, last, saved, dgi, dh0 = bufs
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        B.delta_fwd(g["gi"], heads, g["bias"], h0=g["h0"], o=o, h_last=last, saved=saved, ws=ws)
        B.delta_bwd(g["gi"], saved, heads, g["bias"], do=g["do"], dh_last=g["dh_last"], dgi=dgi, dh0=dh0, ws=ws)
    for seed in range(4):
        other = gpu(case(T, N, heads, seed=10 + seed))
        for k in ("gi", "do", "dh_last", "h0", "bias"):
            g[k].copy_(other[k])
        graph.replay()
        torch.cuda.synchronize()
        want = both(other, heads)
        assert all(torch.equal(a, b) for a, b in zip(bufs, want)), seed


def test_gradients_of_shared_heads_add_up():
    """Three value heads on one key head against three with copies of it."""
    T, N, heads = 100, 2, (3, 1, 16, 24)
    c = case(T, N, heads)
    g = gpu(c)
    q, k, rest = c["gi"][..., :16], c["gi"][..., 16:32], c["gi"][..., 32:]
    spread = dict(c, gi=torch.cat((q, q, q, k, k, k, rest), -1))
    _, _, _, dgi, dh0 = both(g, heads)
    _, _, _, dgi3, dh03 = both(gpu(spread), (3, 3, 16, 24))
    close(dgi[..., 32:], dgi3[..., 96:].double().cpu()), close(dh0, dh03.double().cpu())
    close(dgi[..., :16], dgi3[..., :48].double().cpu().reshape(T, N, 3, 16).sum(2))
    close(dgi[..., 16:32], dgi3[..., 48:96].double().cpu().reshape(T, N, 3, 16).sum(2))


def by_head(x, heads):
    """(name, head, columns) of a row's parts, each head by itself: a head's queries, keys, values and gates."""
    H, Hk, D, Dv = heads
    for name, part, count in zip("qkvab", x.split([Hk * D, Hk * D, H * Dv, H, H], -1), (Hk, Hk, H, H, H)):
        for h, y in enumerate(part.unflatten(-1, (count, -1)).unbind(-2)):
            yield f"d{name} of head {h}", y


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,heads", [(200, (6, 6, 32, 24)), (130, (6, 3, 72, 80)), (64, (6, 2, 16, 40)), (777, (6, 6, 8, 16))])
def test_heads_that_forget(T, heads, dtype):
    """Each head forgets at another rate, from half a step's memory to a millionth: each head's gradients by themselves, down to a gate's, of which next to nothing is left."""
    c = case(T, 2, heads, dtype, lengths=[T, T - 7], seed=3)
    c["bias"][:6] = torch.tensor([1.0, -3.0, -6.0, -9.0, -12.0, -16.0])
    want, got, slack = wanted(c, heads)[3], both(gpu(c), heads)[3], along(c, heads)
    for (name, a), (_, b), (_, more) in zip(by_head(got, heads), by_head(want, heads), by_head(slack, heads)):
        close(a, b, name, more)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_single_gates_that_close(dtype):
    """Single gates close among open ones, at the ends of chunks, of tiles and inside: their gradients by themselves, 1e-5 and less of the open ones'."""
    T, N, heads = 260, 2, (4, 4, 32, 48)
    c = case(T, N, heads, dtype, seed=4)
    c["bias"][:4] = 2.0
    at = [1, 15, 16, 40, 63, 64, 65, 100, 127, 128, 150, 176, 192, 205, 255, 259]
    a = c["gi"][..., -8:-4]
    a[at] = torch.tensor([-10.0, -14.0, -18.0, -22.0]).to(a.dtype)
    want, got = wanted(c, heads)[3], both(gpu(c), heads)[3]
    for (name, x), (_, y) in zip(by_head(got, heads), by_head(want, heads)):
        if name.startswith("da"):
            close(x[at], y[at], name + ", closed"), close(x, y, name)


def of_sequences(c, ns):
    """The case of some of the sequences alone."""
    return {k: v if v is None or k == "bias" else v[:, ns] if k in ("gi", "do") else v[ns] for k, v in c.items()}


def check_some(c, heads, ns, slack=True):
    """check() of some of the sequences, which do not know of each other, and that the others' outputs are numbers."""
    got, part = both(gpu(c), heads), of_sequences(c, ns)
    assert all(bool(torch.isfinite(x).all()) for x in got)
    want, more = wanted(part, heads), along(part, heads) if slack else torch.zeros(part["gi"].shape)
    o, last, saved, dgi, dh0 = got
    for name, a, b in zip(("o", "h_last", "saved", "dh0"), (o[:, ns], last[ns], saved[:, ns], dh0[ns]), (*want[:3], want[4])):
        close(a, b, name)
    for (name, a), (_, b), (_, c) in zip(by_head(dgi[:, ns], heads), by_head(want[3], heads), by_head(more, heads)):
        close(a, b, name, c)


# more than 128 heads of more than 64 columns: eight wavefronts a head, of each type and each number of a head's tiles; just 128: two blocks a head
@pytest.mark.parametrize("T,N,heads,dtype", [(200, 65, (2, 1, 64, 72), "bf16"), (140, 43, (3, 1, 40, 128), "bf16"), (195, 65, (2, 2, 128, 128), "bf16"), (200, 33, (4, 2, 72, 100), "bf16"),
                                             (200, 129, (1, 1, 24, 72), "bf16"), (200, 43, (3, 1, 24, 72), "f32"), (140, 129, (1, 1, 32, 128), "f32"), (200, 65, (2, 1, 64, 100), "f32"),
                                             (195, 33, (4, 2, 128, 128), "f32"), (195, 64, (2, 2, 128, 128), "bf16"), (200, 32, (4, 2, 64, 100), "f32"), (200, 43, (3, 3, 128, 64), "f32"),
                                             (140, 65, (2, 1, 72, 40), "f32")])
def test_many_wide_heads(T, N, heads, dtype):
    lengths = [(37 * n + T // 2) % (T + 1) for n in range(N)]
    lengths[1], lengths[2], lengths[N - 1] = 0, 64, T
    check_some(case(T, N, heads, dtype, lengths=lengths, seed=T + N), heads, [0, 1, 2, N - 1])


# few heads and 48 chunks and more: cut into segments, all widths of a head's tiles, sequences that end in different segments, on their borders and before the first
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,heads,lengths", [(3100, (2, 1, 64, 72), [3100, 1024]), (3201, (1, 1, 100, 128), [2047, 3201]), (3073, (2, 1, 128, 128), [3073, 40]), (3072, (1, 1, 72, 16), [0, 3072]),
                                             (3300, (2, 2, 48, 64), [1025, 3299])])
def test_segments(T, heads, lengths, dtype):
    check_some(case(T, 2, heads, dtype, lengths=lengths, seed=T), heads, [0, 1], slack=False)


def test_offsets_beyond_32_bits():
    """Rows and their gradients of 5.4 GB, outputs of 4.3 GB, whose elements' numbers pass 2^31: windows of steps say what both passes give, as in test_very_long."""
    T, heads = (1 << 27) + 77, (1, 1, 1, 16)
    gen = torch.Generator("cuda").manual_seed(6)
    gi = torch.randn(T, 1, 20, device="cuda", dtype=torch.bfloat16, generator=gen)
    do = torch.randn(T, 1, 16, device="cuda", dtype=torch.bfloat16, generator=gen)
    bias = torch.tensor([-1.0, 0.0], device="cuda")
    gi[..., 18].clamp_(-1, 0.15)
    # (a key of one element is 1 or -1 but for what EPS leaves of it; where it is small its gradient is large beyond measure)
    gi[..., :2] = torch.where(gi[..., :2] < 0, gi[..., :2] - 1, gi[..., :2] + 1)
    o, last, saved = B.delta_fwd(gi, heads, bias)
    dgi, dh0 = B.delta_bwd(gi, saved, heads, bias, do=do)
    assert gi.numel() > 1 << 31 and o.numel() > 1 << 31 and dgi.stride() == gi.stride()
    for at in (0, 2048 * 64 - 20, (1 << 25) + 5, 107374182 - 30, (1 << 26) + 5, 3 * (1 << 25), (1 << 27) - 30, T - 64):
        begin, end = max(at - 128, 0), min(at + 64 + 128, T)
        part = {"gi": gi[begin:end].cpu(), "do": do[begin:end].cpu(), "bias": bias.cpu(), "h0": None, "lengths": None}
        want, slack = wanted(part, heads), along(part, heads)
        here = slice(at - begin, at - begin + 64)
        close(o[at:at + 64], want[0][here], f"o at {at}")
        for (name, a), (_, b), (_, more) in zip(by_head(dgi[at:at + 64], heads), by_head(want[3][here], heads), by_head(slack[here], heads)):
            close(a, b, f"{name} at {at}", more)
    close(last, want[1], "last")
    assert bool(torch.isfinite(dh0).all())

"""Layer norm on the GPU against the 64-bit oracle, on the values as stored.

Bounds, element by element, with u = 2^-24: what a type rounds is off by half a step (bf16 2^-8 of the value, fp32 u); a sum of n floats by at most
n * u of the sum of magnitudes, and the kernels add up at most `chain` values one behind the other in any order; each further float operation by u."""
import numpy as np
import pytest
import torch

from oracle import sequence as S
from paper_2409_11600_amd import binding as B
from parity import guarded, torch_dtype

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
WIDTHS = [1, 2, 7, 8, 64, 65, 130, 256, 257, 512, 768, 1000, 1001, 2048, 2056, 4100, 8192, 8200, 16384, 16385, 40000]


def half(dtype):
    return torch.finfo(torch_dtype(dtype)).eps / 2


def host(t):
    return t.detach().double().cpu().numpy()


def make(seed, rows, C, dtype, offset=0.0):
    g = torch.Generator().manual_seed(seed)
    f = lambda *s: torch.randn(s, generator=g)
    x, res, dy, dsum = ((f(rows, C) + offset).to(torch_dtype(dtype)).cuda() for _ in range(4))
    return x, res, dy, dsum, (1 + 0.3 * f(C)).cuda(), (0.3 * f(C)).cuda()


def in_bound(got, want, bound, what):
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (what, int(bad.sum()), float(np.max(np.abs(got - want)[bad])), float(np.max((np.abs(got - want) / bound)[bad])))


def check_fwd(s, y, mean, invstd, gamma, beta, dtype):
    s, gamma, beta = host(s), host(gamma), host(beta)
    C = s.shape[1]
    want, wmean, winv = S.layernorm_fwd(s, gamma, beta, 1e-5)
    chain = C + 2
    size = np.abs(s).mean(axis=1)
    off_mean = chain * U * size                                 # of the mean, absolute
    in_bound(host(mean), wmean, off_mean + U * np.abs(wmean), "mean")
    var = 1 / winv ** 2 - 1e-5
    # the mean's error shifts each difference (and the variance by its square), differences and squares are rounded, and their sum
    off_var = (chain + 6) * U * var + off_mean ** 2 + 2 * off_mean * np.sqrt(var) * (chain * U) + 2 * U * 1e-5
    rel_inv = 0.5 * off_var * winv ** 2 * (1 + off_var * winv ** 2) + 4 * U
    in_bound(host(invstd), winv, rel_inv * winv, "invstd")
    xh = np.abs(s - wmean[:, None]) * winv[:, None]
    bound = half(dtype) * np.abs(want) + 1.02 * (np.abs(gamma) * (xh * (rel_inv[:, None] + 4 * U) + (off_mean * winv)[:, None]) + 2 * U * (np.abs(beta) + xh * np.abs(gamma)))
    in_bound(host(y), want, bound + 1e-38, "y")


@pytest.mark.parametrize("C", WIDTHS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_forward(C, dtype):
    for rows in (1, 3, 70) if C <= 8200 else (1, 5):
        print(f"layer norm forward rows={rows} C={C} {dtype}", flush=True)
        x, res, _, _, gamma, beta = make(C + rows, rows, C, dtype)
        y, y_ok = guarded((rows, C), x.dtype)
        s, s_ok = guarded((rows, C), x.dtype)
        _, got_s, mean, invstd = B.layernorm_fwd(x, gamma, beta, residual=res, out=y, sum_out=s)
        assert got_s is s
        y_ok(), s_ok()
        exact = host(x) + host(res)
        in_bound(host(s), exact, half(dtype) * np.abs(exact) * (1 + 2.0 ** -8) + U * np.abs(exact), "sum")
        check_fwd(s, y, mean, invstd, gamma, beta, dtype)
        # the same without a place for the sum, and in place of the residual
        y2, none, m2, _ = B.layernorm_fwd(x, gamma, beta, residual=res, save=False)
        assert none is None and m2 is None and torch.equal(y2, y)
        y3, _, _, _ = B.layernorm_fwd(x, gamma, beta, residual=res, sum_out=res)
        assert torch.equal(y3, y) and torch.equal(res, s)
        # and without a residual, on what was the sum
        y4, s4, m4, i4 = B.layernorm_fwd(s, gamma, beta)
        assert s4 is s and torch.equal(y4, y) and torch.equal(m4, mean) and torch.equal(i4, invstd)


@pytest.mark.parametrize("C", WIDTHS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_backward(C, dtype):
    for rows in (1, 3, 70, 700) if C <= 8200 else (1, 40):
        print(f"layer norm backward rows={rows} C={C} {dtype}", flush=True)
        s, _, dy, dsum, gamma, beta = make(C + 7 * rows, rows, C, dtype)
        _, _, mean, invstd = B.layernorm_fwd(s, gamma, beta)
        dx, dx_ok = guarded((rows, C), s.dtype)
        dgamma, dg_ok = guarded((C,), torch.float32)
        dbeta, db_ok = guarded((C,), torch.float32)
        B.layernorm_bwd(dy, s, gamma, mean, invstd, dsum=dsum, dx=dx, dgamma=dgamma, dbeta=dbeta)
        dx_ok(), dg_ok(), db_ok()
        hs, hd, hg, hm, hi = host(s), host(dy), host(gamma), host(mean), host(invstd)
        want, wg, wb = S.layernorm_bwd(hd, hs, hg, hm, hi, host(dsum))
        xh, gh = (hs - hm[:, None]) * hi[:, None], hd * hg
        a, b = np.abs(gh).mean(axis=1, keepdims=True), np.abs(gh * xh).mean(axis=1, keepdims=True)
        chain = C + 8
        parts = hi[:, None] * ((np.abs(gh) + np.abs(xh) * b) * 8 * U + chain * U * (a + np.abs(xh) * b)) + 2 * U * np.abs(host(dsum))
        in_bound(host(dx), want, half(dtype) * np.abs(want) + 1.02 * parts + U * np.abs(want) + 1e-38, "dx")
        in_bound(host(dgamma), wg, (rows + 6) * U * np.abs(hd * xh).sum(axis=0) + 1e-38, "dgamma")
        in_bound(host(dbeta), wb, (rows + 2) * U * np.abs(hd).sum(axis=0) + 1e-38, "dbeta")
        # the same without the gradients of gamma and beta, without dsum, and in its place
        dx2, none, _ = B.layernorm_bwd(dy, s, gamma, mean, invstd, dsum=dsum, want_affine=False)
        assert none is None and torch.equal(dx2, dx)
        before = dsum.clone()
        B.layernorm_bwd(dy, s, gamma, mean, invstd, dsum=dsum, dx=dsum, want_affine=False)
        assert torch.equal(dsum, dx)
        dx3, g3, b3 = B.layernorm_bwd(dy, s, gamma, mean, invstd)
        assert torch.equal(g3, dgamma) and torch.equal(b3, dbeta)
        in_bound(host(dx3), want - host(before), half(dtype) * np.abs(want - host(before)) + 1.02 * parts + U * np.abs(want) + 1e-38, "dx without dsum")
        # added to what is there
        B.layernorm_bwd(dy, s, gamma, mean, invstd, dx=dx, dgamma=g3, dbeta=b3, accumulate=True)
        in_bound(host(g3), 2 * host(dgamma), 2 * U * np.abs(2 * host(dgamma)) + 1e-38, "dgamma, twice")
        in_bound(host(b3), 2 * host(dbeta), 2 * U * np.abs(2 * host(dbeta)) + 1e-38, "dbeta, twice")


@pytest.mark.parametrize("rows", [255, 4097, 20011])
def test_many_rows(rows):
    """Rows that are not whole shares; the sums over them against 64 bits, and the same again bit by bit."""
    for dtype, C in (("f32", 24), ("bf16", 72), ("bf16", 19), ("f32", 256)):
        s, _, dy, _, gamma, beta = make(rows, rows, C, dtype)
        y, _, mean, invstd = B.layernorm_fwd(s, gamma, beta)
        check_fwd(s, y, mean, invstd, gamma, beta, dtype)
        got = B.layernorm_bwd(dy, s, gamma, mean, invstd)
        again = B.layernorm_bwd(dy, s, gamma, mean, invstd)
        assert all(torch.equal(a, b) for a, b in zip(got, again))
        hs, hd = host(s), host(dy)
        _, wg, wb = S.layernorm_bwd(hd, hs, host(gamma), host(mean), host(invstd))
        xh = (hs - host(mean)[:, None]) * host(invstd)[:, None]
        in_bound(host(got[1]), wg, (rows + 6) * U * np.abs(hd * xh).sum(axis=0), "dgamma")
        in_bound(host(got[2]), wb, (rows + 2) * U * np.abs(hd).sum(axis=0), "dbeta")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [65, 512, 20000])
def test_far_from_zero_and_constant(C, dtype):
    """A mean a thousand times the spread (the variance is that of the differences), and rows without any spread: y is beta."""
    x, _, _, _, gamma, beta = make(5, 9, C, dtype, offset=1000.0)
    y, _, mean, invstd = B.layernorm_fwd(x, gamma, beta)
    check_fwd(x, y, mean, invstd, gamma, beta, dtype)
    flat = torch.full((3, C), 0.5, dtype=x.dtype, device="cuda:0")
    y, _, mean, invstd = B.layernorm_fwd(flat, gamma, beta)
    assert torch.equal(mean, torch.full_like(mean, 0.5)) and torch.equal(y, beta.to(x.dtype).expand(3, C))
    in_bound(host(invstd), np.full(3, 1 / np.sqrt(np.float64(np.float32(1e-5)))), 4 * U * 317, "invstd")


@pytest.mark.parametrize("C", [30, 256, 12000])
def test_infinities_and_nan_stay_in_their_rows(C):
    for dtype in ("f32", "bf16"):
        x, res, dy, _, gamma, beta = make(11, 12, C, dtype)
        y0, _, mean, invstd = B.layernorm_fwd(x, gamma, beta)
        dx0 = B.layernorm_bwd(dy, x, gamma, mean, invstd)[0]
        bad = x.clone()
        bad[3, C // 2], bad[7, 0], bad[8, C - 1] = float("inf"), float("nan"), torch.finfo(x.dtype).min
        y, _, m2, i2 = B.layernorm_fwd(bad, gamma, beta)
        dx = B.layernorm_bwd(dy, bad, gamma, m2, i2)[0]
        rest = [r for r in range(12) if r not in (3, 7, 8)]
        assert torch.equal(y[rest], y0[rest]) and torch.equal(dx[rest], dx0[rest])
        assert y[3].isnan().any() and y[7].isnan().all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [1, 3, 5, 13, 31, 64, 65, 130, 200])
def test_constant_rows_of_very_large_values(C, dtype):
    """Rows whose mean times invstd is beyond the largest float though no difference from the mean is (their values a power of two, whose sum and mean are exact; a single column
    also of the type's lowest value): xh is 0, and dx what the means of dy * gamma leave.  Lanes without a part of the row must not put anything into its sums."""
    _, _, dy, dsum, gamma, beta = make(31, 6, C, dtype)
    top = 2.0 ** 120 if C > 1 else torch.finfo(torch_dtype(dtype)).min
    s = torch.full((6, C), top, dtype=dy.dtype, device="cuda:0")
    s[1], s[4] = -top, 1.0
    y, _, mean, invstd = B.layernorm_fwd(s, gamma, beta)
    assert torch.equal(mean, s[:, 0].float()) and torch.equal(y, beta.to(s.dtype).expand(6, C))
    dx, dgamma, dbeta = B.layernorm_bwd(dy, s, gamma, mean, invstd, dsum=dsum)
    hd, hg, hi = host(dy), host(gamma), host(invstd)
    want, wg, wb = S.layernorm_bwd(hd, host(s), hg, host(mean), hi, host(dsum))
    gh = np.abs(hd * hg)
    parts = hi[:, None] * (gh * 8 * U + (C + 8) * U * gh.mean(axis=1, keepdims=True)) + 2 * U * np.abs(host(dsum))
    in_bound(host(dx), want, half(dtype) * np.abs(want) + 1.02 * parts + U * np.abs(want) + 1e-38, "dx")
    assert not wg.any() and not dgamma.any()
    in_bound(host(dbeta), wb, 8 * U * np.abs(hd).sum(axis=0), "dbeta")


@pytest.mark.parametrize("rows,C", [((1 << 31) // 1000 + 40, 1000), ((1 << 22) + 100, 264)])
def test_many_elements_and_many_rows(rows, C):
    """More than 2^31 elements, 2^32 bytes; and more rows than blocks are launched for: the last rows against the same alone."""
    x = torch.zeros((rows, C), dtype=torch.bfloat16, device="cuda:0")
    x[:8].normal_()
    x[-8:].normal_()
    gamma, beta = torch.randn(C, device="cuda:0"), torch.randn(C, device="cuda:0")
    y, _, mean, invstd = B.layernorm_fwd(x, gamma, beta)
    dx, _, _ = B.layernorm_bwd(y, x, gamma, mean, invstd)
    for part in (slice(0, 8), slice(rows - 8, rows)):
        y2, _, m2, i2 = B.layernorm_fwd(x[part].clone(), gamma, beta)
        dx2, _, _ = B.layernorm_bwd(y2, x[part].clone(), gamma, m2, i2)
        assert torch.equal(y[part], y2) and torch.equal(mean[part], m2) and torch.equal(invstd[part], i2) and torch.equal(dx[part], dx2)


def test_no_affine_part():
    x, _, dy, _, gamma, _ = make(1, 33, 100, "f32")
    one, zero = torch.ones_like(gamma), torch.zeros_like(gamma)
    a, b = B.layernorm_fwd(x, None, None), B.layernorm_fwd(x, one, zero)
    assert torch.equal(a[0], b[0])
    assert torch.equal(B.layernorm_bwd(dy, x, None, a[2], a[3])[0], B.layernorm_bwd(dy, x, one, a[2], a[3])[0])
    only = torch.empty_like(gamma)
    both = B.layernorm_bwd(dy, x, one, a[2], a[3])
    B.layernorm_bwd(dy, x, one, a[2], a[3], dbeta=only, want_affine=False)
    assert torch.equal(only, both[2])


def test_gradient_against_differences():
    """dx of the kernel against differences of the kernel's own forward pass: the loss is a sum of dy * y in 64 bits; with a step of 2^-7 the second
    difference's error is h^2 / 6 of a third derivative (below 30 for rows with a spread of about one), the rounding's 2 * u * |y| * |dy| * C / 2h."""
    rows, C, h = 2, 12, 2.0 ** -7
    x, _, dy, _, gamma, beta = make(21, rows, C, "f32")
    _, _, mean, invstd = B.layernorm_fwd(x, gamma, beta)
    dx, dgamma, _ = B.layernorm_bwd(dy, x, gamma, mean, invstd)
    loss = lambda a, g: float((B.layernorm_fwd(a, g, beta)[0].double() * dy.double()).sum())
    size = float((dy.abs().double() * (B.layernorm_fwd(x, gamma, beta)[0].abs().double() + 1)).sum())
    for i in np.ndindex(rows, C):
        e = torch.zeros_like(x)
        e[i] = h
        d = (loss(x + e, gamma) - loss(x - e, gamma)) / (2 * h)
        assert abs(d - float(dx[i])) <= h * h / 6 * 30 * float(dy.abs().max()) + 16 * U * size / h, i
    for c in range(C):
        e = torch.zeros_like(gamma)
        e[c] = h
        d = (loss(x, gamma + e) - loss(x, gamma - e)) / (2 * h)
        assert abs(d - float(dgamma[c])) <= 16 * U * size / h, c


def test_on_a_stream_and_in_a_graph():
    """Work on a stream of its own, and a captured pass replayed on new values between eager calls."""
    x, res, dy, _, gamma, beta = make(2, 500, 96, "bf16")
    ws = B.Workspace("cuda:0")
    bufs = [torch.empty_like(x) for _ in range(3)] + [torch.empty(500, device="cuda:0") for _ in range(2)] + [torch.empty(96, device="cuda:0") for _ in range(2)]

    def step():
        y, s, dx, mean, invstd, dg, db = bufs
        B.layernorm_fwd(x, gamma, beta, residual=res, out=y, sum_out=s, save_mean=mean, save_invstd=invstd)
        B.layernorm_bwd(dy, s, gamma, mean, invstd, dx=dx, dgamma=dg, dbeta=db, ws=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        x.copy_(torch.randn(x.shape, device="cuda:0").to(x.dtype))
        graph.replay()
        torch.cuda.synchronize()
        got = [b.clone() for b in bufs]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, bufs)), k

"""AdamW with 8-bit moments on the GPU: the moments bit by bit those of the oracle's float32 step (the operations that decide them are single float
operations, each rounded to nearest), the weights to a few of its roundings, and what the rounding at random is for."""
import numpy as np
import pytest
import torch

from oracle import sequence as S
from paper_2409_11600_amd import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8)


def values(t):
    return S.e4m3_values()[t.view(torch.uint8).cpu().numpy()]


class Tensors:
    """Tensors with their state, each kind in one buffer with canaries around and between them."""

    def __init__(self, sizes, seed, copy=True, gap=256):
        self.sizes, r = sizes, np.random.default_rng(seed)
        at, self.at, bat, self.bat = gap, [], 16, []
        for n in sizes:
            self.at.append(at)
            self.bat.append(bat)
            at += -(-n // 256) * 256 + gap
            bat += -(-n // 256) + 3
        dev = lambda a: torch.from_numpy(a).cuda()
        self.w, self.g = dev(r.normal(size=at).astype(np.float32)), dev((r.normal(size=at) * 10.0 ** r.uniform(-6, 0, at)).astype(np.float32))
        code = lambda top: dev(r.integers(0, top, at).astype(np.uint8))
        self.m, self.r = code(256).view(torch.uint8), code(127)
        self.m[(self.m & 127) == 127] = 0
        self.r[self.r == 0] = 1
        pw = lambda: dev((2.0 ** r.integers(-20, -10, bat)).astype(np.float32))
        self.sm, self.sr, self.lp = pw(), pw(), self.w.to(torch.bfloat16) if copy else None
        self.before = [None if t is None else t.clone() for t in self.all()]

    def all(self):
        return [self.w, self.g, self.m, self.r, self.sm, self.sr, self.lp]

    def part(self, k, tensors=None):
        w, g, m, r, sm, sr, lp = tensors or self.all()
        n, a, b = self.sizes[k], self.at[k], self.bat[k]
        cut, blocks = slice(a, a + n), slice(b, b + -(-n // 256))
        return w[cut], g[cut], m[cut].view(torch.float8_e4m3fn), r[cut].view(torch.float8_e4m3fn), sm[blocks], sr[blocks], None if lp is None else lp[cut]

    def table(self, decays):
        return B.param8_table((*self.part(k), decays[k % len(decays)]) for k in range(len(self.sizes)))

    def check(self, step, seed, decays, scale=1.0):
        for k, n in enumerate(self.sizes):
            w, g, m, r, sm, sr, lp = self.part(k, self.before)
            ww, qm, qr, wsm, wsr, mn, rn = S.adamw8_step(w.cpu().numpy(), g.cpu().numpy(), values(m), values(r), sm.cpu().numpy(), sr.cpu().numpy(), step, seed, k,
                                                         weight_decay=decays[k % len(decays)], grad_scale=scale, **HYPER)
            gw, gg, gm, gr, gsm, gsr, glp = self.part(k)
            assert np.array_equal(gsm.cpu().numpy(), wsm) and np.array_equal(gsr.cpu().numpy(), wsr), (k, n)
            assert np.array_equal(values(gm), qm, equal_nan=True) and np.array_equal(values(gr), qr, equal_nan=True), (k, n)
            assert not gg.any()
            step_size = np.abs(ww.astype(np.float64) - w.cpu().numpy())
            got = gw.double().cpu().numpy()
            # the update's quotient to four roundings, and one each of the decayed weight and of the difference
            assert (np.abs(got - ww) <= 4 * U * (np.abs(ww) + step_size) + 6 * U * step_size + 1e-37).all(), (k, n)
            if glp is not None:
                assert torch.equal(glp, gw.to(torch.bfloat16))
        # nothing between the tensors has changed
        inside = torch.zeros_like(self.w, dtype=torch.bool)
        blocks = torch.zeros_like(self.sm, dtype=torch.bool)
        for a, b, n in zip(self.at, self.bat, self.sizes):
            inside[a:a + n] = True
            blocks[b:b + -(-n // 256)] = True
        for now, old, mask in zip(self.all(), self.before, [inside] * 4 + [blocks] * 2 + [inside]):
            assert now is None or torch.equal(now[~mask], old[~mask])


@pytest.mark.parametrize("sizes", [[1], [3], [255], [256], [257], [1023, 1, 4096], [5, 700, 256, 31, 100000], [64] * 45, [300 + k for k in range(90)], [1 << 20]])
@pytest.mark.parametrize("copy", [False, True])
def test_step(sizes, copy):
    print(f"adamw8 {len(sizes)} tensors, first {sizes[0]}, copy {copy}", flush=True)
    t = Tensors(sizes, len(sizes) + sizes[0], copy)
    decays = [0.0, 1e-2, 0.3]
    scale = torch.full((1,), 0.37, device="cuda:0")
    B.adamw8_step_multi(t.table(decays), 11, 0xDEADBEEF, grad_scale=scale, **HYPER)
    torch.cuda.synchronize()
    t.check(11, 0xDEADBEEF, decays, 0.37)


def test_from_nothing():
    """The first step of a state of zeros moves a weight by lr against its gradient's sign; a zero gradient moves nothing and leaves zeros."""
    n = 1000
    g = torch.randn(n, device="cuda:0")
    g[::7] = 0
    w = torch.randn(n, device="cuda:0")
    w0, g0, state = w.clone(), g.clone(), B.adamw8_state(n)
    B.adamw8_step_multi(B.param8_table([(w, g, *state, None, 0.0)]), 1, 3, **HYPER)
    assert torch.equal(w[::7], w0[::7]) and (values(state[0])[::7] == 0).all() and (values(state[1])[::7] == 0).all()
    moved = (w0 - w).double().cpu().numpy()
    # the step's quotient is 1 to eps / |g| and a few roundings; w is rounded twice
    g64 = np.abs(g0.double().cpu().numpy())
    assert (np.abs(moved - 1e-3 * np.sign(g0.cpu().numpy())) <= 1e-3 * (1e-8 / np.maximum(g64, 1e-30) + 40 * U) * (g64 > 0) + 2 * U * np.abs(w0.cpu().numpy())).all()
    # a state and gradients of nothing, again and again
    for k in range(2, 5):
        g.zero_()
        B.adamw8_step_multi(B.param8_table([(w, g, *state, None, 0.0)]), k, k, **HYPER)
    assert torch.isfinite(w).all() and torch.equal(w[::7], w0[::7])


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_what_is_not_finite_stays_with_its_element(bad):
    t, clean = Tensors([1000], 6), Tensors([1000], 6)
    at = t.at[0] + 300
    t.g[at] = bad
    clean.g[at] = 0
    for x in (t, clean):
        B.adamw8_step_multi(x.table([0.0]), 5, 8, **HYPER)
    keep = torch.ones(1000, dtype=torch.bool, device="cuda:0")
    keep[300] = False
    for k, (a, b) in enumerate(zip(t.part(0), clean.part(0))):
        a, b = a.float(), b.float()
        if k in (4, 5):
            assert torch.equal(a, b) and torch.isfinite(a).all()
        else:
            assert torch.equal(a[keep], b[keep])
    assert not torch.isfinite(t.part(0)[0][300]) and np.isnan(values(t.part(0)[3])[300])


def test_tiny_and_huge_gradients():
    """From denormal gradients to ones whose squares overflow: what the oracle's float step gives, and an r above zero is never held as zero."""
    t = Tensors([2048], 9)
    g = t.part(0)[1]
    g[:512] *= 1e-38
    g[512:1024] *= 1e-20
    g[1024:1536] *= 1e18
    g[1536:] *= 1e25
    t.before[1] = t.g.clone()
    B.adamw8_step_multi(t.table([0.0]), 3, 4, **HYPER)
    t.check(3, 4, [0.0])
    r = values(t.part(0)[3])
    assert (r[np.isfinite(r)] > 0).all()


def test_a_tensor_beyond_32_bits():
    """More than 2^32 elements: the last ones move, and are held, as their indexes say; the others, without a gradient, stay."""
    end = 700
    n = (1 << 32) + end
    w, g = torch.zeros(n, device="cuda:0"), torch.zeros(n, device="cuda:0")
    state = B.adamw8_state(n)
    r = np.random.default_rng(8)
    w0, g0 = r.normal(size=end).astype(np.float32), r.normal(size=end).astype(np.float32)
    w[-end:], g[-end:] = torch.from_numpy(w0).cuda(), torch.from_numpy(g0).cuda()
    B.adamw8_step_multi(B.param8_table([(w, g, *state, None, 0.0)]), 1, 77, **HYPER)
    torch.cuda.synchronize()
    i = np.arange(n - end, n, dtype=np.uint64)          # (the last 700 begin a block: 2^32 is whole blocks)
    u = S.mix(i * np.uint64(0x9E3779B9) + (i >> np.uint64(32)) * np.uint64(0x85A308D3) + S.mix(77))
    zero, scales = np.zeros(end), np.zeros(3)
    _, _, _, sm, sr, mn, rn = S.adamw8_step(w0, g0, zero, zero, scales, scales, 1, 0, 0, weight_decay=0.0, **HYPER)
    want_m = S.held(mn, sm, (u & np.uint64(0xFFFF)).astype(np.float64))
    want_r = S.held(rn, sr, (u >> np.uint64(16)).astype(np.float64))
    want_r = np.where((rn > 0) & (want_r < 2.0 ** -9), 2.0 ** -9, want_r)
    assert np.array_equal(values(state[0][-end:]), want_m) and np.array_equal(values(state[1][-end:]), want_r)
    assert np.array_equal(state[2][-3:].cpu().numpy(), sm) and not w[:-end].any() and not state[1][:-end].view(torch.uint8).any()


def test_rounding_has_the_right_mean():
    """Held moments, averaged over seeds, are the moments: the mean of K roundings is off by less than 6 / (2 sqrt K) of a place (its standard deviation is half a
    place at most)."""
    n, K = 512, 400
    r = np.random.default_rng(2)
    g = torch.from_numpy(r.normal(size=n).astype(np.float32)).cuda()
    zero = B.adamw8_state(n)
    total_m, total_r = np.zeros(n), np.zeros(n)
    for seed in range(K):
        w, gg = torch.zeros(n, device="cuda:0"), g.clone()
        state = [t.clone() for t in zero]
        B.adamw8_step_multi(B.param8_table([(w, gg, *state, None, 0.0)]), 1, seed, **HYPER)
        total_m += values(state[0]) * np.repeat(state[2].cpu().numpy(), 256)
        total_r += values(state[1]) * np.repeat(state[3].cpu().numpy(), 256)
    _, _, _, sm, sr, mn, rn = S.adamw8_step(np.zeros(n), g.cpu().numpy(), np.zeros(n), np.zeros(n), np.zeros(2), np.zeros(2), 1, 0, 0, weight_decay=0.0, **HYPER)
    for total, x, scales in ((total_m, mn, sm), (total_r, rn, sr)):
        place = np.maximum(2.0 ** (np.floor(np.log2(np.maximum(np.abs(x) / np.repeat(scales, 256), 2.0 ** -6))) - 3), 2.0 ** -9) * np.repeat(scales, 256)
        assert (np.abs(total / K - x) <= (3 / np.sqrt(K) + 2.0 ** -15) * place).all()


def test_training_with_it_goes_as_with_32_bits():
    """A quadratic with noisy gradients: after 400 steps the mean distance is that of the 32-bit step within a quarter, and r has followed a gradient that became a
    hundred times smaller (rounded to nearest it could not)."""
    n = 8192
    gen = torch.Generator(device="cuda").manual_seed(3)
    target = torch.randn(n, device="cuda:0", generator=gen)
    w8, w32 = torch.zeros(n, device="cuda:0"), torch.zeros(n, device="cuda:0")
    g8, g32, m, v = (torch.zeros(n, device="cuda:0") for _ in range(4))
    state = B.adamw8_state(n)
    tab = B.param8_table([(w8, g8, *state, None, 0.0)])
    for k in range(1, 401):
        noise = 0.1 * torch.randn(n, device="cuda:0", generator=gen)
        g8.copy_(w8 - target + noise)
        g32.copy_(w32 - target + noise)
        B.adamw8_step_multi(tab, k, 1000 + k, 1e-2)
        B.adamw_step(w32, g32, m, v, k, 1e-2)
    d8, d32 = float((w8 - target).abs().mean()), float((w32 - target).abs().mean())
    assert d8 <= 1.25 * d32, (d8, d32)
    tiny, r0 = 1e-3, None
    for k in range(401, 2401):
        g8.fill_(tiny)
        B.adamw8_step_multi(tab, k, 1000 + k, 0.0)
        if k == 401:
            r0 = state[1].float() * state[3].repeat_interleave(256)
    r1 = state[1].float() * state[3].repeat_interleave(256)
    # 2000 steps take v to 0.999^2000 = 0.135 of itself, r to 0.37
    assert 0.30 <= float(r1.mean() / r0.mean()) <= 0.44


def test_on_a_stream_and_in_a_graph():
    t = Tensors([700, 33, 5000], 12)
    tab = t.table([1e-2])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.adamw8_step_multi(tab, 2, 5, **HYPER)
    torch.cuda.current_stream().wait_stream(side)
    t.check(2, 5, [1e-2])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.adamw8_step_multi(tab, 2, 5, **HYPER)
    for k in range(3):
        for now, old in zip(t.all(), t.before):
            now.copy_(old)
        graph.replay()
        torch.cuda.synchronize()
        t.check(2, 5, [1e-2])

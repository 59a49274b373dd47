"""The loss against a teacher's top logits, against oracle/learning.py in 64 bits; its gradient against torch's of that form.

Tolerances.  A row's sum of K exponentials is made of at most K / 256 / 8 + 40 additions one after the other, each exponential within 3 units of 2^-24 (the argument's rounding counts with the
argument, which is large only where the exponential is small): relative 2^-24 * (K / 2048 + 50) at most, 2^-24 * sqrt(K / 2048 + 50) as such roundings add up; 64 * 2^-24 holds both up to K = 131072.  The
loss adds p * (differences of logarithms) of up to 30: 30 * 4 * 2^-24 a place, taken relative to the largest row.  A gradient is rounded to its type once more: half a step, 2^-8 in bf16."""
import math

import pytest
import torch

from oracle import learning as O
from paper_2409_11600_amd import binding as B

pytestmark = pytest.mark.gpu
F32 = 64 * 2.0 ** -24
LOSS = 128 * 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def case(N, K, M, dtype="f32", seed=0, ld=None, weights=None, gone=False):
    gen = torch.Generator().manual_seed(seed)
    buf = torch.full((N, ld or K), 9.0, dtype=TYPES[dtype])
    buf[:, :K] = (2 * torch.randn(N, K, generator=gen)).to(TYPES[dtype])
    index = torch.randint(0, K, (N, M), generator=gen, dtype=torch.int32)          # (the same index may come twice)
    if gone:
        index[torch.rand(N, M, generator=gen) < 0.4] = -1
        index[0] = -7
    w = None if weights is None else torch.where(torch.rand(N, generator=gen) < 0.4, torch.zeros(N), torch.rand(N, generator=gen) + 0.1) if weights == "some" else torch.zeros(N)
    return buf, index, 3 * torch.randn(N, M, generator=gen), w


def wanted(z, index, teacher, tau, w, dloss):
    z = z.double().requires_grad_(True)
    loss, rows = O.distill(z, index, teacher.double(), tau, None if w is None else w.double())
    grad = torch.autograd.grad(dloss * loss, z)[0] if loss.requires_grad else torch.zeros_like(z)
    return loss.detach(), rows.detach(), grad


def check(buf, index, teacher, w, K, tau=1.5, dloss=0.7, accumulate=False, in_place=False):
    z = buf[:, :K]
    loss, rows, grad = wanted(z, index, teacher, tau, w, dloss)
    gbuf, gi, gt, gw = buf.cuda(), index.cuda(), teacher.cuda(), None if w is None else w.cuda()
    gz = gbuf[:, :K]
    got, per_row, saved = B.distill_fwd(gz, gi, gt, tau=tau, weights=gw)
    top = max(rows.abs().max().item(), 1e-3)
    assert (per_row.double().cpu() - rows).abs().max() <= LOSS * max(top, 30)
    assert abs(got.item() - loss.item()) <= LOSS * max(top, 30)
    total = float(len(z)) if w is None else w.double().sum().item()
    assert abs(saved[-1, 0].item() - total) <= 2.0 ** -20 * max(total, 1)
    half = 2.0 ** -8 if buf.dtype == torch.bfloat16 else 0.0
    before = None
    if in_place:
        out = B.distill_bwd(gz, gi, gt, saved, tau=tau, dloss=dloss, weights=gw, out=gz)
        obuf = gbuf
    else:
        obuf = torch.full_like(gbuf, 5.0)
        if accumulate:
            obuf[:, :K] = torch.randn(obuf[:, :K].shape, device="cuda", generator=torch.Generator("cuda").manual_seed(3)).to(obuf.dtype) * 1e-3
            before = obuf[:, :K].double().cpu()
        out = B.distill_bwd(gz, gi, gt, saved, tau=tau, dloss=dloss, weights=gw, out=obuf[:, :K], accumulate=accumulate)
    want = grad if before is None else grad + before
    # q and p are within F32 of themselves, their difference is not: scale by the row's largest of the two
    c = (torch.full((len(z),), 1 / len(z), dtype=torch.float64) if w is None else w.double() / max(total, 1e-30)) * abs(dloss) * tau
    far = (out.double().cpu() - want).abs()
    assert bool((far <= F32 * c[:, None] + half * want.abs() + (2.0 ** -24 * want.abs()) + 1e-37).all()), (far.max(), c.max())
    if K < buf.shape[1]:
        assert bool((obuf[:, K:] == (9 if in_place else 5)).all())
    return out


# few rows and many, rows of one block and of several, odd widths, rows with room between them
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,K,M,ld", [(1, 2, 1, None), (3, 1, 2, None), (5, 64, 3, None), (4, 1001, 40, None), (7, 1001, 16, 1010), (2, 50001, 300, None), (1, 131072, 64, None), (1200, 333, 7, 335),
                                      (3, 9000, 1024, 9001)])
def test_sizes(N, K, M, ld, dtype):
    buf, index, teacher, _ = case(N, K, M, dtype, seed=K, ld=ld)
    check(buf, index, teacher, None, K)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("how", ["accumulate", "in place", "plain"])
@pytest.mark.parametrize("weights", ["some", "none of them", None])
def test_weights_and_places(weights, how, dtype):
    for N, K, M in ((6, 700, 9), (2, 40000, 33)):
        buf, index, teacher, w = case(N, K, M, dtype, seed=N, weights=weights, gone=True)
        check(buf, index, teacher, w, K, accumulate=how == "accumulate", in_place=how == "in place")


def test_many_rows():
    """More than one block's share of the loss."""
    buf, index, teacher, w = case(70001, 16, 2, weights="some")
    check(buf, index, teacher, w, 16)


def test_rows_without_weight_are_not_read():
    buf, index, teacher, _ = case(4, 500, 5)
    w = torch.tensor([1.0, 0.0, 2.0, 0.0])
    want = check(buf, index, teacher, w, 500)
    buf[1], teacher[3], index[3, 0] = math.nan, math.inf, 5000
    loss, per_row, saved = B.distill_fwd(buf.cuda(), index.cuda(), teacher.cuda(), tau=1.5, weights=w.cuda())
    assert bool(torch.isfinite(loss).all()) and not per_row[[1, 3]].any() and not saved[[1, 3]].any()
    assert torch.equal(B.distill_bwd(buf.cuda(), index.cuda(), teacher.cuda(), saved, tau=1.5, dloss=0.7, weights=w.cuda()), want)


def test_rows_without_a_place():
    """Loss and gradient 0, whatever the logits hold."""
    buf, index, teacher, _ = case(3, 300, 4)
    index[1] = -1
    buf[1] = math.nan
    loss, per_row, saved = B.distill_fwd(buf.cuda(), index.cuda(), teacher.cuda())
    assert per_row[1] == 0 and bool(torch.isfinite(loss).all())
    out = B.distill_bwd(buf.cuda(), index.cuda(), teacher.cuda(), saved)
    assert not out[1].any() and bool(torch.isfinite(out).all())


def test_infinities_and_wrong_indices():
    buf, index, teacher, _ = case(6, 400, 5)
    index[:] = torch.arange(5, dtype=torch.int32) * 7
    buf[0, 50:] = -math.inf                         # masked words
    buf[1, 7] = -math.inf                           # one that the teacher says
    teacher[2, 1:] = -math.inf                      # a teacher that is sure
    index[3, 2] = 400                               # no such word
    buf[4, 3] = math.nan
    buf[5] = -math.inf
    loss, per_row, saved = B.distill_fwd(buf.cuda(), index.cuda(), teacher.cuda())
    rows = O.distill_rows(buf[:3].double(), index[:3], teacher[:3].double())
    assert abs(per_row[0].item() - rows[0].item()) <= LOSS * 30 and abs(per_row[2].item() - rows[2].item()) <= LOSS * 30
    assert per_row[1] == math.inf and bool(per_row[3:].isnan().all()) and bool(loss.isnan().all())
    out = B.distill_bwd(buf.cuda(), index.cuda(), teacher.cuda(), saved).double().cpu()
    q = torch.softmax(buf[:3].double(), 1)
    p = torch.zeros(3, 400, dtype=torch.float64).scatter_add(1, index[:3].long(), torch.softmax(teacher[:3].double(), 1))
    assert (out[:3] - (q - p) / 6).abs().max() <= F32 / 6
    assert not out[0, 50:].any() and bool(out[3:].isnan().all())


def test_the_same_index_many_times():
    """Its places add up, in their order: the same bits each time."""
    buf, index, teacher, _ = case(2, 100, 60)
    index[:] = 17
    index[1, ::2] = 99
    a = check(buf, index, teacher, None, 100)
    for _ in range(5):
        assert torch.equal(a, check(buf, index, teacher, None, 100))


@pytest.mark.parametrize("tau", [0.05, 1.0, 30.0])
def test_temperatures(tau):
    buf, index, teacher, _ = case(5, 900, 20)
    z = buf.double().requires_grad_(True)
    loss, rows = O.distill(z, index, teacher.double(), tau)
    (grad,) = torch.autograd.grad(loss, z)
    got, per_row, saved = B.distill_fwd(buf.cuda(), index.cuda(), teacher.cuda(), tau=tau)
    # differences of up to 20 / tau in the exponents, each within 2^-24 of itself, and tau^2 of their mean
    tol = 2.0 ** -24 * (64 + 40 / tau)
    assert (per_row.double().cpu() - rows.detach()).abs().max() <= tol * tau * tau * max(30, 40 / tau)
    out = B.distill_bwd(buf.cuda(), index.cuda(), teacher.cuda(), saved, tau=tau)
    assert (out.double().cpu() - grad).abs().max() <= tol * tau / 5


@pytest.mark.parametrize("K", [50, 40000])
def test_large_logits(K):
    """Far from 0 (3e4 units of tau, where neighbours are 0.002 apart), only the differences count."""
    buf, index, teacher, _ = case(3, K, 9)
    check(buf + 20000, index, teacher - 20000, None, K, tau=0.7)


def test_captured():
    bufs = [tuple(x.cuda() for x in case(9, 5000, 12, "bf16", seed=s, weights="some")) for s in range(4)]
    z, index, teacher, w = (x.clone() for x in bufs[0])
    ws = B.Workspace()
    loss, rows, saved = B.distill_fwd(z, index, teacher, weights=w, ws=ws)
    out = torch.empty_like(z)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        B.distill_fwd(z, index, teacher, weights=w, per_row=rows, loss=loss, saved=saved, ws=ws)
        B.distill_bwd(z, index, teacher, saved, weights=w, out=out)
    for other in bufs:
        for a, b in zip((z, index, teacher, w), other):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        want = B.distill_fwd(*other[:3], weights=other[3])
        assert all(torch.equal(a, b) for a, b in zip((loss, rows, saved), want))
        assert torch.equal(out, B.distill_bwd(*other[:3], want[2], weights=other[3]))


# rows of 65536 columns and more are shared by several blocks forwards, whose parts another launch joins: every way of leaving rows out, odd widths and rows with room between, few rows and many
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,K,M,ld,how", [(3, 65535, 20, None, "plain"), (3, 65536, 20, None, "accumulate"), (9, 70001, 33, 70008, "in place"), (5, 66001, 1, 66001, "plain"), (70, 65552, 7, None, "in place")])
@pytest.mark.parametrize("weights", ["some", "none of them", None])
def test_long_rows(N, K, M, ld, how, weights, dtype):
    buf, index, teacher, w = case(N, K, M, dtype, seed=K + N, ld=ld, weights=weights, gone=True)
    check(buf, index, teacher, w, K, accumulate=how == "accumulate", in_place=how == "in place")


def test_long_rows_far_from_zero():
    buf, index, teacher, _ = case(3, 80000, 9)
    check(buf + 20000, index, teacher - 20000, None, 80000, tau=0.7)


@pytest.mark.parametrize("K", [65536, 100001])
def test_long_rows_that_are_left_out(K):
    """Rows without weight are not read, rows without a place have nothing, whatever they hold; masked words, a part of a row that is all masked, wrong indices and NaN stay in their rows."""
    buf, index, teacher, _ = case(8, K, 5)
    index[:] = torch.arange(5, dtype=torch.int32) * (K // 6)
    w = torch.tensor([1.0, 0.0, 2.0, 0.5, 1.0, 3.0, 0.0, 1.5])
    want = check(buf, index, teacher, w, K)
    buf[1], teacher[6], index[6, 0], buf[6, 5] = math.nan, math.inf, K + 7, -math.inf
    per_row, saved = B.distill_fwd(buf.cuda(), index.cuda(), teacher.cuda(), tau=1.5, weights=w.cuda())[1:]
    assert bool(torch.isfinite(per_row).all()) and not per_row[[1, 6]].any() and not saved[[1, 6]].any()
    assert torch.equal(B.distill_bwd(buf.cuda(), index.cuda(), teacher.cuda(), saved, tau=1.5, dloss=0.7, weights=w.cuda()), want)
    buf[0, K // 2 + 1:] = -math.inf         # (the places of the first half alone count)
    index[0, 3:] = -1
    index[2] = -1
    buf[2, 0] = math.nan
    index[3, 2] = K
    buf[4, K - 1] = math.nan
    buf[5] = -math.inf
    loss, per_row, saved = B.distill_fwd(buf.cuda(), index.cuda(), teacher.cuda(), tau=1.5, weights=w.cuda())
    rows = O.distill_rows(buf[[0, 7]].double(), index[[0, 7]], teacher[[0, 7]].double(), 1.5)
    assert (per_row[[0, 7]].double().cpu() - rows).abs().max() <= LOSS * 30
    assert per_row[2] == 0 and bool(per_row[3:6].isnan().all()) and bool(loss.isnan().all())
    out = B.distill_bwd(buf.cuda(), index.cuda(), teacher.cuda(), saved, tau=1.5, dloss=0.7, weights=w.cuda())
    assert not out[[1, 2, 6]].any() and not out[0, K // 2 + 1:].any() and bool(out[3:6].isnan().all()) and bool(torch.isfinite(out[[0, 7]]).all())
    assert torch.equal(out[7], want[7])


def test_long_rows_captured():
    bufs = [tuple(x.cuda() for x in case(9, 70000, 12, "bf16", seed=s, weights="some")) for s in range(3)]
    z, index, teacher, w = (x.clone() for x in bufs[0])
    ws = B.Workspace()
    loss, rows, saved = B.distill_fwd(z, index, teacher, weights=w, ws=ws)
    out = torch.empty_like(z)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        B.distill_fwd(z, index, teacher, weights=w, per_row=rows, loss=loss, saved=saved, ws=ws)
        B.distill_bwd(z, index, teacher, saved, weights=w, out=out)
    for other in bufs:
        for a, b in zip((z, index, teacher, w), other):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        want = B.distill_fwd(*other[:3], weights=other[3])
        assert all(torch.equal(a, b) for a, b in zip((loss, rows, saved), want))
        assert torch.equal(out, B.distill_bwd(*other[:3], want[2], weights=other[3]))


@pytest.mark.parametrize("by,dloss", [(2.0 ** 100, 2.0 ** 30), (2.0 ** -100, 2.0 ** -40)])
def test_only_shares_of_the_weights_count(by, dloss):
    """Weights that are all larger or smaller by a power of two, with a factor of the loss that together with them leaves the range of a float: the same bits."""
    buf, index, teacher, w = (x.cuda() for x in case(6, 500, 7, weights="some", seed=2))
    assert bool(w.any())
    (loss, rows, saved), (loss2, rows2, saved2) = (B.distill_fwd(buf, index, teacher, weights=x) for x in (w, w * by))
    assert torch.equal(loss, loss2) and torch.equal(rows, rows2)
    want = B.distill_bwd(buf, index, teacher, saved, weights=w, dloss=dloss)
    assert bool(torch.isfinite(want).all()) and bool(want.any())
    assert torch.equal(B.distill_bwd(buf, index, teacher, saved2, weights=w * by, dloss=dloss), want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tau", [0.5, 2.0])
@pytest.mark.parametrize("K", [901, 70000])
def test_words_masked_by_the_lowest_value(K, tau, dtype):
    """Their share is 0, also where the value / tau is out of range; whole lanes' and blocks' parts of a row may be masked."""
    buf, index, teacher, _ = case(3, K, 9, dtype, seed=K)
    buf[:, ::3] = torch.finfo(TYPES[dtype]).min
    buf[1, K // 3:] = torch.finfo(TYPES[dtype]).min
    index = index % (K // 3) // 3 * 3 + 1
    out = check(buf, index, teacher, None, K, tau=tau)
    assert not out[:, ::3].any() and not out[1, K // 3:].any()

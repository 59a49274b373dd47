"""The scaled embedding, the delta rule and the distillation loss as a model uses them: a language model of one block that learns from a teacher, its loss and all gradients against the same model in
64 bits, in a graph against the eager run, and token by token against the whole.

Tolerance: every gradient passes through about twenty products of up to 192 terms (the ten of the delta rule's two passes among them), each rounding 2^-24 of the partial sums, which add up like
roots: 20 * sqrt(192) * 2^-24 = 1.7e-5 of its norm."""
import math

import pytest
import torch

from oracle import learning as O
from paper_2409_11600_amd import binding as B

pytestmark = pytest.mark.gpu
TOL = 20 * math.sqrt(192) * 2.0 ** -24
T, N, V, E, M, PAD, TAU, HEADS = 90, 5, 300, 32, 12, 0, 2.0, (4, 2, 16, 8)
H, HK, D, DV = HEADS
W = 2 * HK * D + H * (DV + 2)
SCALE = math.sqrt(E)


def model(seed=0):
    gen = torch.Generator().manual_seed(seed)
    normal = lambda *s: torch.randn(s, generator=gen)
    w = {"table": normal(V, E) / SCALE, "w_in": normal(W, E) / SCALE, "b_in": torch.cat((1 + 3 * torch.rand(H, generator=gen), normal(H))), "w_out": normal(V, H * DV) / math.sqrt(H * DV)}
    lengths = torch.tensor([90, 0, 1, 65, 40], dtype=torch.int32)
    tokens = torch.randint(1, V, (T, N), generator=gen, dtype=torch.int32)
    live = torch.arange(T)[:, None] < lengths
    tokens[~live] = PAD
    batch = {"tokens": tokens, "lengths": lengths, "index": torch.randint(0, V, (T * N, M), generator=gen, dtype=torch.int32), "teacher": 2 * normal(T * N, M), "weights": live.reshape(-1).float()}
    return w, batch


class Student:
    """The calls of a training step, on buffers made once."""

    def __init__(self, w, batch):
        self.w, self.b, self.ws = {k: v.cuda() for k, v in w.items()}, {k: v.cuda() for k, v in batch.items()}, B.Workspace()
        self.grad = {k: torch.empty_like(v) for k, v in self.w.items()}
        e = lambda *s: torch.empty(s, device="cuda")
        self.x, self.gi, self.o, self.logits, self.last = e(T * N, E), e(T, N, W), e(T, N, H * DV), e(T * N, V), e(N, H, D, DV)
        self.saved, self.loss, self.rows, self.held = e(-(-T // 64), N, H, D, DV), e(1), e(T * N), e(T * N + 1, 2)
        self.dgi, self.do, self.dx = e(T, N, W), e(T, N, H * DV), e(T * N, E)

    def step(self):
        w, b, g, ws = self.w, self.b, self.grad, self.ws
        B.embedding_scaled_fwd(b["tokens"], w["table"], SCALE, pad=PAD, out=self.x)
        B.linear_fwd(self.x, w["w_in"], None, out=self.gi.view(T * N, W), ws=ws)
        B.delta_fwd(self.gi, HEADS, w["b_in"], lengths=b["lengths"], o=self.o, h_last=self.last, saved=self.saved, ws=ws)
        B.linear_fwd(self.o.view(T * N, H * DV), w["w_out"], None, out=self.logits, ws=ws)
        B.distill_fwd(self.logits, b["index"], b["teacher"], tau=TAU, weights=b["weights"], per_row=self.rows, loss=self.loss, saved=self.held, ws=ws)
        B.distill_bwd(self.logits, b["index"], b["teacher"], self.held, tau=TAU, weights=b["weights"], out=self.logits)         # the gradient in the logits' place
        B.linear_wgrad(self.o.view(T * N, H * DV), self.logits, dw=g["w_out"], want_db=False, ws=ws)
        B.linear_dgrad(self.logits, w["w_out"], out=self.do.view(T * N, H * DV), ws=ws)
        B.delta_bwd(self.gi, self.saved, HEADS, w["b_in"], do=self.do, lengths=b["lengths"], dgi=self.dgi, want_dh0=False, ws=ws)
        flat = self.dgi.view(T * N, W)
        torch.sum(flat[:, -2 * H:], 0, out=g["b_in"])
        B.linear_wgrad(self.x, flat, dw=g["w_in"], want_db=False, ws=ws)
        B.linear_dgrad(flat, w["w_in"], out=self.dx, ws=ws)
        B.embedding_scaled_bwd(b["tokens"], self.dx, V, SCALE, pad=PAD, dtable=g["table"], ws=ws)
        return self.loss


def in_64_bits(w, b):
    w = {k: v.double().requires_grad_(True) for k, v in w.items()}
    x = O.embedding(b["tokens"].reshape(-1), w["table"], SCALE, pad=PAD)
    o, last, _ = O.delta((x @ w["w_in"].t()).view(T, N, W), HEADS, w["b_in"], lengths=b["lengths"])
    logits = o.reshape(T * N, -1) @ w["w_out"].t()
    loss, _ = O.distill(logits, b["index"], b["teacher"].double(), TAU, b["weights"].double())
    return loss, dict(zip(w, torch.autograd.grad(loss, list(w.values())))), logits


def test_training_step():
    w, b = model()
    s = Student(w, b)
    loss = s.step()
    want, grads, _ = in_64_bits(w, b)
    assert abs(loss.item() - want.item()) <= TOL * abs(want.item())
    for k, g in grads.items():
        assert (s.grad[k].double().cpu() - g).norm() <= TOL * g.norm(), k
    assert not s.grad["table"][PAD].any()


def test_training_step_in_a_graph():
    first, second = model(1), model(2)
    s = Student(*first)
    s.step()
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        s.step()
    for w, b in (second, first, second):
        for k in s.w:
            s.w[k].copy_(w[k])
        for k in s.b:
            s.b[k].copy_(b[k])
        graph.replay()
        torch.cuda.synchronize()
        other = Student(w, b)
        loss = other.step()
        assert torch.equal(s.loss, loss) and all(torch.equal(s.grad[k], other.grad[k]) for k in s.grad if k != "b_in")
        assert (s.grad["b_in"] - other.grad["b_in"]).norm() <= TOL * other.grad["b_in"].norm()


def test_token_by_token():
    w, b = model(3)
    _, _, logits = in_64_bits(w, b)
    s = Student(w, b)
    table = torch.zeros(N + 3, H, D, DV, device="cuda")
    places = torch.tensor([6, 0, 3, 1, 7], dtype=torch.int32, device="cuda")
    for t in range(40):
        x = B.embedding_scaled_fwd(s.b["tokens"][t].clone(), s.w["table"], SCALE, pad=PAD)
        live = (s.b["lengths"] > t).to(torch.int32)
        o = B.delta_step(B.linear_fwd(x, s.w["w_in"], None, ws=s.ws), table, HEADS, s.w["b_in"], slots=torch.where(live > 0, places, -1).to(torch.int32))
        got = B.linear_fwd(o, s.w["w_out"], None, ws=s.ws).double().cpu()
        want = logits.detach().view(T, N, V)[t]
        assert (got - want).norm() <= TOL * want.norm() + 1e-30, t

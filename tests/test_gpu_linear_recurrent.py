"""The classifier made of layer norm, the gated linear recurrence and 8-bit AdamW, as a whole: a training step against the oracle, training, tokens one by one."""
import numpy as np
import pytest
import torch

import nsk_inputs as gen
from oracle import sequence as S
from oracle import train as T
from paper_2409_11600_amd.linear_recurrent import GpuLinearRecurrentClassifier, TokenStream, matrices, parameter_names
from parity import TOL, max_rel_err

pytestmark = pytest.mark.gpu


def host(t):
    return t.detach().double().cpu().numpy()


def model(seed, T_, N, E, H, V, K, L, ragged=True):
    tokens = ((gen.uniform(seed, 0, (T_, N)) * V).astype(np.int32)) % V
    labels = ((gen.uniform(seed, 1, (N,)) * K).astype(np.int32)) % K
    lengths = 1 + ((gen.uniform(seed, 2, (N,)) * T_).astype(np.int32)) % T_ if ragged else None
    p = {"table": gen.normal(seed, 3, (V, E)), "gamma": 1 + 0.1 * gen.normal(seed, 4, (H,)), "beta": 0.1 * gen.normal(seed, 5, (H,)),
         "w_cls": gen.normal(seed, 6, (K, H)) / np.sqrt(H), "b_cls": 0.1 * gen.normal(seed, 7, (K,))}
    for k in range(L):
        s = 100 * (k + 1)
        p |= {f"gamma{k}": 1 + 0.1 * gen.normal(seed, s, (E,)), f"beta{k}": 0.1 * gen.normal(seed, s + 1, (E,)), f"w_in{k}": gen.normal(seed, s + 2, (3 * H, E)) / np.sqrt(E),
              f"b_in{k}": np.concatenate((1 + gen.normal(seed, s + 3, (H,)), np.zeros(2 * H)))}
        if k < L - 1:
            p[f"w_out{k}"] = gen.normal(seed, s + 4, (E, H)) / np.sqrt(H)
    return tokens, labels, lengths, {k: np.asarray(v, np.float32) for k, v in p.items()}


@pytest.mark.parametrize("shape", [(6, 4, 16, 16, 50, 2, 1), (21, 5, 32, 24, 60, 3, 2), (40, 8, 24, 40, 100, 2, 3)])
@pytest.mark.parametrize("ragged", [False, True])
def test_a_training_step_matches_the_oracle(shape, ragged):
    T_, N, E, H, V, K, L = shape
    print(f"linear recurrent classifier T={T_} N={N} E={E} H={H} V={V} K={K} L={L} ragged={ragged}", flush=True)
    tokens, labels, lengths, p = model(900 + T_, *shape, ragged)
    m = GpuLinearRecurrentClassifier(tokens, labels, p, lengths, lr=1e-3, weight_decay=1e-2, clip=0.05, seed=5)
    assert m.order == parameter_names(L) and set(m.order) == set(p)
    m.forward()
    m.backward()
    torch.cuda.synchronize()
    loss, logits, finals, grads = S.classifier_step(tokens, labels, p, lengths)
    assert abs(float(m.loss) - loss) <= 1e-5 * abs(loss) and max_rel_err(host(m.logits), logits) <= TOL["f32"]
    for k in range(L):
        assert max_rel_err(host(m.h[k]), finals[k]) <= TOL["f32"]
    for k in m.order:
        assert max_rel_err(host(m.grad[k]), grads[k]) <= 2 * TOL["f32"], k
    before = {k: host(m.grad[k]).reshape(-1) for k in m.order}
    m.update()
    torch.cuda.synchronize()
    scale = T.clip_scale([before[k] for k in m.order], 0.05)
    assert scale < 1.0
    zero = lambda n: np.zeros(n)
    for i, k in enumerate(m.order):
        n = p[k].size
        decay = 1e-2 if k in matrices(L) or k == "w_cls" else 0.0
        want = S.adamw8_step(p[k].reshape(-1), before[k], zero(n), zero(n), zero(-(-n // 256)), zero(-(-n // 256)), 1, 6, i, 1e-3, 0.9, 0.999, 1e-8, decay, scale, real=np.float64)
        # (a gradient near eps moves its weight by any part of lr: the step's sign and size follow the gradient's own rounding there)
        sure = np.abs(before[k]) * scale > 1e-6
        moved = host(m.master[k]).reshape(-1) - p[k].reshape(-1)
        assert np.abs(moved - (want[0] - p[k].reshape(-1)))[sure].max(initial=0) <= 1e-3 * 1e-3 + 2.0 ** -23 * np.abs(p[k]).max(), k
        assert not m.grad[k].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_it_learns(dtype):
    """A batch is learnt by heart; the loss of the first step is the oracle's."""
    tokens, labels, lengths, p = model(77, 20, 16, 32, 32, 64, 2, 2)
    m = GpuLinearRecurrentClassifier(tokens, labels, p, lengths, dtype=dtype, lr=1e-2, weight_decay=0.0, clip=5.0)
    q = {k: (gen.to_bf16_grid(v) if dtype == "bf16" and k in matrices(2) else v) for k, v in p.items()}
    loss = S.classifier_step(tokens, labels, q, lengths)[0]
    losses = []
    for _ in range(40):
        m.step()
        torch.cuda.synchronize()
        losses.append(float(m.loss))
    assert abs(losses[0] - loss) <= (2e-2 if dtype == "bf16" else 1e-4) * abs(loss)
    assert np.all(np.isfinite(losses)) and losses[-1] < 0.5 * losses[0], losses[::8]
    for k in matrices(2):
        assert torch.equal(m.w[k], m.master[k].to(m.dt))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tokens_one_by_one_give_the_logits_of_the_sequences(dtype):
    T_, N, places = 25, 6, 11
    tokens, labels, lengths, p = model(78, T_, N, 32, 48, 64, 3, 2)
    m = GpuLinearRecurrentClassifier(tokens, labels, p, lengths, dtype=dtype)
    m.forward()
    want = host(m.logits)
    stream = TokenStream(m, places)
    place = torch.tensor([7, 0, 10, 3, 5, 2], dtype=torch.int32, device="cuda:0")
    for s in stream.states:
        s.fill_(float("nan"))           # (what an earlier sequence left)
    for n in range(N):
        stream.begin(int(place[n]))
    tok = torch.from_numpy(tokens).cuda()
    got = np.zeros_like(want)
    for t in range(T_):
        live = torch.from_numpy(lengths > t).cuda()
        logits = stream.step(tok[t].clone(), torch.where(live, place, -1).to(torch.int32))
        assert torch.isnan(logits[~live]).all() and torch.isfinite(logits[live]).all()
        ends = np.asarray(lengths) == t + 1
        got[ends] = host(logits)[ends]
    assert max_rel_err(got, want) <= TOL[dtype]


@pytest.mark.parametrize("n", [1, 4, 6])
def test_tokens_without_slots_are_those_of_the_first_places(n):
    tokens, labels, lengths, p = model(80, 9, 6, 32, 48, 64, 3, 2)
    m = GpuLinearRecurrentClassifier(tokens, labels, p, lengths)
    one, other = TokenStream(m, 6), TokenStream(m, 6)
    tok, first = torch.from_numpy(tokens).cuda(), torch.arange(n, dtype=torch.int32, device="cuda:0")
    for t in range(9):
        got, want = one.step(tok[t, :n].clone()), other.step(tok[t, :n].clone(), first)
        assert got.shape == (n, 3) and torch.equal(got, want) and torch.isfinite(got).all()
    assert all(torch.equal(a, b) and not a[n:].any() for a, b in zip(one.states, other.states))
    before = [s.clone() for s in one.states]
    with pytest.raises(ValueError):
        one.step(torch.zeros(7, dtype=torch.int32, device="cuda:0"))
    assert all(torch.equal(a, b) for a, b in zip(one.states, before))


def test_forward_and_backward_in_a_graph():
    tokens, labels, lengths, p = model(79, 30, 8, 32, 64, 64, 2, 2)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        m = GpuLinearRecurrentClassifier(tokens, labels, p, lengths, dtype="bf16")
        m.step()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            m.forward()
            m.backward()
        for _ in range(4):
            graph.replay()
            stream.synchronize()
            got = [m.grad[k].clone() for k in m.order] + [m.loss.clone()]
            m.forward()
            m.backward()
            stream.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, [m.grad[k] for k in m.order] + [m.loss]))
            m.update()
            stream.synchronize()

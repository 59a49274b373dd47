"""A sequence classifier whose recurrence is linear in its state: embedding -> blocks of layer norm, product, gated linear recurrence and (in all but the last)
product back onto the residual stream -> layer norm of the last block's final states -> output layer -> cross entropy; gradient clip and AdamW with 8-bit moments.

It stands next to the GRU classifier (recurrent.py) and takes the same batches, here with a length for each sequence.  Where that one has 2T steps that wait for each
other, all steps of a block are one call here.  Sequencing and buffer management only: every arithmetic step is a libnsk entry point; all buffers are created in the
constructor, a step allocates nothing, and forward() and backward() can be captured into a HIP graph (update() takes another step and seed each time, which a
graph would keep).

TokenStream is the same network for tokens that come one by one: the states of any number of live sequences lie in tables, and a step takes a token for some of them.
"""
from __future__ import annotations

from typing import Dict, Optional

import numpy as np
import torch

from . import binding as B


def parameter_names(layers: int):
    """Names of the parameters in the order of the optimizer's table."""
    names = ["table"]
    for k in range(layers):
        names += [f"gamma{k}", f"beta{k}", f"w_in{k}", f"b_in{k}"] + ([f"w_out{k}"] if k < layers - 1 else [])
    return names + ["gamma", "beta", "w_cls", "b_cls"]


def matrices(layers: int):
    """Those that have a copy in the storage type and weight decay (the output layer w_cls has the decay alone: it works on float states)."""
    return ["table"] + [f"w_in{k}" for k in range(layers)] + [f"w_out{k}" for k in range(layers - 1)]


class GpuLinearRecurrentClassifier:
    """params: table [V,E]; for block k gamma{k}, beta{k} [E], w_in{k} [3H,E], b_in{k} [3H] (gates f, c, o) and, but for the last, w_out{k} [E,H];
    gamma, beta [H]; w_cls [K,H], b_cls [K].  tokens: [T,N], time-major; lengths: [N] or None; tokens behind a sequence's end may be any in the vocabulary."""

    def __init__(self, tokens: np.ndarray, labels: np.ndarray, params: Dict[str, np.ndarray], lengths: Optional[np.ndarray] = None, dtype: str = "f32", lr: float = 1e-3,
                 weight_decay: float = 1e-4, clip: Optional[float] = 5.0, seed: int = 0, device: str = "cuda:0"):
        dev = torch.device(device)
        self.device = dev
        self.dt = dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.L = L = sum(1 for k in params if k.startswith("w_in"))
        self.T, self.N = T, N = tokens.shape
        self.V, self.E = V, E = params["table"].shape
        self.H, self.K = H, K = params["w_cls"].shape[1], params["w_cls"].shape[0]
        self.lr, self.clip, self.seed, self.t = lr, clip, seed, 0
        ints = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(dev)
        f32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(dev)
        self.tokens, self.labels = ints(tokens.reshape(-1)), ints(labels)
        self.lengths = None if lengths is None else ints(lengths)
        self.order, large = parameter_names(L), matrices(L)
        self.master = {k: f32(params[k]) for k in self.order}
        lp = dt == torch.bfloat16
        self.w = {k: (v.to(dt) if lp and k in large else v) for k, v in self.master.items()}
        self.grad = {k: torch.zeros_like(v) for k, v in self.master.items()}
        self.state = {k: B.adamw8_state(self.master[k].numel(), dev) for k in self.order}
        self.records = B.param8_table((self.master[k], self.grad[k], *self.state[k], self.w[k] if lp and k in large else None,
                                       weight_decay if k in large or k == "w_cls" else 0.0) for k in self.order)
        z = lambda *s: torch.zeros(s, dtype=dt, device=dev)
        floats = lambda *s: torch.zeros(s, dtype=torch.float32, device=dev)
        rows = T * N
        self.s = [z(rows, E) for _ in range(L)]             # the residual stream in front of each block
        self.u = [z(rows, E) for _ in range(L)]
        self.gi = [z(T, N, 3 * H) for _ in range(L)]
        self.y = [z(T, N, H) for _ in range(L - 1)]
        self.branch = z(rows, E)
        self.mean, self.invstd = [floats(rows) for _ in range(L)], [floats(rows) for _ in range(L)]
        self.saved = [floats(-(-T // B.NSK_GLR_STRETCH), N, H) for _ in range(L)]
        self.h = [floats(N, H) for _ in range(L)]           # the states behind the last step
        self.z, self.z_mean, self.z_invstd = floats(N, H), floats(N), floats(N)
        self.logits, self.dlogits, self.dz, self.dh = floats(N, K), floats(N, K), floats(N, H), floats(N, H)
        self.per_sample, self.loss = floats(N), floats(1)
        self.ds, self.du, self.dgi, self.dy = z(rows, E), z(rows, E), z(T, N, 3 * H), z(T, N, H)
        self.partials, self.sumsq, self.scale = floats(B.NSK_SUMSQ_PARTIALS), floats(1), floats(1)
        self.ws = B.Workspace(dev)

    def forward(self):
        w, rows = self.w, self.T * self.N
        B.embedding_fwd(self.tokens, w["table"], out=self.s[0])
        for k in range(self.L):
            x, residual, total = (self.s[0], None, None) if k == 0 else (self.branch, self.s[k - 1], self.s[k])
            B.layernorm_fwd(x, w[f"gamma{k}"], w[f"beta{k}"], residual=residual, out=self.u[k], sum_out=total, save_mean=self.mean[k], save_invstd=self.invstd[k])
            B.linear_fwd(self.u[k], w[f"w_in{k}"], None, out=self.gi[k].view(rows, 3 * self.H), ws=self.ws)
            last = k == self.L - 1
            B.glr_fwd(self.gi[k], w[f"b_in{k}"], lengths=self.lengths, y=None if last else self.y[k], h_last=self.h[k], saved=self.saved[k], want_y=not last, ws=self.ws)
            if not last:
                B.linear_fwd(self.y[k].view(rows, self.H), w[f"w_out{k}"], None, out=self.branch, ws=self.ws)
        B.layernorm_fwd(self.h[-1], w["gamma"], w["beta"], out=self.z, save_mean=self.z_mean, save_invstd=self.z_invstd)
        B.linear_fwd(self.z, w["w_cls"], w["b_cls"], out=self.logits, ws=self.ws)
        B.softmax_xent_fwd(self.logits, self.labels, per_sample=self.per_sample, loss=self.loss)

    def backward(self):
        w, g, rows = self.w, self.grad, self.T * self.N
        B.softmax_xent_bwd(self.logits, self.labels, 1.0, out=self.dlogits)
        B.linear_wgrad(self.z, self.dlogits, dw=g["w_cls"], db=g["b_cls"], ws=self.ws)
        B.linear_dgrad(self.dlogits, w["w_cls"], out=self.dz, ws=self.ws)
        B.layernorm_bwd(self.dz, self.h[-1], w["gamma"], self.z_mean, self.z_invstd, dx=self.dh, dgamma=g["gamma"], dbeta=g["beta"], ws=self.ws)
        flat = self.dgi.view(rows, 3 * self.H)
        for k in reversed(range(self.L)):
            last = k == self.L - 1
            if not last:                                    # ds: the gradient of the stream behind this block, which its branch was added to
                B.linear_wgrad(self.y[k].view(rows, self.H), self.ds, dw=g[f"w_out{k}"], want_db=False, ws=self.ws)
                B.linear_dgrad(self.ds, w[f"w_out{k}"], out=self.dy.view(rows, self.H), ws=self.ws)
            B.glr_bwd(self.gi[k], self.saved[k], w[f"b_in{k}"], dy=None if last else self.dy, dh_last=self.dh if last else None, lengths=self.lengths, dgi=self.dgi,
                      want_dh0=False, ws=self.ws)
            B.linear_wgrad(self.u[k], flat, dw=g[f"w_in{k}"], db=g[f"b_in{k}"], ws=self.ws)
            B.linear_dgrad(flat, w[f"w_in{k}"], out=self.du, ws=self.ws)
            B.layernorm_bwd(self.du, self.s[k], w[f"gamma{k}"], self.mean[k], self.invstd[k], dsum=None if last else self.ds, dx=self.ds, dgamma=g[f"gamma{k}"],
                            dbeta=g[f"beta{k}"], ws=self.ws)
        B.embedding_bwd(self.tokens, self.ds, self.V, dtable=g["table"])

    def update(self):
        self.t += 1
        scale = None
        if self.clip is not None:
            scale = B.clip_scale([self.grad[k] for k in self.order], self.clip, self.partials, self.sumsq, self.scale)
        B.adamw8_step_multi(self.records, self.t, self.seed + self.t, self.lr, grad_scale=scale)

    def step(self):
        self.forward()
        self.backward()
        self.update()


class TokenStream:
    """The classifier's network on tokens that come one by one.  `places`: how many sequences can be live; each has a row in the tables of states."""

    def __init__(self, model: GpuLinearRecurrentClassifier, places: int):
        self.m, self.places = model, places
        self.states = [torch.zeros((places, model.H), dtype=torch.float32, device=model.device) for _ in range(model.L)]
        self.ws = B.Workspace(model.device)

    def begin(self, place: int):
        """A new sequence at this place."""
        for s in self.states:
            s[place].zero_()

    def step(self, tokens: torch.Tensor, slots: Optional[torch.Tensor] = None) -> torch.Tensor:
        """tokens: int32 [n], one for each of the sequences at the places `slots` (int32 [n], none twice; None: the first n, of which there have to be so many).
        Returns the logits [n, K] behind them, float; a slot that is no place is idle, and its logits are NaN."""
        if slots is None and tokens.numel() > self.places:
            raise ValueError(f"{tokens.numel()} tokens for the first places of {self.places}")
        m, w, ws = self.m, self.m.w, self.ws
        x, residual = B.embedding_fwd(tokens, w["table"]), None
        for k in range(m.L):
            total = torch.empty_like(x) if residual is not None else None
            u, s, _, _ = B.layernorm_fwd(x, w[f"gamma{k}"], w[f"beta{k}"], residual=residual, sum_out=total, save=False)
            last = k == m.L - 1
            y = B.glr_step(B.linear_fwd(u, w[f"w_in{k}"], None, ws=ws), self.states[k], w[f"b_in{k}"], slots=slots, want_y=not last)
            if not last:
                x, residual = B.linear_fwd(y, w[f"w_out{k}"], None, ws=ws), s
        h = self.states[-1][:tokens.numel()] if slots is None else B.embedding_fwd(slots, self.states[-1])
        return B.linear_fwd(B.layernorm_fwd(h, w["gamma"], w["beta"], save=False)[0], w["w_cls"], w["b_cls"], ws=ws)

"""The operators of the sequence models next to the GRU classifier: layer norm with its residual add, the gated linear recurrence (all steps
at once in both directions, and one token for each of many sequences) and AdamW with its moments in 8 bits.

A case names the call ("call": ln_fwd, ln_bwd, glr_fwd, glr_bwd, glr_step, adamw8), its type and its sizes.  `run` is one call: in elementary
torch operations where `own` is false, through paper_2409_11600_amd.binding where it is true.

Layer norm over the last axis, s = x + residual as stored, biased variance:
  y = (s - mean) * invstd * gamma + beta;   with gh = dy * gamma, xh = (s - mean) * invstd, means over the last axis:
  dx = invstd * (gh - mean(gh) - xh * mean(gh * xh)) + dsum;   dgamma = sum over rows of dy * xh;   dbeta = sum over rows of dy.
Recurrence, gates in the order (f, c, o) of gi [T,N,3H], per sequence n and channel, for t < lengths[n] (later steps: h stays, y = 0):
  f = sigmoid(gi_f + b_f), c = gi_c + b_c, o = sigmoid(gi_o + b_o);   h_t = f h_{t-1} + (1 - f) c;   y_t = o h_t.
  Its backward pass also takes the states that enter the steps 0, 16, 32, ... (float), which the forward pass leaves.
AdamW: m and r = sqrt(v) are e4m3 values times a power of two for each 256 elements, rounded at random (the numbers come from a seed).
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5
STRETCH = 16                # steps between two saved states
BLOCK = 256                 # elements that share a scale
ADAM = {"lr": 1e-3, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "weight_decay": 1e-4, "step": 7}

# The tensors of the GRU classifier (vocabulary 32768, 256 units, two classes), and of a residual network for 32 x 32 images: 31 layers of 3x3
# filters of 16, 32 and 64 channels with the two vectors of a normalisation each, and the output layer.
GRU_SIZES = [32768 * 256, 768 * 256, 768 * 256, 768, 768, 2 * 256, 2]
CIFAR_SIZES = [n for k, c, count in ((3, 16, 1), (16, 16, 10), (16, 32, 1), (32, 32, 9), (32, 64, 1), (64, 64, 9)) for _ in range(count) for n in (9 * k * c, c, c)] + [640, 10]


def listed():
    text = lambda sizes: ",".join(str(n) for n in sizes)
    return [
        # one token for each of 50 sequences: latency alone
        {"name": "ln_token_bf16", "call": "ln_fwd", "dtype": "bf16", "rows": 50, "C": 256, "residual": True},
        # all tokens of the recurrent experiment, 200 steps of 50 sequences, with the gradient of the residual stream
        {"name": "ln_bwd_gru_f32", "call": "ln_bwd", "dtype": "f32", "rows": 10000, "C": 256, "residual": True},
        # a large batch of long sequences in a wider model
        {"name": "ln_large_bf16", "call": "ln_fwd", "dtype": "bf16", "rows": 65536, "C": 768, "residual": True},
        # an odd width: rows that begin on no vector's boundary
        {"name": "ln_bwd_odd_bf16", "call": "ln_bwd", "dtype": "bf16", "rows": 30011, "C": 1001, "residual": False},
        # serving: one token for each of 50 sequences
        {"name": "glr_token_bf16", "call": "glr_step", "dtype": "bf16", "N": 50, "H": 256, "slots": 64},
        # the recurrent experiment's sequences
        {"name": "glr_gru_f32", "call": "glr_fwd", "dtype": "f32", "T": 200, "N": 50, "H": 256, "ragged": False},
        # a batch of texts of different lengths, among them none and one token, an uneven width
        {"name": "glr_bwd_ragged_f32", "call": "glr_bwd", "dtype": "f32", "T": 777, "N": 33, "H": 201, "ragged": True},
        # a large batch of long sequences in a wider model
        {"name": "glr_bwd_large_bf16", "call": "glr_bwd", "dtype": "bf16", "T": 2048, "N": 32, "H": 768, "ragged": False},
        # one very long sequence: few channels, and all of the parallel work along the time
        {"name": "glr_long_bf16", "call": "glr_fwd", "dtype": "bf16", "T": 65536, "N": 1, "H": 512, "ragged": False},
        # the GRU classifier's weights, one large table and small ones
        {"name": "adamw8_gru", "call": "adamw8", "copy": False, "sizes": text(GRU_SIZES)},
        # many small tensors: the cost of the launches
        {"name": "adamw8_cifar", "call": "adamw8", "copy": True, "sizes": text(CIFAR_SIZES)},
        # a model of 64 million weights, with the bf16 copies that its kernels read
        {"name": "adamw8_large", "call": "adamw8", "copy": True, "sizes": text([32768 * 768] + [2304 * 768, 768 * 768, 2304, 768, 768] * 16 + [1000 * 769])},
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    call = rng.choice(["ln_fwd", "ln_bwd", "glr_fwd", "glr_bwd", "glr_step", "adamw8"])
    dtype = rng.choice(["f32", "bf16"])
    if call in ("ln_fwd", "ln_bwd"):
        C = rng.choice([_log(rng, 8, 8192), 8 * _log(rng, 1, 1024)])
        return {"call": call, "dtype": dtype, "rows": _log(rng, 1, 24_000_000 // C), "C": C, "residual": rng.random() < 0.5}
    if call == "glr_step":
        N = _log(rng, 1, 4096)
        return {"call": call, "dtype": dtype, "N": N, "H": rng.choice([_log(rng, 16, 2048), 8 * _log(rng, 2, 256)]), "slots": N + _log(rng, 1, 256)}
    if call in ("glr_fwd", "glr_bwd"):
        H = rng.choice([_log(rng, 16, 2048), 8 * _log(rng, 2, 256)])
        T = _log(rng, 1, 16384)
        return {"call": call, "dtype": dtype, "T": T, "N": _log(rng, 1, max(1, min(512, 16_000_000 // (T * H)))), "H": H, "ragged": rng.random() < 0.5}
    sizes = [_log(rng, 1, rng.choice([4096, 200_000, 8_000_000])) for _ in range(_log(rng, 1, 80))]
    while sum(sizes) > 60_000_000:
        sizes.pop()
    return {"call": call, "copy": rng.random() < 0.5, "sizes": ",".join(str(n) for n in sizes)}


def _sizes(case):
    return [int(n) for n in case["sizes"].split(",")]


def _lengths(case, gen):
    """A length for each sequence: from nothing to all steps, the first three at the ends of the range."""
    if not case["ragged"]:
        return None
    T, N = case["T"], case["N"]
    lengths = torch.randint(0, T + 1, (N,), generator=gen, device="cuda", dtype=torch.int32)
    ends = torch.tensor([T, 0, 1], dtype=torch.int32, device="cuda")[:N]
    lengths[:ends.numel()] = torch.minimum(ends, torch.full_like(ends, T))
    return lengths


def _scales(amax):
    """The power of two for which amax / scale lies in (224, 448], the upper end of e4m3; 2^-126 at least."""
    e = ((amax.view(torch.int32) + 0x1FFFFF) >> 23) - 8
    return (e.clamp(min=1) << 23).view(torch.float32)


def _blocks(x):
    return x.view(-1, BLOCK)


def _held(x):
    """(e4m3 values, scales) that hold the float vector x, to nearest."""
    s = _scales(_blocks(x).abs().amax(1))
    return (_blocks(x) / s[:, None]).view(-1).to(torch.float8_e4m3fn), s


def _padded(sizes, device):
    return torch.tensor([-(-n // BLOCK) * BLOCK for n in sizes], device=device)


def _places(sizes, device):
    """For each element of the buffers: its index in its tensor, and the tensor's."""
    padded = _padded(sizes, device)
    which = torch.arange(len(sizes), device=device).repeat_interleave(padded)
    return torch.arange(which.numel(), device=device) - (padded.cumsum(0) - padded)[which], which


def _tensors(state):
    """(w, grad, m, r, scale_m, scale_r, w_lp) of each tensor, parts of the buffers."""
    at = 0
    for n in _sizes(state["case"]):
        blocks = -(-n // BLOCK)
        part = lambda k: None if state[k] is None else state[k][at * BLOCK:at * BLOCK + n]
        scale = lambda k: state[k][at:at + blocks]
        yield part("w"), part("grad"), part("m"), part("r"), scale("scale_m"), scale("scale_r"), part("w_lp")
        at += blocks


def _buffers(state):
    return {k: state[k] for k in ("w", "grad", "m", "r", "scale_m", "scale_r", "w_lp") if state[k] is not None}


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 1_000_003 + 17)
    normal = lambda *s: torch.randn(s, generator=gen, device="cuda")
    state = {"case": case}
    if case["call"] == "adamw8":
        # one buffer for each kind of state, the tensors in it on whole blocks, zeros between them
        n = sum(-(-k // BLOCK) * BLOCK for k in _sizes(case))
        at, _ = _places(_sizes(case), "cuda")
        live = at < torch.tensor(_sizes(case), device="cuda").repeat_interleave(_padded(_sizes(case), "cuda"))
        size = live * 10.0 ** (-4 + 2 * torch.rand((n,), generator=gen, device="cuda"))     # gradients of very different sizes
        w = live * 0.05 * normal(n)
        (m, sm), (r, sr) = _held(0.3 * normal(n) * size), _held(size)
        state |= {"w": w, "grad": normal(n) * size, "m": m, "r": r, "scale_m": sm, "scale_r": sr, "w_lp": w.to(torch.bfloat16) if case["copy"] else None}
        state["seed"] = int(seed) * 7919 % (1 << 32)
        state["grad_scale"] = torch.full((1,), 0.7, device="cuda")
        if own:     # the list of tensors that a training loop keeps
            from paper_2409_11600_amd import binding as B
            state["table"] = B.param8_table((*tensors, ADAM["weight_decay"]) for tensors in _tensors(state))
        return state
    dt = TYPES[case["dtype"]]
    if case["call"] in ("ln_fwd", "ln_bwd"):
        rows, C = case["rows"], case["C"]
        state["gamma"], state["beta"] = 1 + 0.1 * normal(C), 0.1 * normal(C)
        x = (0.5 * normal(rows, 1) + normal(rows, C)).to(dt)
        other = normal(rows, C).to(dt) if case["residual"] else None
        if case["call"] == "ln_fwd":
            return {**state, "x": x, "residual": other}
        mean = x.float().mean(1)
        invstd = torch.rsqrt((x.float() - mean[:, None]).square().mean(1) + EPS)
        return {**state, "s": x, "dy": normal(rows, C).to(dt), "dsum": other, "mean": mean, "invstd": invstd}
    N, H = case["N"], case["H"]
    state["bias"] = torch.cat((1.0 + 2.0 * normal(H), 0.1 * normal(2 * H)))       # memories from a step to many
    if case["call"] == "glr_step":
        state["gi"] = normal(N, 3 * H).to(dt)
        state["table"] = normal(case["slots"], H)
        state["slots"] = torch.randperm(case["slots"], generator=gen, device="cuda")[:N].to(torch.int32)
        return state
    T = case["T"]
    state |= {"gi": normal(T, N, 3 * H).to(dt), "h0": normal(N, H), "lengths": _lengths(case, gen)}
    if case["call"] == "glr_bwd":
        state |= {"dy": normal(T, N, H).to(dt), "dh_last": normal(N, H)}
        f, x, _, _, _ = _gates(state["gi"], state["bias"], state["lengths"])
        h = _states(f, x, state["h0"])
        state["saved"] = torch.cat((state["h0"][None], h[:-1]))[::STRETCH].contiguous()
    return state


# ---------------------------------------------------------------------------------------------------------------- the plain forms

def _scan(a, b):
    """h_t = a_t h_{t-1} + b_t along the first axis from zero, in as many rounds as T has binary digits."""
    d = 1
    while d < a.shape[0]:
        b = torch.cat((b[:d], b[d:] + a[d:] * b[:-d]))
        a = torch.cat((a[:d], a[d:] * a[:-d]))
        d *= 2
    return b


def _gates(gi, bias, lengths):
    """(f, (1 - f) c, o, c, 1 - f) in float; (1, 0, 0, 0, 0) in steps that a sequence does not have."""
    f, c, o = (gi.float() + bias).chunk(3, dim=-1)
    keep, f, o = 1 / (1 + torch.exp(f)), 1 / (1 + torch.exp(-f)), 1 / (1 + torch.exp(-o))
    if lengths is not None:
        live = (torch.arange(gi.shape[0], device=gi.device)[:, None] < lengths)[..., None]
        zero = torch.zeros((), device=gi.device)
        f, keep, c, o = torch.where(live, f, zero + 1), torch.where(live, keep, zero), torch.where(live, c, zero), torch.where(live, o, zero)
    return f, keep * c, o, c, keep


def _states(f, x, h0):
    return _scan(f, torch.cat((x[:1] + f[:1] * h0, x[1:])))


def _mix(x):
    """A 32-bit number that depends on all bits of x, in whole numbers of 64 bits."""
    x = ((x ^ (x >> 16)) * 0x243F6A89) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0xB7E15163) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _random(sizes, seed, device):
    """32 bits for each element: of its index in its tensor, the tensor's index and the seed."""
    i, which = _places(sizes, device)
    return _mix((i * 0x9E3779B9 + (i >> 32) * 0x85A308D3 + _mix((seed + which * 0x9E3779B9) & 0xFFFFFFFF)) & 0xFFFFFFFF)


def _rounded(x, scales, bits):
    """The e4m3 values that hold x >= 0: up with the probability that makes their mean x, by 16 random bits.  What is not finite becomes NaN."""
    y = (_blocks(x) / scales[:, None]).view(-1)
    small = y < 2.0 ** -6                   # there steps are 2^-9, as from 2^-6 to 2^-5
    z = torch.where(small, y + 2.0 ** -6, y)
    q = ((z.view(torch.int32) + (bits << 4).to(torch.int32)) & ~0xFFFFF).view(torch.float32)
    return torch.where(torch.isfinite(x), torch.where(small, q - 2.0 ** -6, q), math.nan)


def _finite(x):
    return torch.where(torch.isfinite(x), x, 0)


def _adamw8(state):
    a = ADAM
    one, b1, b2 = np.float32(1), np.float32(a["beta1"]), np.float32(a["beta2"])
    c1, c2 = 1 / (1 - float(b1) ** a["step"]), math.sqrt(1 / (1 - float(b2) ** a["step"]))
    value = lambda k: (_blocks(state[k].float()) * state["scale_" + k][:, None]).view(-1)
    g = state["grad"] * state["grad_scale"]
    m = value("m") * float(b1) + g * float(one - b1)
    r = value("r")
    r = torch.sqrt(r * r * float(b2) + g * g * float(one - b2))
    w = state["w"] * float(one - np.float32(a["lr"]) * np.float32(a["weight_decay"])) - a["lr"] * (m * c1 / (r * c2 + a["eps"]))
    bits = _random(_sizes(state["case"]), state["seed"], w.device)
    sm, sr = (_scales(_blocks(_finite(v).abs()).amax(1)) for v in (m, r))
    qm = torch.copysign(_rounded(m.abs(), sm, bits & 0xFFFF), m)
    qr = _rounded(r, sr, bits >> 16)
    qr = torch.where(r > 0, torch.clamp(qr, min=2.0 ** -9), qr)
    for k, v in (("w", w), ("m", qm.to(torch.float8_e4m3fn)), ("r", qr.to(torch.float8_e4m3fn)), ("scale_m", sm), ("scale_r", sr)):
        state[k].copy_(v)
    state["grad"].zero_()
    if state["w_lp"] is not None:
        state["w_lp"].copy_(w)
    return _buffers(state)


def _plain(state):
    case, call = state["case"], state["case"]["call"]
    if call == "adamw8":
        return _adamw8(state)
    dt = TYPES[case["dtype"]]
    if call == "ln_fwd":
        s = state["x"] if state["residual"] is None else (state["x"].float() + state["residual"].float()).to(dt)
        v = s.float()
        mean = v.mean(1)
        d = v - mean[:, None]
        invstd = torch.rsqrt(d.square().mean(1) + EPS)
        y = (d * invstd[:, None] * state["gamma"] + state["beta"]).to(dt)
        return {"y": y, "mean": mean, "invstd": invstd, **({} if state["residual"] is None else {"sum": s})}
    if call == "ln_bwd":
        dy = state["dy"].float()
        xh = (state["s"].float() - state["mean"][:, None]) * state["invstd"][:, None]
        gh = dy * state["gamma"]
        dx = state["invstd"][:, None] * (gh - gh.mean(1, keepdim=True) - xh * (gh * xh).mean(1, keepdim=True))
        if state["dsum"] is not None:
            dx = dx + state["dsum"].float()
        return {"dx": dx.to(dt), "dgamma": (dy * xh).sum(0), "dbeta": dy.sum(0)}
    if call == "glr_step":
        f, x, o, _, _ = _gates(state["gi"], state["bias"], None)
        at = state["slots"].long()
        h = f * state["table"][at] + x
        state["table"][at] = h
        return {"y": (o * h).to(dt), "table": state["table"]}
    f, x, o, c, keep = _gates(state["gi"], state["bias"], state["lengths"])
    h = _states(f, x, state["h0"])
    if call == "glr_fwd":
        return {"y": (o * h).to(dt), "h_last": h[-1], "saved": torch.cat((state["h0"][None], h[:-1]))[::STRETCH].contiguous()}
    dy = state["dy"].float()
    before = torch.cat((state["h0"][None], h[:-1]))
    u = dy * o                              # what enters the recurrence from above; G_t = u_t + f_{t+1} G_{t+1}
    u[-1] += state["dh_last"]
    G = _scan(torch.cat((f[:1], f[1:].flip(0))), u.flip(0)).flip(0)
    df, dc, do = G * (before - c) * f * keep, G * keep, dy * h * o * (1 - o)
    return {"dgi": torch.cat((df, dc, do), dim=-1).to(dt), "dh0": f[0] * G[0]}


# ---------------------------------------------------------------------------------------------------------------- the framework's calls

_WORKSPACES = {}


def _workspace():
    """The scratch memory that a program keeps for the calls of a stream (calls on another one may run beside them)."""
    from paper_2409_11600_amd import binding as B
    stream = B._stream()
    if stream not in _WORKSPACES:
        _WORKSPACES[stream] = B.Workspace("cuda:0")
    return _WORKSPACES[stream]


def _own(state):
    from paper_2409_11600_amd import binding as B
    call = state["case"]["call"]
    if call == "ln_fwd":
        y, s, mean, invstd = B.layernorm_fwd(state["x"], state["gamma"], state["beta"], eps=EPS, residual=state["residual"])
        return {"y": y, "mean": mean, "invstd": invstd, **({} if state["residual"] is None else {"sum": s})}
    if call == "ln_bwd":
        dx, dgamma, dbeta = B.layernorm_bwd(state["dy"], state["s"], state["gamma"], state["mean"], state["invstd"], dsum=state["dsum"], ws=_workspace())
        return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    if call == "glr_step":
        return {"y": B.glr_step(state["gi"], state["table"], state["bias"], slots=state["slots"]), "table": state["table"]}
    if call == "glr_fwd":
        y, h_last, saved = B.glr_fwd(state["gi"], state["bias"], h0=state["h0"], lengths=state["lengths"], ws=_workspace())
        return {"y": y, "h_last": h_last, "saved": saved}
    if call == "glr_bwd":
        dgi, dh0 = B.glr_bwd(state["gi"], state["saved"], state["bias"], dy=state["dy"], dh_last=state["dh_last"], lengths=state["lengths"], ws=_workspace())
        return {"dgi": dgi, "dh0": dh0}
    B.adamw8_step_multi(state["table"], ADAM["step"], state["seed"], ADAM["lr"], beta1=ADAM["beta1"], beta2=ADAM["beta2"], eps=ADAM["eps"],
                        grad_scale=state["grad_scale"])
    return _buffers(state)


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------------------------------------------- work, and the results in 64 bits

def work(case):
    call = case["call"]
    if call == "adamw8":
        n = sum(_sizes(case))
        blocks = sum(-(-k // BLOCK) for k in _sizes(case))
        return {"bytes": (20 + (2 if case["copy"] else 0)) * n + 16 * blocks, "flops": 20 * n}
    size = 4 if case["dtype"] == "f32" else 2
    if call == "ln_fwd":
        n, C = case["rows"] * case["C"], case["C"]
        return {"bytes": (4 if case["residual"] else 2) * size * n + 8 * case["rows"] + 8 * C, "flops": 8 * n}
    if call == "ln_bwd":
        n, C = case["rows"] * case["C"], case["C"]
        return {"bytes": (4 if case["residual"] else 3) * size * n + 8 * case["rows"] + 12 * C, "flops": 14 * n}
    N, H = case["N"], case["H"]
    if call == "glr_step":
        return {"bytes": N * H * (4 * size + 8) + 12 * H, "flops": 15 * N * H}
    n = case["T"] * N * H
    if case["ragged"]:                      # half of the steps on average; the others' y or dgi is zero and written
        read = n / 2
    else:
        read = n
    saved = 4 * -(-case["T"] // STRETCH) * N * H
    if call == "glr_fwd":
        return {"bytes": size * (3 * read + n) + saved + 8 * N * H + 12 * H, "flops": 15 * read}
    return {"bytes": size * (4 * read + 3 * n) + saved + 8 * N * H + 12 * H, "flops": 30 * read}


def _exact_adamw8(state):
    a = ADAM
    b1, b2 = float(np.float32(a["beta1"])), float(np.float32(a["beta2"]))
    wide = lambda k: state[k].double()
    spread = lambda scales: scales.double().repeat_interleave(BLOCK)
    g = wide("grad") * wide("grad_scale")
    m = b1 * wide("m") * spread(state["scale_m"]) + (1 - b1) * g
    v = b2 * (wide("r") * spread(state["scale_r"])) ** 2 + (1 - b2) * g * g
    r = v.sqrt()
    w = wide("w") * (1 - a["lr"] * a["weight_decay"]) - a["lr"] * (m / (1 - b1 ** a["step"])) / ((v / (1 - b2 ** a["step"])).sqrt() + a["eps"])
    bits = _random(_sizes(state["case"]), state["seed"], "cuda")
    out = {"w": w, "grad": torch.zeros_like(w)}
    for k, x, u in (("m", m, bits & 0xFFFF), ("r", r, bits >> 16)):
        scale = 2.0 ** torch.ceil(torch.log2(torch.clamp(x.abs().view(-1, BLOCK).amax(1), min=1e-300) / 448)).clamp(min=-126)
        y = x.abs() / spread(scale)
        step = 2.0 ** (torch.floor(torch.log2(torch.clamp(y, min=2.0 ** -6))) - 3)
        out[k], out["scale_" + k] = torch.copysign(torch.floor(y / step + u.double() / 65536) * step, x), scale
    out["r"] = torch.where(r > 0, out["r"].clamp(min=2.0 ** -9), out["r"])
    return out if state["w_lp"] is None else {**out, "w_lp": w}


def exact(case, seed):
    state = prepare(case, seed)
    call = case["call"]
    if call == "adamw8":
        return _exact_adamw8(state)
    d = {k: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v for k, v in state.items()}
    if call == "ln_fwd":
        s = state["x"].double()
        if state["residual"] is not None:       # the sum is an output in the inputs' type, and it is that which is normalised
            s = (s + d["residual"]).to(TYPES[case["dtype"]]).double()
        var, mean = torch.var_mean(s, dim=1, correction=0)
        invstd = 1 / torch.sqrt(var + EPS)
        out = {"y": (s - mean[:, None]) * invstd[:, None] * d["gamma"] + d["beta"], "mean": mean, "invstd": invstd}
        return out if state["residual"] is None else {**out, "sum": state["x"].double() + d["residual"]}
    if call == "ln_bwd":
        C = case["C"]
        xh = (d["s"] - d["mean"][:, None]) * d["invstd"][:, None]
        gh = d["dy"] * d["gamma"]
        dx = (C * gh - gh.sum(1, keepdim=True) - xh * (gh * xh).sum(1, keepdim=True)) * (d["invstd"] / C)[:, None]
        return {"dx": dx if d["dsum"] is None else dx + d["dsum"], "dgamma": torch.einsum("rc,rc->c", d["dy"], xh), "dbeta": d["dy"].sum(0)}
    H = case["H"]
    if call == "glr_step":
        z = d["gi"] + d["bias"]
        f, at = torch.sigmoid(z[:, :H]), state["slots"].long()
        table = d["table"].clone()
        table[at] = f * table[at] + torch.sigmoid(-z[:, :H]) * z[:, H:2 * H]
        return {"y": torch.sigmoid(z[:, 2 * H:]) * table[at], "table": table}
    # step by step, forwards and then backwards
    T, h, zero = case["T"], d["h0"], torch.zeros_like(d["h0"])
    back = call == "glr_bwd"
    states, ys = [h], []
    gates = lambda t: torch.sigmoid(d["gi"][t] + d["bias"])
    live = lambda t: None if state["lengths"] is None else (state["lengths"] > t)[:, None]
    pick = lambda t, a, b: a if live(t) is None else torch.where(live(t), a, b)
    for t in range(T):
        z = gates(t)
        h = pick(t, h + (torch.sigmoid(-(d["gi"][t, :, :H] + d["bias"][:H]))) * (d["gi"][t, :, H:2 * H] + d["bias"][H:2 * H] - h), h)
        if back or (t + 1) % STRETCH == 0:
            states.append(h)
        if not back:
            ys.append(pick(t, z[:, 2 * H:] * h, zero))
    if not back:
        return {"y": torch.stack(ys), "h_last": h, "saved": torch.stack(states[:-(-T // STRETCH)])}
    G, out = d["dh_last"], torch.zeros(d["gi"].shape, dtype=torch.float64, device="cuda")
    for t in reversed(range(T)):
        z = gates(t)
        f, o, c = z[:, :H], z[:, 2 * H:], d["gi"][t, :, H:2 * H] + d["bias"][H:2 * H]
        keep = torch.sigmoid(-(d["gi"][t, :, :H] + d["bias"][:H]))
        G = G + pick(t, d["dy"][t] * o, zero)
        out[t, :, :H] = pick(t, G * (states[t] - c) * f * keep, zero)
        out[t, :, H:2 * H] = pick(t, G * keep, zero)
        out[t, :, 2 * H:] = pick(t, d["dy"][t] * states[t + 1] * o * (1 - o), zero)
        G = pick(t, G * f, G)
    return {"dgi": out, "dh0": G}

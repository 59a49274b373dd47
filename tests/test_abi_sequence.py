"""Refusals of the calls for sequence models, on the host alone: bad sizes, strides, pointers and workspaces, before anything touches a device."""
import ctypes

import pytest
import torch

from paper_2409_11600_amd import binding as B

P = ctypes.c_void_p(0x10000)             # 16-byte aligned, never dereferenced on these paths
ODD = ctypes.c_void_p(0x10004)


def replaced(args, k, v):
    return [v if i == k else a for i, a in enumerate(args)]


def test_layer_norm_refusals():
    L = B.lib()
    good = dict(rows=4, C=8, dtype=B.NSK_F32, eps=1e-5)
    desc = lambda **k: ctypes.byref(B.nsk_layernorm_desc_t(*{**good, **k}.values()))
    fwd, bwd = [P] * 8 + [None], [P] * 9 + [0, P, 1 << 30, None]
    for bad in (dict(rows=0), dict(rows=-1), dict(C=0), dict(C=-5), dict(dtype=2), dict(rows=1 << 60)):
        assert L.nsk_layernorm_bwd_workspace_bytes(desc(**bad)) == 0
        assert L.nsk_layernorm_fwd(desc(**bad), *fwd) == B.NSK_ERR_BAD_DESC
        assert L.nsk_layernorm_bwd(desc(**bad), *bwd) == B.NSK_ERR_BAD_DESC
    assert L.nsk_layernorm_fwd(desc(C=(1 << 24) + 1), *fwd) == B.NSK_ERR_UNSUPPORTED and L.nsk_layernorm_bwd(desc(C=(1 << 24) + 1), *bwd) == B.NSK_ERR_UNSUPPORTED
    for eps in (0.0, -1.0, float("nan")):
        assert L.nsk_layernorm_fwd(desc(eps=eps), *fwd) == B.NSK_ERR_BAD_DESC
    assert L.nsk_layernorm_fwd(None, *fwd) == B.NSK_ERR_NULL and L.nsk_layernorm_bwd(None, *bwd) == B.NSK_ERR_NULL
    for k in (0, 5):                     # x, y
        assert L.nsk_layernorm_fwd(desc(), *replaced(fwd, k, None)) == B.NSK_ERR_NULL
    assert L.nsk_layernorm_fwd(desc(), *replaced(fwd, 1, None)) == B.NSK_ERR_BAD_DESC       # a place for a sum of one
    for k in range(8):
        assert L.nsk_layernorm_fwd(desc(), *replaced(fwd, k, ODD)) == B.NSK_ERR_ALIGNMENT
    for k in (0, 1, 4, 5, 6):            # s, dy, mean, invstd, dx
        assert L.nsk_layernorm_bwd(desc(), *replaced(bwd, k, None)) == B.NSK_ERR_NULL
    for k in range(9):
        assert L.nsk_layernorm_bwd(desc(), *replaced(bwd, k, ODD)) == B.NSK_ERR_ALIGNMENT
    need = L.nsk_layernorm_bwd_workspace_bytes(desc())
    assert need > 0
    assert L.nsk_layernorm_bwd(desc(), *replaced(bwd, 11, need - 1)) == B.NSK_ERR_WORKSPACE
    assert L.nsk_layernorm_bwd(desc(), *replaced(bwd, 10, None)) == B.NSK_ERR_WORKSPACE


def test_recurrence_refusals():
    L = B.lib()
    good = dict(T=40, N=3, H=8, dtype=B.NSK_F32, gi_t=0, gi_n=0, y_t=0, y_n=0)
    desc = lambda **k: ctypes.byref(B.nsk_glr_desc_t(*{**good, **k}.values()))
    fwd, bwd = [P] * 7 + [P, 1 << 40, None], [P] * 8 + [P, 1 << 40, None]
    bad_ones = [dict(T=0), dict(N=0), dict(H=0), dict(T=-1), dict(dtype=2), dict(gi_t=72), dict(gi_n=24), dict(gi_t=71, gi_n=24), dict(gi_t=72, gi_n=23), dict(gi_t=-72, gi_n=24),
                dict(gi_t=24, gi_n=24), dict(gi_t=30, gi_n=1000), dict(y_t=8, y_n=8), dict(y_t=24, y_n=7), dict(gi_t=1 << 60, gi_n=24), dict(T=1 << 30, N=1 << 30, H=1 << 20)]
    for bad in bad_ones:
        assert L.nsk_glr_saved_bytes(desc(**bad)) == 0 and L.nsk_glr_workspace_bytes(desc(**bad), B.NSK_PASS_FWD) == 0, bad
        assert L.nsk_glr_fwd(desc(**bad), *fwd) == B.NSK_ERR_BAD_DESC, bad
        assert L.nsk_glr_bwd(desc(**bad), *bwd) == B.NSK_ERR_BAD_DESC, bad
    for much in (dict(T=(1 << 30) + 1), dict(T=1 << 20, N=1 << 14, H=64), dict(T=1, N=1 << 26, H=1)):       # more threads than a launch has
        assert L.nsk_glr_fwd(desc(**much), *fwd) == B.NSK_ERR_UNSUPPORTED and L.nsk_glr_bwd(desc(**much), *bwd) == B.NSK_ERR_UNSUPPORTED, much
        assert L.nsk_glr_workspace_bytes(desc(**much), B.NSK_PASS_FWD) == 0
    assert L.nsk_glr_saved_bytes(desc()) == 3 * 3 * 8 * 4
    assert L.nsk_glr_saved_bytes(desc(gi_t=24, gi_n=960, y_t=8, y_n=320)) == 3 * 3 * 8 * 4      # batch-major
    assert L.nsk_glr_saved_bytes(desc(T=1, gi_t=1, gi_n=24)) == 3 * 8 * 4                        # the stride of a single step says nothing
    assert L.nsk_glr_fwd(None, *fwd) == B.NSK_ERR_NULL and L.nsk_glr_bwd(None, *bwd) == B.NSK_ERR_NULL
    assert L.nsk_glr_fwd(desc(), *replaced(fwd, 0, None)) == B.NSK_ERR_NULL
    assert L.nsk_glr_fwd(desc(), *replaced(replaced(fwd, 4, None), 5, None)) == B.NSK_ERR_NULL   # neither y nor h_last
    for k in range(7):
        assert L.nsk_glr_fwd(desc(), *replaced(fwd, k, ODD)) == B.NSK_ERR_ALIGNMENT, k
    for k in (0, 3, 6):                  # gi, saved, dgi
        assert L.nsk_glr_bwd(desc(), *replaced(bwd, k, None)) == B.NSK_ERR_NULL
    assert L.nsk_glr_bwd(desc(), *replaced(replaced(bwd, 4, None), 5, None)) == B.NSK_ERR_NULL   # neither dy nor dh_last
    for k in range(8):
        assert L.nsk_glr_bwd(desc(), *replaced(bwd, k, ODD)) == B.NSK_ERR_ALIGNMENT, k
    long = dict(T=60000, N=1, H=64)      # sizes whose steps are shared out, if any are
    for which, call, args in ((B.NSK_PASS_FWD, L.nsk_glr_fwd, fwd), (B.NSK_PASS_DGRAD, L.nsk_glr_bwd, bwd)):
        need = L.nsk_glr_workspace_bytes(desc(**long), which)
        if need:
            assert call(desc(**long), *args[:-2], need - 1, None) == B.NSK_ERR_WORKSPACE
            assert call(desc(**long), *args[:-3], None, need, None) == B.NSK_ERR_WORKSPACE
    assert L.nsk_glr_workspace_bytes(desc(**long), B.NSK_PASS_WGRAD) == 0


def test_token_refusals():
    L = B.lib()
    args = [P] * 5 + [None]
    for sizes in ((B.NSK_F32, 0, 8, 4), (B.NSK_F32, 2, 0, 4), (B.NSK_F32, 2, 8, 0), (3, 2, 8, 4), (B.NSK_BF16, -1, 8, 4)):
        assert L.nsk_glr_step(*sizes, *args) == B.NSK_ERR_BAD_DESC
    assert L.nsk_glr_step(B.NSK_F32, 1 << 26, 8, 4, *args) == B.NSK_ERR_UNSUPPORTED
    for k in (0, 3):                     # gi, state
        assert L.nsk_glr_step(B.NSK_F32, 2, 8, 4, *replaced(args, k, None)) == B.NSK_ERR_NULL
    for k in range(5):
        assert L.nsk_glr_step(B.NSK_F32, 2, 8, 4, *replaced(args, k, ODD)) == B.NSK_ERR_ALIGNMENT


def test_optimizer_refusals():
    L = B.lib()
    hyper = dict(step=1, seed=0, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8)

    def call(count=1, grad_scale=None, fields=None, no_table=False, **k):
        rec = dict(w=P, grad=P, m=P, r=P, scale_m=P, scale_r=P, w_lp=P, n=10, weight_decay=0.0)
        tab = (B.nsk_param8_t * 2)()
        for i, f in enumerate(({}, fields or {})):      # the second record is the bad one: nothing is launched for the first
            tab[i] = B.nsk_param8_t(*{**rec, **f}.values())
        return L.nsk_adamw8_step_multi(2 * count, None if no_table else tab, *{**hyper, **k}.values(), grad_scale, None)

    assert call(count=0) == B.NSK_ERR_BAD_DESC and call(count=-1) == B.NSK_ERR_BAD_DESC
    for bad in (dict(step=0), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=float("nan"))):
        assert call(**bad) == B.NSK_ERR_BAD_DESC
    assert call(no_table=True) == B.NSK_ERR_NULL
    assert call(fields=dict(n=0)) == B.NSK_ERR_BAD_DESC
    for k in ("w", "grad", "m", "r", "scale_m", "scale_r"):
        assert call(fields={k: None}) == B.NSK_ERR_NULL
    for k in ("w", "grad", "m", "r", "w_lp"):
        assert call(fields={k: ODD}) == B.NSK_ERR_ALIGNMENT
    for k in ("scale_m", "scale_r"):
        assert call(fields={k: ctypes.c_void_p(0x10002)}) == B.NSK_ERR_ALIGNMENT
    assert call(grad_scale=ctypes.c_void_p(0x10002)) == B.NSK_ERR_ALIGNMENT


def test_binding_refusals():
    """What the binding's own checks turn away, on tensors of the host (none of them reaches the library)."""
    z = torch.zeros
    with pytest.raises(TypeError):
        B.layernorm_fwd(z(4, 8, dtype=torch.float16))
    with pytest.raises(ValueError):
        B.layernorm_fwd(z(4, 8))                                    # not on the GPU
    for k in (dict(gamma=z(7)), dict(beta=z(8, dtype=torch.bfloat16)), dict(residual=z(4, 9)), dict(residual=z(4, 8, dtype=torch.bfloat16)), dict(save_mean=z(5))):
        with pytest.raises(ValueError):
            B.layernorm_fwd(z(4, 8), **k)
    with pytest.raises(ValueError):
        B.layernorm_bwd(z(4, 8), z(4, 8), z(8), z(4), z(5))
    with pytest.raises(ValueError):
        B.glr_fwd(z(5, 2, 10))                                      # no three gates
    for k in (dict(bias=z(11)), dict(h0=z(2, 5)), dict(lengths=z(2)), dict(lengths=z(3, dtype=torch.int32)), dict(y=z(5, 2, 3)), dict(saved=z(2, 2, 4))):
        with pytest.raises(ValueError):
            B.glr_fwd(z(5, 2, 12), **k)
    gi = z(5, 2, 12)
    for bad in (gi[:1].expand(5, 2, 12), z(5, 2, 24)[..., ::2]):      # rows that overlap, rows with gaps
        with pytest.raises(ValueError):
            B._rows_ptr(bad)
    with pytest.raises(ValueError):
        B.glr_step(z(2, 10), z(2, 3))
    with pytest.raises(ValueError):
        B.glr_step(z(2, 12), z(2, 5))
    n = 300
    state = B.adamw8_state(n, "cpu")
    assert [t.numel() for t in state] == [n, n, 2, 2]
    with pytest.raises(AssertionError):
        B.param8_table([(z(n), z(n - 1), *state, None, 0.0)])
    with pytest.raises(AssertionError):
        B.param8_table([(z(n), z(n), state[0], state[1], state[2], z(1), None, 0.0)])


def test_more_tokens_than_places():
    """Tokens without slots are those of the first places: more of them are turned away before any state has moved on."""
    from types import SimpleNamespace
    from paper_2409_11600_amd.linear_recurrent import TokenStream
    stream = TokenStream(SimpleNamespace(H=4, L=2, device="cpu", w={"table": torch.zeros(5, 4)}), 3)
    with pytest.raises(ValueError, match="4 tokens"):
        stream.step(torch.zeros(4, dtype=torch.int32))


def test_an_outgrown_workspace_is_kept():
    """What a captured graph or another stream's work may still use is not handed back while the workspace lives; no call that fits makes a new buffer, and ones that want
    a little more each time do not make a thousand."""
    import gc
    import weakref
    ws = B.Workspace("cpu")
    assert ws.get(0) == (None, 0)
    at, size = ws.get(64)
    assert size == 64 and ws.get(16) == (at, 64) and ws.get(64) == (at, 64)
    first = weakref.ref(ws.buf)
    assert ws.get(1 << 20)[1] == 1 << 20 and ws.get(100)[1] == 1 << 20
    gc.collect()
    assert first() is not None and first().data_ptr() == at
    seen = set()
    for n in range(1000, 2000):
        at, size = (ws if n > 1000 else (ws := B.Workspace("cpu"))).get(n)
        assert size == n and ws.buf.data_ptr() == at and ws.buf.numel() >= n
        seen.add(at)
    assert len(seen) <= 3 and sum(b.numel() for b in ws.outgrown) <= 2 * ws.buf.numel()

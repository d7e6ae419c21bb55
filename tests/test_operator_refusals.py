"""Calls of the operators around stage (b) that are refused, before any device call: the error code of
each argument error, and the binding's checks.  CPU only.  The context handed to the C calls is a block
of zeros, which is all that the argument checks look at; no call here gets past them."""
import ctypes as C

import pytest
import torch

from paper_2602_14338_b200 import binding as B

INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3
P = 4096                                    # a "pointer" that is aligned; never followed


@pytest.fixture(scope="module")
def lib():
    from paper_2602_14338_b200 import build

    build.build()
    return B.load_library()


@pytest.fixture(scope="module")
def fake():
    return C.create_string_buffer(1 << 16)


def cfg(dtype=B.AERO_BF16):
    return C.byref(B.cfg_default(dtype=dtype))


def test_rmsnorm_refusals(lib, fake):
    def fwd(ctx=fake, c=None, T=4, d=64, x=P, r=P, gamma=P, eps=1e-6, s=P, h=P, rstd=P, q=P, qs=P):
        return lib.aero_rmsnorm_fwd(ctx, c or cfg(), T, d, x, r, gamma, eps, s, h, rstd, q, qs)

    assert fwd(ctx=None) == INVALID and fwd(x=None) == INVALID and fwd(gamma=None) == INVALID
    assert fwd(T=-1) == INVALID and fwd(T=1 << 31) == INVALID and fwd(d=0) == INVALID
    assert fwd(eps=0.0) == INVALID and fwd(eps=float("nan")) == INVALID
    assert fwd(q=None) == INVALID and fwd(qs=None) == INVALID              # q and its scales only together
    assert fwd(s=None, h=None, rstd=None, q=None, qs=None) == INVALID      # nothing to write
    assert fwd(x=P + 1) == INVALID and fwd(h=P + 1) == INVALID             # not element-aligned
    assert fwd(d=16385) == UNSUPPORTED and fwd(c=cfg(7)) == UNSUPPORTED

    need = lib.aero_rmsnorm_workspace_bytes(4, 64)
    assert need >= 4 * 64 * 4

    def bwd(ctx=fake, T=4, d=64, dh=P, ds=None, s=P, gamma=P, rstd=P, dx=P, dg=P, ws=P, wsb=need):
        return lib.aero_rmsnorm_bwd(ctx, cfg(), T, d, dh, ds, s, gamma, rstd, dx, dg, 0, ws, wsb)

    for name in ("dh", "s", "gamma", "rstd", "dx", "dg", "ws", "ctx"):
        assert bwd(**{name: None}) == INVALID, name
    assert bwd(ws=P + 16) == INVALID and bwd(wsb=need - 1) == WORKSPACE and bwd(d=20000) == UNSUPPORTED
    assert bwd(ds=P + 1) == INVALID

    def quant(ctx=fake, T=4, d=64, x=P, q=P, qs=P):
        return lib.aero_quantize_rows(ctx, cfg(), T, d, x, q, qs)

    assert quant(ctx=None) == INVALID and quant(x=None) == INVALID and quant(q=None) == INVALID and quant(qs=None) == INVALID
    assert quant(d=16385) == UNSUPPORTED and quant(x=P + 1) == INVALID


def test_statistics_of_the_norm_over_gamma_are_refused(lib, fake):
    """gamma is read by other rows while a row's rstd and q_scale are written (same type, and same shape where T = d)."""
    def fwd(gamma, rstd, q, qs):
        return lib.aero_rmsnorm_fwd(fake, cfg(B.AERO_FP32), 64, 64, 2 * P, None, gamma, 1e-6, None, None, rstd, q, qs)

    assert fwd(P, P, None, None) == INVALID and fwd(P, None, 3 * P, P) == INVALID


def test_embed_refusals(lib, fake):
    def fwd(ctx=fake, T=4, d=64, V=10, y=P, W=P, X=P, c=None):
        return lib.aero_embed_fwd(ctx, c or cfg(), T, d, V, y, W, 1.0, X)

    assert fwd(ctx=None) == INVALID and fwd(y=None) == INVALID and fwd(W=None) == INVALID and fwd(X=None) == INVALID
    assert fwd(V=0) == INVALID and fwd(T=-1) == INVALID and fwd(d=-8) == INVALID and fwd(W=P + 1) == INVALID
    assert fwd(d=65537) == UNSUPPORTED and fwd(c=cfg(3)) == UNSUPPORTED

    need = lib.aero_embed_workspace_bytes(5000, 64, 10)
    assert need > 4 * 4 * 5000 and lib.aero_embed_workspace_bytes(4, 64, 10) <= 256

    def bwd(ctx=fake, T=5000, d=64, V=10, y=P, dX=P, dW=P, ws=P, wsb=need):
        return lib.aero_embed_bwd(ctx, cfg(), T, d, V, y, dX, 1.0, dW, 1, ws, wsb)

    for name in ("ctx", "y", "dX", "dW", "ws"):
        assert bwd(**{name: None}) == INVALID, name
    assert bwd(ws=P + 16) == INVALID and bwd(wsb=need - 1) == WORKSPACE and bwd(T=1 << 31) == INVALID


def test_lmhead_q8_refusals(lib, fake):
    def call(ctx=fake, T=4, d=64, V=10, h=P, hs=P, w=P, ws=P, dt=B.AERO_BF16, out=P):
        return lib.aero_lmhead_q8(ctx, T, d, V, h, hs, w, ws, dt, out)

    for name in ("ctx", "h", "hs", "w", "ws", "out"):
        assert call(**{name: None}) == INVALID, name
    assert call(T=-1) == INVALID and call(V=0) == INVALID and call(d=0) == INVALID
    assert call(T=(1 << 30) + 1) == INVALID
    assert call(d=72) == UNSUPPORTED and call(d=65552) == UNSUPPORTED and call(dt=5) == UNSUPPORTED
    assert call(h=P + 8) == INVALID and call(w=P + 8) == INVALID and call(out=P + 1) == INVALID


def test_distill_refusals(lib, fake):
    T, d, V, R, K = 300, 64, 200, 3, 5
    need = (lib.aero_distill_fwd_workspace_bytes(T, d, V, R, K), lib.aero_distill_bwd_workspace_bytes(T, d, V, R, K, 128, 1),
            lib.aero_distill_fwd_bwd_workspace_bytes(T, d, V, R, K, 128, 1))

    def args(kw):
        a = dict(ctx=fake, c=cfg(), T=T, d=d, V=V, R=R, K=K, H=P, W=P, ids=P, logits=P, tlse=None, cs=P, w=P, keep=P,
                 lse=P, kl=P, loss=P, met=None, gs=1.0, dH=P, dW=P, dt=1, acc=0, ws=P, wsb=None)
        a.update(kw)
        return a

    def fwd(**kw):
        a = args(kw)
        return lib.aero_distill_fwd(*[a[k] for k in "ctx c T d V R K H W ids logits tlse cs w keep lse kl loss met ws".split()],
                                    need[0] if a["wsb"] is None else a["wsb"])

    def bwd(**kw):
        a = args(kw)
        return lib.aero_distill_bwd(*[a[k] for k in "ctx c T d V R K H W ids logits tlse cs w keep lse gs dH dW dt acc ws".split()],
                                    need[1] if a["wsb"] is None else a["wsb"])

    def both(**kw):
        a = args(kw)
        return lib.aero_distill_fwd_bwd(
            *[a[k] for k in "ctx c T d V R K H W ids logits tlse cs w keep lse kl loss met gs dH dW dt acc ws".split()],
            need[2] if a["wsb"] is None else a["wsb"])

    for call, own in ((fwd, "lse kl loss"), (bwd, "lse dH dW"), (both, "lse kl loss dH dW")):
        for name in ("ctx H W ids logits cs w keep ws " + own).split():
            assert call(**{name: None}) == INVALID, name
        assert call(K=0) == INVALID and call(T=-1) == INVALID and call(T=1 << 31) == INVALID and call(R=-1) == INVALID
        assert call(K=257) == UNSUPPORTED and call(d=96) == UNSUPPORTED and call(c=cfg(9)) == UNSUPPORTED
        assert call(c=cfg(B.AERO_FP32), d=1025) == UNSUPPORTED
        assert call(H=P + 8) == INVALID and call(W=P + 8) == INVALID and call(ws=P + 16) == INVALID
        assert call(wsb=64) == WORKSPACE
    for call in (bwd, both):
        assert call(dH=P + 8) == INVALID and call(dW=P + 4) == INVALID
        assert call(dt=7) == UNSUPPORTED and call(dt=B.AERO_BF16, acc=1) == INVALID
        assert call(dt=B.AERO_BF16, c=cfg(B.AERO_FP32)) == UNSUPPORTED
    # a bf16 dW of several chunks needs room for its fp32 sums; of one chunk it does not
    assert both(dt=B.AERO_BF16) == WORKSPACE and bwd(dt=B.AERO_BF16) == WORKSPACE
    size = lambda chunk, dt: lib.aero_distill_fwd_bwd_workspace_bytes(T, d, V, R, K, chunk, dt)
    assert size(128, B.AERO_BF16) - size(128, B.AERO_FP32) >= 4 * V * d
    assert size(T + 128 * (R + 2), B.AERO_BF16) == size(T + 128 * (R + 2), B.AERO_FP32)


def test_binding_checks_type_shape_device_and_layout():
    ctx = B.Context.__new__(B.Context)
    ctx.device = torch.device("cpu")
    ctx.h = None
    x = torch.zeros(4, 8)
    assert ctx._arg(None, torch.float32, (4, 8), "x") is None
    assert ctx._arg(x, torch.float32, (4, 8), "x") == x.data_ptr()
    with pytest.raises(B.AeroError, match="shape"):
        ctx._arg(x, torch.float32, (4, 9), "x")
    with pytest.raises(B.AeroError, match="dtype"):
        ctx._arg(x, torch.bfloat16, (4, 8), "x")
    with pytest.raises(B.AeroError, match="contiguous"):
        ctx._arg(torch.zeros(8, 4).t(), torch.float32, (4, 8), "x")
    ctx.device = torch.device("cuda", 1)
    with pytest.raises(B.AeroError, match="cuda:1"):
        ctx._arg(x, torch.float32, (4, 8), "x")

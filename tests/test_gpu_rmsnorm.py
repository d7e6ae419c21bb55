"""GPU tests of the final RMS norm (aero_rmsnorm_fwd / _bwd) and the 8-bit rows (aero_quantize_rows)
against the fp64 statement.

Tolerances.  u = 2^-24 is fp32's rounding, HALF[t] = eps(t)/2 the rounding of an output.  A sum of n
fp32 terms held as partial sums is off by at most depth * u times the sum of magnitudes; the depth here
is at most 32 terms per thread + 5 shuffles + 32 warps, below 2^7, so 2^-17 of the magnitudes covers the
sum and the handful of products after it."""
import numpy as np
import pytest
import torch

from oracle import model_ends as M
from paper_2602_14338_b200 import binding as B

pytestmark = pytest.mark.gpu

F32 = 2.0 ** -17
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(0)
    yield c
    assert c.last_status() == 0
    c.close()


def cfg_of(dtype):
    return B.cfg_default(dtype=B.AERO_BF16 if dtype == "bf16" else B.AERO_FP32)


def rows(T, d, dt, seed, shift=0):
    """[T,d] values of very different row scales; `shift` elements off a 16-byte boundary."""
    g = torch.Generator().manual_seed(seed)
    v = torch.randn(T, d, generator=g) * torch.exp(2.0 * torch.randn(T, 1, generator=g))
    flat = torch.empty(T * d + shift, dtype=dt, device="cuda")
    out = flat[shift:].view(T, d)
    out.copy_(v)
    return out


def f64(t):
    return t.double().cpu().numpy()


SHAPES = [(1, 1), (1, 1536), (3, 8), (7, 33), (5, 200), (300, 1536), (33, 3584), (2, 4104), (2, 8192), (2, 16384), (3, 4099),
          (700, 64), (2, 16383)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,d", SHAPES)
@pytest.mark.parametrize("residual,shift", [(True, 0), (False, 0), (True, 1)])
def test_forward(ctx, dtype, T, d, residual, shift):
    dt = DT[dtype]
    x, r = rows(T, d, dt, 1, shift), rows(T, d, dt, 2) if residual else None
    gamma = (1 + 0.3 * torch.randn(d, generator=torch.Generator().manual_seed(3))).to(dt).cuda()
    out = ctx.rmsnorm_fwd(cfg_of(dtype), x, gamma, residual=r, eps=1e-5, quant=True)
    s, rstd, h = M.rmsnorm_fwd(f64(x), f64(gamma), None if r is None else f64(r), 1e-5)
    assert (np.abs(f64(out["rstd"]) - rstd) <= F32 * rstd).all()
    if residual:
        mag = np.abs(f64(x)) + np.abs(f64(r))
        assert (np.abs(f64(out["sum"]) - s) <= HALF[dt] * np.abs(s) + 2.0 ** -23 * mag).all()
    # (the sum of two rows is off by u of their magnitudes, which the norm passes on)
    slack = F32 * np.abs(h) + (2.0 ** -23 * mag * rstd[:, None] * np.abs(f64(gamma)) if residual else 0)
    assert (np.abs(f64(out["h"]) - h) <= HALF[dt] * np.abs(h) + slack).all()
    step = M.row_scales(h)
    assert (np.abs(f64(out["q_scale"]) - step) <= 2 * F32 * step).all()
    q = out["q"].cpu().numpy().astype(np.float64)
    assert np.abs(q).max() <= 127
    assert (np.abs(q * step[:, None] - h) <= 0.5 * step[:, None] * (1 + 1e-2)).all()


def test_forward_outputs_are_optional_and_may_be_the_inputs(ctx):
    cfg = cfg_of("bf16")
    x, r = rows(9, 1536, torch.bfloat16, 5), rows(9, 1536, torch.bfloat16, 6)
    gamma = torch.ones(1536, dtype=torch.bfloat16, device="cuda")
    ref = ctx.rmsnorm_fwd(cfg, x, gamma, residual=r)
    only = ctx.rmsnorm_fwd(cfg, x, gamma, residual=r, h=False)
    assert set(only) == {"rstd", "sum"} and torch.equal(only["sum"], ref["sum"])
    x2, r2 = x.clone(), r.clone()
    out = ctx.rmsnorm_fwd(cfg, x2, gamma, residual=r2, out=dict(sum=r2, h=x2))
    assert out["sum"] is r2 and torch.equal(r2, ref["sum"]) and torch.equal(x2, ref["h"])


def test_outputs_of_an_earlier_call_are_not_returned_as_this_ones(ctx):
    cfg = cfg_of("bf16")
    gamma = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    first = ctx.rmsnorm_fwd(cfg, rows(9, 64, torch.bfloat16, 5), gamma, quant=True)
    assert set(first) == {"rstd", "h", "q", "q_scale"}
    again = ctx.rmsnorm_fwd(cfg, rows(9, 64, torch.bfloat16, 6), gamma, out=first)
    assert set(again) == {"rstd", "h"} and again["h"] is first["h"]
    again = ctx.rmsnorm_fwd(cfg, rows(9, 64, torch.bfloat16, 6), gamma, h=False, quant=True, out=first)
    assert set(again) == {"rstd", "q", "q_scale"} and again["q"] is first["q"]


def test_rows_of_zeros_nan_and_infinities(ctx):
    cfg = cfg_of("fp32")
    x = torch.ones(5, 96, device="cuda")
    x[0] = 0
    x[1, 7] = float("nan")
    x[2, 3] = float("inf")
    x[3] = 1e-38                                   # 127 / max would overflow without care
    gamma = torch.ones(96, device="cuda")
    out = ctx.rmsnorm_fwd(cfg, x, gamma, eps=1e-6, quant=True)
    assert out["q_scale"][0] == 0 and not out["q"][0].any() and not out["h"][0].any()
    assert torch.isnan(out["h"][1]).all() and torch.isnan(out["q_scale"][1])
    assert not torch.isfinite(out["q_scale"][2])
    assert torch.equal(out["q"][4], torch.full((96,), 127, dtype=torch.int8, device="cuda"))
    q, scale = ctx.quantize_rows(cfg, x)
    assert scale[0] == 0 and not q[0].any() and torch.isnan(scale[1]) and torch.isinf(scale[2])
    assert (q[3] == 127).all() and (q[4] == 127).all()
    # rows next to the bad ones are untouched by them
    assert torch.allclose(out["h"][4], torch.ones(96, device="cuda"), atol=1e-5)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("dtype,d", [("fp32", 96), ("bf16", 1536), ("bf16", 3584), ("fp32", 3584), ("bf16", 97), ("fp32", 5001)])
def test_a_gamma_that_is_no_number_shows_in_the_scale(ctx, dtype, d, bad):
    """A row per warp, per block in whole vectors and in single elements: h is no number in that column, and the 8-bit row's scale
    says so too."""
    x = torch.ones(3, d, dtype=DT[dtype], device="cuda")
    x[1] = 0.5
    gamma = torch.ones(d, dtype=DT[dtype], device="cuda")
    gamma[d - 7] = bad
    out = ctx.rmsnorm_fwd(cfg_of(dtype), x, gamma, quant=True)
    assert not torch.isfinite(out["h"][:, d - 7]).any() and torch.isfinite(out["h"][:, :d - 7]).all()
    assert not torch.isfinite(out["q_scale"]).any()
    assert torch.isfinite(out["rstd"]).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,d", SHAPES + [(1300, 96)])
@pytest.mark.parametrize("dsum,shift", [(True, 0), (False, 0), (True, 1)])
def test_backward(ctx, dtype, T, d, dsum, shift):
    dt = DT[dtype]
    s, dh = rows(T, d, dt, 11, shift), rows(T, d, dt, 12)
    ds = rows(T, d, dt, 13) if dsum else None
    gamma = (1 + 0.3 * torch.randn(d, generator=torch.Generator().manual_seed(3))).to(dt).cuda()
    rstd = torch.rsqrt(s.double().square().mean(1) + 1e-5).float()
    dx, dg = ctx.rmsnorm_bwd(cfg_of(dtype), dh, s, gamma, rstd, dsum=ds)
    S, DH, G, R = f64(s), f64(dh), f64(gamma), f64(rstd)
    rdx, rdg = M.rmsnorm_bwd(DH, S, G, R, None if ds is None else f64(ds))
    hat = np.abs(S) * R[:, None]
    gdh = np.abs(DH * G)
    mag = R[:, None] * (gdh + hat * (gdh * hat).mean(axis=1, keepdims=True)) + (0 if ds is None else np.abs(f64(ds)))
    assert (np.abs(f64(dx) - rdx) <= HALF[dt] * np.abs(rdx) + F32 * mag).all()
    # dgamma: up to T / 592 rows in a block one after the other, then 592 / 32 + 32 partial sums
    depth = T / 592 + 64
    assert (np.abs(f64(dg) - rdg) <= depth * 2.0 ** -24 * (np.abs(DH) * hat).sum(axis=0) + 1e-30).all()
    # added to, and the same bits again
    base = torch.randn(d, device="cuda")
    _, dg2 = ctx.rmsnorm_bwd(cfg_of(dtype), dh, s, gamma, rstd, dsum=ds, dgamma=base.clone(), accumulate_dgamma=True)
    assert torch.equal(dg2, base + dg)
    dx3, dg3 = ctx.rmsnorm_bwd(cfg_of(dtype), dh.clone(), s, gamma, rstd, dsum=ds)
    assert torch.equal(dx3, dx) and torch.equal(dg3, dg)
    # dx over dh
    over = dh.clone()
    ctx.rmsnorm_bwd(cfg_of(dtype), over, s, gamma, rstd, dsum=ds, dx=over)
    assert torch.equal(over, dx) or shift


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,d", [(9, 1536), (700, 96), (5, 3584), (300, 97), (3, 5001)])
@pytest.mark.parametrize("shift", [0, 1])
def test_dx_over_each_of_its_inputs(ctx, dtype, T, d, shift):
    """dx may be the array of dh, of s or of dsum, in whole vectors and in single elements: the same bits as into one of its own."""
    dt = DT[dtype]
    s, dh, ds = rows(T, d, dt, 41, shift), rows(T, d, dt, 42, shift), rows(T, d, dt, 43, shift)
    gamma = (1 + 0.3 * torch.randn(d, generator=torch.Generator().manual_seed(3))).to(dt).cuda()
    rstd = torch.rsqrt(s.double().square().mean(1) + 1e-5).float()
    own = torch.empty(T * d + shift, dtype=dt, device="cuda")[shift:].view(T, d)
    _, want_dg = ctx.rmsnorm_bwd(cfg_of(dtype), dh, s, gamma, rstd, dsum=ds, dx=own)
    for i in range(3):
        a = [t.clone() if shift == 0 else rows(T, d, dt, 41 + k, shift) for k, t in enumerate((s, dh, ds))]
        dx, dg = ctx.rmsnorm_bwd(cfg_of(dtype), a[1], a[0], gamma, rstd, dsum=a[2], dx=a[i])
        assert dx is a[i] and torch.equal(dx, own) and torch.equal(dg, want_dg)


def test_no_rows(ctx):
    cfg = cfg_of("bf16")
    e = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    gamma = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    out = ctx.rmsnorm_fwd(cfg, e, gamma, quant=True)
    assert out["h"].shape == (0, 64) and out["q"].shape == (0, 64)
    dx, dg = ctx.rmsnorm_bwd(cfg, e, e, gamma, torch.empty(0, device="cuda"), dgamma=torch.full((64,), 7.0, device="cuda"))
    assert dx.shape == (0, 64) and not dg.any()
    q, scale = ctx.quantize_rows(cfg, e)
    assert q.shape == (0, 64) and scale.shape == (0,)


def test_captured_and_replayed(ctx):
    """Forward and backward in a CUDA graph, replayed on new contents of the same buffers; an eager call of
    another size in between does not disturb the graph's workspace."""
    side = torch.cuda.Stream()
    c = B.Context(0, stream=side)
    cfg = cfg_of("bf16")
    x = rows(40, 1536, torch.bfloat16, 21)
    dh = rows(40, 1536, torch.bfloat16, 22)
    gamma = torch.ones(1536, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        out = c.rmsnorm_fwd(cfg, x, gamma)
        c.rmsnorm_bwd(cfg, dh, x, gamma, out["rstd"])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        out = c.rmsnorm_fwd(cfg, x, gamma)
        dx, dg = c.rmsnorm_bwd(cfg, dh, x, gamma, out["rstd"])
    for seed in (31, 32):
        x.copy_(rows(40, 1536, torch.bfloat16, seed))
        dh.copy_(rows(40, 1536, torch.bfloat16, seed + 100))
        big = rows(3000, 1536, torch.bfloat16, seed)
        ctx.rmsnorm_bwd(cfg, big, big, gamma, torch.ones(3000, device="cuda"))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        want = ctx.rmsnorm_fwd(cfg, x, gamma)
        wdx, wdg = ctx.rmsnorm_bwd(cfg, dh, x, gamma, want["rstd"])
        assert torch.equal(out["h"], want["h"]) and torch.equal(dx, wdx) and torch.equal(dg, wdg)
    assert c.last_status() == 0
    del g
    c.close()

"""GPU tests of rows in 4-bit floating point (aero_quantize_fp4, aero_dequantize_fp4) and of the lm_head product of them
(aero_lmhead_fp4) against the fp64 statement.

Tolerances.  Scales and codes of bf16 rows are exact: quotients of values of 8, 4 and 3 significant bits are either half way between two
codes or at least 2^-8 of themselves from there, further than any rounding.  With fp32 rows a quotient within 2^-23 of half way may
go to either side, and so may a block's scale: the value is then one code further than the nearest, which is allowed for quotients that
near alone.  The product: every term is exact; an instruction adds 64 of them to the accumulator, each aligned to the largest with at
least 24 bits (2^-23 of it lost at most, as much again for the accumulator), so that a sum of d terms is off by at most
(d / 64 + 64) 2^-23 of the sum of their magnitudes; two products with the rows' scales (powers of two here) are exact.
What is smaller than fp32's normal numbers (rows of 1e-30 against one another make 1e-58) may become zero: 2^-126."""
import numpy as np
import pytest
import torch

from oracle import pref_step as M
from paper_2602_14338_b200 import binding as B

pytestmark = pytest.mark.gpu

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


def f64(t):
    return t.double().cpu().numpy()


def values(T, d, dt, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, d, generator=g) * torch.exp(2.0 * torch.randn(T, 1, generator=g)) * torch.exp(torch.randn(d, generator=g))
    if T > 2:
        x[1] = 0.0                                            # a row of zeros
        x[2, : d // 2] = 0.0                                  # and blocks of zeros
    if T > 4:
        x[3] *= 1e-30
        x[4, 0] *= 1e6                                        # one large value: other blocks' scales leave e4m3's normal range
    return x.to(dt).cuda()


def decoded(rows):
    return M.fp4_values(rows.codes.cpu().numpy(), rows.scales.cpu().numpy(), None if rows.row_scale is None else f64(rows.row_scale),
                        rows.rows, rows.cols, rows.block)


SHAPES = [(1, 32), (3, 64), (1, 1536), (5, 224), (127, 256), (129, 288), (300, 1536), (33, 3584), (6, 4128), (5, 16384), (2, 65536)]


@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,d", SHAPES)
def test_rows_there_and_back(ctx, T, d, dtype, block):
    x = values(T, d, DT[dtype], 1)
    rows = ctx.quantize_fp4(cfg_of(dtype), x, block=block)
    value, scale, row = M.quantize_fp4(f64(x), block)
    got = decoded(rows)
    if block == 16:
        assert np.array_equal(f64(rows.row_scale), row)
    if dtype == "bf16":
        assert (got == value).all()
    else:
        off = got != value
        if off.any():
            # only where the quotient, or that of the block's scale, is within 2^-23 of half way
            wide = np.repeat(np.where(scale > 0, scale, 1.0), block, axis=1)
            y = np.abs(f64(x)) / wide
            mid = (M.E2M1[1:] + M.E2M1[:-1]) / 2
            near = np.abs(y[..., None] / mid - 1).min(-1) <= 2.0 ** -22
            assert np.all(near[off])
    # rows and columns that fill up the tiles are zeros
    at, half, where = M.fp4_places(T, d, block)
    codes, scales = rows.codes.cpu().numpy().copy(), rows.scales.cpu().numpy().copy()
    codes[at.ravel()] = 0
    scales[where.ravel()] = 0
    assert not codes.any() and not scales.any()
    for out in (torch.bfloat16, torch.float32):
        back = ctx.dequantize_fp4(rows, out_dtype=out)
        assert torch.equal(back.cpu().double(), torch.from_numpy(got).to(out).double())


def test_ties_of_codes_and_scales(ctx):
    """Every tie of the code with every scale, and neighbours of ties in bf16."""
    mids = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    scale = torch.arange(1, 127, dtype=torch.uint8).view(torch.float8_e4m3fn).float()
    tie = (mids[None, :] * scale[:, None]).bfloat16()
    assert torch.equal(tie.float(), mids[None, :] * scale[:, None])
    bits = tie.view(torch.int16)
    x = torch.zeros(126, 32, dtype=torch.bfloat16)
    x[:, 0] = 6 * scale                                       # the block's scale comes out as the code itself
    x[:, 1:8], x[:, 8:15] = tie, -tie
    x[:, 16] = 6 * scale
    x[:, 17:24], x[:, 24:31] = (bits + 1).view(torch.bfloat16), -((bits - 1).view(torch.bfloat16))
    x = torch.cat((x, torch.zeros(126, 32, dtype=torch.bfloat16)), 1)
    x[:, 32] = 2688                                           # keeps the row's scale at 1
    rows = ctx.quantize_fp4(cfg_of("bf16"), x.cuda(), block=16)
    assert torch.all(rows.row_scale == 1)
    value, _, _ = M.quantize_fp4(x.double().numpy(), 16)
    assert (decoded(rows) == value).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("block", [16, 32])
def test_rows_that_are_no_numbers(ctx, dtype, block):
    x = values(6, 96, DT[dtype], 2)
    x[1, 3], x[2, 40], x[5, 95] = float("nan"), float("inf"), float("-inf")
    back = ctx.dequantize_fp4(ctx.quantize_fp4(cfg_of(dtype), x, block=block)).cpu()
    nan = torch.zeros(6, 96, dtype=torch.bool)
    if block == 16:
        nan[[1, 2, 5]] = True
    else:
        nan[1, :32], nan[2, 32:64], nan[5, 64:] = True, True, True
    assert torch.equal(torch.isnan(back), nan) and torch.isfinite(back[~nan]).all()


@pytest.mark.parametrize("size", [2.0 ** -126, 2.0 ** -133, 3e38])
@pytest.mark.parametrize("block", [16, 32])
def test_smallest_and_largest_rows(ctx, size, block):
    x = (torch.randn(4, 64, generator=torch.Generator().manual_seed(3)).clamp(-1, 1).double() * size).bfloat16().cuda()
    rows = ctx.quantize_fp4(cfg_of("bf16"), x, block=block)
    value, _, row = M.quantize_fp4(f64(x), block)
    assert (decoded(rows) == value).all()


def product_of(ctx, T, d, V, block, out, seed=5):
    h, w = values(T, d, torch.bfloat16, seed), values(V, d, torch.bfloat16, seed + 1)
    cfg = cfg_of("bf16")
    hr, wr = ctx.quantize_fp4(cfg, h, block=block), ctx.quantize_fp4(cfg, w, block=block)
    z = torch.full((T + 1, V), 7.0, dtype=out, device="cuda")
    got = ctx.lmhead_fp4(hr, wr, out_dtype=out, out=z[:T])
    assert torch.all(z[T:] == 7.0)                            # rows behind the last are left as they were
    a, b = ctx.dequantize_fp4(hr, torch.float32).double(), ctx.dequantize_fp4(wr, torch.float32).double()
    return got.double(), a @ b.T, a.abs() @ b.abs().T


def check_product(got, want, size, d, out):
    tol = (d / 64 + 64) * 2.0 ** -23 * size + 2.0 ** -126
    assert torch.all((got - want).abs() <= tol + HALF[out] * (want.abs() + tol))


PRODUCTS = [(1, 32, 1), (1, 256, 128), (1, 1536, 1000), (2, 64, 31), (17, 288, 129), (61, 1536, 5000), (64, 3584, 777), (127, 512, 4097),
            (128, 256, 40000), (3, 16384, 300), (1, 65536, 33), (129, 256, 500), (200, 1536, 3001), (192, 64, 128), (193, 320, 40000),
            (385, 3584, 1000), (1000, 96, 260), (2048, 512, 2049), (150, 65536, 300)]


@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,d,V", PRODUCTS)
def test_product(ctx, T, d, V, block, out):
    got, want, size = product_of(ctx, T, d, V, block, out)
    check_product(got, want, size, d, out)


@pytest.mark.parametrize("T", [5, 300])
def test_captured_on_another_stream_beside_another_call(ctx, T):
    """A chain captured on a stream of its own and replayed while the first context runs the same on another stream, on other inputs."""
    d, V = 512, 3000
    cfg = cfg_of("bf16")
    x, w = values(T, d, torch.bfloat16, 1), values(V, d, torch.bfloat16, 2)
    want = ctx.lmhead_fp4(ctx.quantize_fp4(cfg, x), ctx.quantize_fp4(cfg, w), out_dtype=torch.float32)
    x2 = x.flip(0).contiguous()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    own = B.Context(0, stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        rows = own.quantize_fp4(cfg, x)
        z = own.lmhead_fp4(rows, own.quantize_fp4(cfg, w), out_dtype=torch.float32)
        back = own.dequantize_fp4(rows)
    for _ in range(3):
        z.fill_(float("nan"))
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            graph.replay()
        other = ctx.lmhead_fp4(ctx.quantize_fp4(cfg, x2), ctx.quantize_fp4(cfg, w), out_dtype=torch.float32)
        torch.cuda.synchronize()
        assert torch.equal(z, want) and torch.equal(other, want.flip(0))
    assert torch.equal(back, ctx.dequantize_fp4(ctx.quantize_fp4(cfg, x)))
    assert own.last_status() == 0
    del graph
    own.close()


@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("T", [1, 33, 128])
def test_scales_that_change_from_slab_to_slab(ctx, T, block):
    """A row of many slabs whose scales differ by powers of two from one slab of 256 columns to the next, up to 2^7 and back: a slab
    multiplied with scales of another one would be off by its whole size.  Several turns of the ring, many rows of W for each CTA."""
    d, V = 256 * 40, 148 * 160
    cfg = cfg_of("bf16")
    g = torch.Generator(device="cuda").manual_seed(9)
    size = torch.exp2(((torch.arange(d, device="cuda") // 256 * 5) % 8).float())
    h = (torch.randn(T, d, generator=g, device="cuda") * size).bfloat16()
    w = (torch.randn(V, d, generator=g, device="cuda") * size.flip(0)).bfloat16()
    hr, wr = ctx.quantize_fp4(cfg, h, block=block), ctx.quantize_fp4(cfg, w, block=block)
    a, b = ctx.dequantize_fp4(hr, torch.float32), ctx.dequantize_fp4(wr, torch.float32)
    got = ctx.lmhead_fp4(hr, wr, out_dtype=torch.float32)
    again = ctx.lmhead_fp4(hr, wr, out_dtype=torch.float32)
    assert torch.equal(got, again)
    for v in range(0, V, 4736):
        part = b[v:v + 4736].double()
        check_product(got[:, v:v + 4736].double(), a.double() @ part.T, a.double().abs() @ part.abs().T, d, torch.float32)


@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T", [1, 7, 61, 130, 700])
def test_product_of_rows_that_are_no_numbers(ctx, T, block, out):
    """A NaN or an infinity in a row of tokens or of W: that row's logits are NaN, all others stay what they are."""
    d, V = 288, 700
    h, w = values(T, d, torch.bfloat16, 5), values(V, d, torch.bfloat16, 6)
    cfg = cfg_of("bf16")
    want = ctx.lmhead_fp4(ctx.quantize_fp4(cfg, h, block=block), ctx.quantize_fp4(cfg, w, block=block), out_dtype=out)
    rows, cols = sorted({0, T // 2, T - 1}), [0, 130, 255, 699]
    for i, r in enumerate(rows):
        h[r, (37 * i) % d] = (float("nan"), float("inf"), -float("inf"))[i]
    for i, c in enumerate(cols):
        w[c, (101 * i + 5) % d] = (float("inf"), float("nan"), -float("inf"), float("nan"))[i]
    got = ctx.lmhead_fp4(ctx.quantize_fp4(cfg, h, block=block), ctx.quantize_fp4(cfg, w, block=block), out_dtype=out)
    nan = torch.zeros(T, V, dtype=torch.bool, device="cuda")
    nan[rows], nan[:, cols] = True, True
    assert torch.equal(torch.isnan(got), nan) and torch.equal(got[~nan], want[~nan])

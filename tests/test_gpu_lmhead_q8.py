"""GPU tests of the 8-bit lm_head product (aero_lmhead_q8) against the exact integer product in fp64.

Tolerance: the integer sum is exact; its conversion to fp32 and the two products with the scales are off
by 2^-24 each, the output's rounding by eps/2."""
import numpy as np
import pytest
import torch

from oracle import model_ends as M
from paper_2602_14338_b200 import binding as B

pytestmark = pytest.mark.gpu

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(0)
    yield c
    assert c.last_status() == 0
    c.close()


def problem(T, d, V, seed=0):
    rng = np.random.default_rng(seed)
    return (rng.integers(-128, 128, (T, d)).astype(np.int8), (rng.random(T) + 0.1).astype(np.float32),
            rng.integers(-128, 128, (V, d)).astype(np.int8), (rng.random(V) + 0.1).astype(np.float32))


SHAPES = [(1, 16, 1), (1, 64, 31), (1, 1536, 5000), (2, 48, 33), (15, 128, 257), (16, 144, 128), (17, 1536, 129), (61, 272, 4737),
          (100, 64, 1000), (128, 512, 300), (129, 128, 300), (160, 1536, 255), (161, 64, 513), (256, 256, 1000), (257, 80, 700),
          (600, 384, 2050), (1, 3584, 20000), (300, 3584, 1111)]


@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,d,V", SHAPES)
def test_product(ctx, T, d, V, out_dtype):
    h8, sh, w8, sw = problem(T, d, V, T + d + V)
    # the result lies inside a larger buffer whose other values must stay
    flat = torch.full(((T + 2) * V,), 77.0, dtype=out_dtype, device="cuda")
    out = flat[V:(T + 1) * V].view(T, V)
    t = lambda a: torch.from_numpy(a).cuda()
    got = ctx.lmhead_q8(t(h8), t(sh), t(w8), t(sw), out_dtype=out_dtype, out=out)
    ref = M.lmhead_q8(h8, sh, w8, sw)
    assert (np.abs(got.double().cpu().numpy() - ref) <= (HALF[out_dtype] + 4 * 2.0 ** -24) * np.abs(ref)).all()
    assert (flat[:V] == 77).all() and (flat[(T + 1) * V:] == 77).all()
    assert ctx.last_status() == 0


def test_largest_sums_are_exact(ctx):
    """The largest magnitude of the integer sum at the largest d: 128 * 128 * 65536 = 2^30."""
    d = 65536
    h8 = torch.full((3, d), -128, dtype=torch.int8, device="cuda")
    w8 = torch.full((40, d), -128, dtype=torch.int8, device="cuda")
    w8[7] = 127
    w8[9, ::2] = 127
    one = torch.ones(40, device="cuda")
    z = ctx.lmhead_q8(h8, one[:3].contiguous(), w8, one, out_dtype=torch.float32)
    assert (z[:, 0] == 2.0 ** 30).all() and (z[:, 7] == -128.0 * 127 * d).all() and (z[:, 9] == 64.0 * d).all()


def test_no_tokens(ctx):
    e = torch.empty(0, 64, dtype=torch.int8, device="cuda")
    w = torch.zeros(10, 64, dtype=torch.int8, device="cuda")
    assert ctx.lmhead_q8(e, torch.empty(0, device="cuda"), w, torch.ones(10, device="cuda")).shape == (0, 10)


@pytest.mark.parametrize("T", [3, 200])
def test_captured_and_replayed(ctx, T):
    side = torch.cuda.Stream()
    c = B.Context(0, stream=side)
    t = lambda a: torch.from_numpy(a).cuda()
    bufs = [t(a) for a in problem(T, 256, 777, 1)]
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        c.lmhead_q8(*bufs)
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        out = c.lmhead_q8(*bufs)
    for seed in (2, 3):
        for b, a in zip(bufs, problem(T, 256, 777, seed)):
            b.copy_(t(a))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ctx.lmhead_q8(*bufs))
    assert c.last_status() == 0
    del g
    c.close()

"""GPU tests of the tied embedding (aero_embed_fwd / _bwd) against the fp64 statement.

Tolerances: the lookup is one fp32 product (2^-24) and one rounding to the row's type (eps/2).  A token's
gradient is a sum of n rows, off by at most (n + 4) 2^-24 times the sum of their magnitudes."""
import numpy as np
import pytest
import torch

from oracle import model_ends as M
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


def tokens(T, V, kind, seed=0):
    rng = np.random.default_rng(seed)
    if kind == "same":
        y = np.full(T, V - 1)
    elif kind == "two":
        y = rng.integers(0, 2, T) * (V - 1)
    elif kind == "none":
        y = np.full(T, M.NO_TOKEN)
    else:
        y = np.minimum((V ** rng.random(T) - 1).astype(np.int64), V - 1)
        y = rng.permutation(V)[y]
        y[rng.random(T) < 0.05] = M.NO_TOKEN
    return y.astype(np.int32)


def shifted(a, dt, shift):
    flat = torch.empty(a.size + shift, dtype=dt, device="cuda")
    out = flat[shift:].view(*a.shape)
    out.copy_(torch.from_numpy(a))
    return out


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,V,d,shift", [(0, 5, 8, 0), (1, 1, 1, 0), (1, 1000, 1536, 0), (77, 300, 33, 0), (500, 1000, 3584, 0),
                                         (500, 1000, 200, 1), (3000, 7, 1032, 0)])
def test_lookup(ctx, dtype, T, V, d, shift):
    dt = DT[dtype]
    W = shifted(np.random.default_rng(1).standard_normal((V, d)), dt, shift)
    y = tokens(T, V, "text", 2)
    X = ctx.embed_fwd(cfg_of(dtype), W, torch.from_numpy(y).cuda(), scale=1.7)
    ref = M.embed_fwd(W.double().cpu().numpy(), y, float(np.float32(1.7)))
    assert (np.abs(X.double().cpu().numpy() - ref) <= (HALF[dt] + 2.0 ** -23) * np.abs(ref)).all()
    assert ctx.last_status() == 0


CASES = [(0, 9, 8, "text"), (1, 1, 1, "same"), (1, 1000, 1536, "text"), (5, 3, 33, "two"), (777, 500, 1536, "text"),
         (2048, 40, 264, "text"), (2049, 40, 264, "text"), (2100, 1, 24, "same"), (4096, 5000, 100, "text"),
         (4097, 3, 72, "two"), (9000, 150000, 40, "text"), (20000, 700, 136, "text"), (20000, 1000, 72, "same"),
         (2500, 33, 64, "none"), (70001, 511, 16, "text"), (6000, 512, 3, "text"), (33000, 262143, 8, "text"),
         (2816, 5000, 100, "text"), (2817, 5000, 100, "text"), (3500, 1, 8, "same"), (3500, 2, 8, "two"), (5000, 33, 64, "none"),
         (600000, 1000, 4, "text")]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T,V,d,kind", CASES)
def test_gradient(ctx, dtype, T, V, d, kind):
    dt = DT[dtype]
    cfg = cfg_of(dtype)
    dX = shifted(np.random.default_rng(3).standard_normal((T, d)) * 0.01, dt, 0)
    y = tokens(T, V, kind, 4)
    yt = torch.from_numpy(y).cuda()
    scale = 40.0
    dW = ctx.embed_bwd(cfg, dX, yt, V, scale=scale)
    ref, mag = M.embed_bwd(dX.double().cpu().numpy(), y, V, scale)
    n = np.bincount(y[y >= 0], minlength=V)[:, None]
    got = dW.double().cpu().numpy()
    assert (np.abs(got - ref) <= (n + 4) * 2.0 ** -24 * mag).all()
    assert not got[n[:, 0] == 0].any()
    # the same bits again, and added to what is there
    assert torch.equal(ctx.embed_bwd(cfg, dX, yt, V, scale=scale), dW)
    base = torch.randn(V, d, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
    acc = ctx.embed_bwd(cfg, dX, yt, V, scale=scale, dW=base.clone(), accumulate_dW=True)
    b64 = base.double().cpu().numpy()
    assert (np.abs(acc.double().cpu().numpy() - (b64 + ref)) <= (n + 4) * 2.0 ** -24 * (mag + np.abs(b64))).all()
    assert torch.equal(acc[torch.from_numpy(n[:, 0] == 0).cuda()], base[torch.from_numpy(n[:, 0] == 0).cuda()])
    assert ctx.last_status() == 0


@pytest.mark.parametrize("T", [300, 3000])
def test_gradient_of_unaligned_rows(ctx, T):
    y = tokens(T, 50, "text", 6)
    a = np.random.default_rng(7).standard_normal((T, 64))
    ref = ctx.embed_bwd(cfg_of("bf16"), shifted(a, torch.bfloat16, 0), torch.from_numpy(y).cuda(), 50)
    got = ctx.embed_bwd(cfg_of("bf16"), shifted(a, torch.bfloat16, 3), torch.from_numpy(y).cuda(), 50)
    assert torch.allclose(got, ref, rtol=1e-5, atol=1e-5)


@pytest.mark.parametrize("T", [300, 3000])
def test_bad_tokens_raise_the_status_bit_and_count_for_nothing(ctx, T):
    V, d = 100, 72
    y = tokens(T, V, "text", 8)
    bad = y.copy()
    bad[[3, 250]] = [V, -2]
    bad[17] = 2 ** 31 - 1
    good = np.where((bad < 0) | (bad >= V), M.NO_TOKEN, bad)
    dX = shifted(np.random.default_rng(9).standard_normal((T, d)), torch.bfloat16, 0)
    W = shifted(np.random.default_rng(9).standard_normal((V, d)), torch.bfloat16, 0)
    cfg = cfg_of("bf16")
    want = ctx.embed_bwd(cfg, dX, torch.from_numpy(good).cuda(), V)
    wantx = ctx.embed_fwd(cfg, W, torch.from_numpy(good).cuda())
    assert ctx.last_status() == 0
    assert torch.equal(ctx.embed_bwd(cfg, dX, torch.from_numpy(bad).cuda(), V), want)
    assert ctx.last_status() == B.AERO_ST_BAD_TARGET
    assert torch.equal(ctx.embed_fwd(cfg, W, torch.from_numpy(bad).cuda()), wantx)
    assert ctx.last_status() == B.AERO_ST_BAD_TARGET


def test_two_graphs_replayed_at_once_have_workspaces_of_their_own(ctx):
    V, d, T = 900, 256, 6000
    cfg = cfg_of("bf16")
    runs = []
    for k in range(2):
        side = torch.cuda.Stream()
        c = B.Context(0, stream=side)
        dX = shifted(np.random.default_rng(20 + k).standard_normal((T, d)), torch.bfloat16, 0)
        y = torch.from_numpy(tokens(T, V, "text", 30 + k)).cuda()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            c.embed_bwd(cfg, dX, y, V)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            dW = c.embed_bwd(cfg, dX, y, V)
        runs.append((side, c, g, dX, y, dW))
    for _ in range(20):
        for side, _, g, *_ in runs:
            with torch.cuda.stream(side):
                g.replay()
    torch.cuda.synchronize()
    for side, c, g, dX, y, dW in runs:
        assert torch.equal(dW, ctx.embed_bwd(cfg, dX, y, V))
        assert c.last_status() == 0


def test_gradient_of_the_most_tokens(ctx):
    """2^31 - 1 rows, the most a call takes: the rounded-up numbers of sort blocks and of tiles pass 32 bits on the way.  Rows of
    one element, 0 or 1, over 300 tokens, so that every sum is a whole number below 2^24 and exact in any order."""
    T, V, piece = 2 ** 31 - 1, 300, 1 << 27
    g = torch.Generator(device="cuda").manual_seed(9)
    y = torch.empty(T, dtype=torch.int32, device="cuda")
    dX = torch.empty(T, 1, dtype=torch.bfloat16, device="cuda")
    want = torch.zeros(V, dtype=torch.int64, device="cuda")
    for a in range(0, T, piece):
        n = min(piece, T - a)
        ids = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
        one = torch.randint(0, 2, (n,), generator=g, device="cuda", dtype=torch.int8)
        y[a:a + n], dX[a:a + n, 0] = ids, one
        want += torch.bincount(ids[one.bool()], minlength=V)
    y[-1], dX[-1] = V - 1, 1.0
    want[V - 1] += 1 - int(one[-1]) if int(ids[-1]) == V - 1 else 1
    if int(ids[-1]) != V - 1:
        want[int(ids[-1])] -= int(one[-1])
    del ids, one
    dW = ctx.embed_bwd(cfg_of("bf16"), dX, y, V)
    assert int(want.max()) < 2 ** 24 and torch.equal(dW[:, 0].long(), want) and torch.equal(dW[:, 0], want.float())
    dW = ctx.embed_bwd(cfg_of("bf16"), dX, y, V, dW=dW, accumulate_dW=True)
    assert torch.equal(dW[:, 0], 2 * want.float())
    assert ctx.last_status() == 0
    del y, dX, dW
    torch.cuda.empty_cache()                       # some 60 GB

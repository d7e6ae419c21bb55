"""GPU tests of the preference loss on pairs of rollouts (aero_pref_fwd, _bwd, _fwd_bwd) against the fp64 statement.

Tolerances.  A logit on the tensor cores is a chain of d / 16 additions that lose up to 2^-23 of the partial sums, which S, the largest
sum of |h w|, bounds; the sum of V exponentials adds one of 32 columns at a time, 2^-24 each, and ex2 is off by 2^-22: together
TOL = (d / 16 + 2) 2^-23 S + (V / 32 + 64) 2^-24 for a log-prob (fp32 path: (d + 2) 2^-24 S + (V + 64) 2^-24).  A rollout of n scored tokens
adds n of them (one, as a mean); a margin two rollouts, times beta; coef the loss's second derivative (1/4, 2 or 0) times that, and
its own rounding.  dz is rounded to bf16 twice at most, the outputs once: 2^-8 each of the magnitudes that enter; as a norm, three
independent roundings of 2^-8 / sqrt(3) at most are 4e-3, with coef's own error 6e-3."""
import numpy as np
import pytest
import torch

from oracle import pref_step as M
from paper_2602_14338_b200 import binding as B

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
KIND = dict(logistic=B.AERO_PREF_LOGISTIC, square=B.AERO_PREF_SQUARE, hinge=B.AERO_PREF_HINGE)
NAMES = ("logp", "lse", "ratio", "margin", "coef", "loss", "metrics")


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


def batch(T, d, V, cs, pairs, dtype, seed=0, lean=4.0):
    g = torch.Generator().manual_seed(seed)
    W = (torch.randn(V, d, generator=g) * d ** -0.5).to(DT[dtype]).cuda()
    y = torch.randint(0, V, (T,), generator=g)
    H = torch.randn(T, d, generator=g)
    H[::3] += lean * W.cpu().float()[y[::3]]
    y[torch.rand(T, generator=g) < 0.1] = B.AERO_NO_TOKEN
    ref = -torch.rand(T, generator=g) * 8
    return dict(H=H.to(DT[dtype]).cuda(), W=W, y=y.int().cuda(), cs=torch.tensor(cs, dtype=torch.int64, device="cuda"),
                pairs=torch.tensor(pairs, dtype=torch.int32, device="cuda").reshape(-1, 2), ref=ref.cuda())


def args(b):
    return b["H"], b["W"], b["y"], b["cs"], b["pairs"]


def oracle(b, **kw):
    return M.preference(f64(b["H"]), f64(b["W"]), b["y"].tolist(), b["cs"].tolist(), b["pairs"].tolist(), f64(b["ref"]), **kw)


def check_forward(b, got, want, kw, dtype):
    d, V = b["H"].shape[1], b["W"].shape[0]
    S = float((f64(b["H"].abs()) @ f64(b["W"].abs()).T).max()) if len(b["H"]) else 0.0
    tol = (d / 16 + 2) * 2.0 ** -23 * S + (V / 32 + 64) * 2.0 ** -24 if dtype == "bf16" else (d + 2) * 2.0 ** -24 * S + (V + 64) * 2.0 ** -24
    n = np.array([((b["y"][x:z] >= 0).sum().item() if not kw.get("mean") else 1) for x, z in zip(b["cs"].tolist(), b["cs"][1:].tolist())])
    tr = n * tol + 2.0 ** -23 * np.abs(want["ratio"]) + 1e-30
    assert (np.abs(f64(got["logp"]) - want["logp"]) <= tol + 2.0 ** -23 * np.abs(want["logp"])).all()
    scored = b["y"].cpu().numpy() >= 0
    assert (np.abs(f64(got["lse"]) - want["lse"]) <= tol + 2.0 ** -23 * np.abs(want["lse"]))[scored].all()
    assert (np.abs(f64(got["ratio"]) - want["ratio"]) <= tr).all()
    beta = kw.get("beta", 0.1)
    worst = 2 * beta * (tr.max() if len(tr) else 0.0)
    assert (np.abs(f64(got["margin"]) - want["margin"]) <= worst + 2.0 ** -22 * (np.abs(want["margin"]) + 1)).all()
    curve = dict(logistic=0.25, square=2.0, hinge=0.0)[kw.get("kind", "logistic")]
    weights = f64(b["weight"]) if "weight" in b else np.full(len(b["pairs"]), 1.0 / max(1, len(b["pairs"])))
    per = len(b["pairs"]) * (np.abs(weights).max() if len(weights) else 0.0) * beta * curve * worst
    assert (np.abs(f64(got["coef"]) - want["coef"]) <= 2.0 ** -22 * np.abs(want["coef"]).max(initial=0) + per).all()
    slope = 1 + 2 * np.abs(want["margin"]).max(initial=0)
    assert abs(got["loss"].item() - want["loss"]) <= np.abs(weights).sum() * slope * worst + 2.0 ** -22 * abs(want["loss"])
    m = f64(got["metrics"])
    assert m[3] == want["metrics"][3] and np.abs(m[1:3] - want["metrics"][1:3]).max() <= worst + 2.0 ** -22 * np.abs(want["metrics"][1:3]).max()
    assert abs(m[0] - want["metrics"][0]) <= 2.0 ** -23


def check_grads(b, dH, dW, want, scale, dtype, before=None):
    H, W, dz = np.abs(f64(b["H"])), np.abs(f64(b["W"])), np.abs(want["dz"]) * abs(scale)
    u = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -16
    for got, ref, size in ((f64(dH), want["dH"] * scale, dz @ W), (f64(dW), want["dW"] * scale, dz.T @ H)):
        held = 0.0
        if before is not None and got.shape == want["dW"].shape:
            got, held = got - before, 2.0 ** -23 * np.abs(before)      # the sum's rounding, at the size of what it is added to
        half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -23
        assert (np.abs(got - ref) <= 3 * u * size + half * np.abs(ref) + held).all()
        assert np.linalg.norm(got - ref) <= (6e-3 if dtype == "bf16" else 1e-4) * np.linalg.norm(ref) + np.linalg.norm(held) + 1e-30
    live = want["dz"].any(axis=1)
    assert not dH[torch.from_numpy(~live).cuda()].any()


# ragged rollouts, one without tokens, one in no pair; a rollout in several pairs, an empty place, a rollout against itself
CS = [0, 40, 41, 41, 170, 300, 333]
PAIRS = [(0, 3), (0, 4), (4, 1), (-1, -1), (3, 3), (2, 0), (4, 3)]
KINDS = [dict(kind="logistic"), dict(kind="logistic", smoothing=0.1, margin=0.3, beta=0.05), dict(kind="square", mean=True, beta=1.0),
         dict(kind="hinge", beta=0.01), dict(kind="logistic", mean=True, beta=2.0)]


def pref_cfg(kw):
    return B.pref_cfg_default(kind=KIND[kw["kind"]], mean=int(kw.get("mean", False)), beta=kw.get("beta", 0.1), margin=kw.get("margin", 0.0),
                              label_smoothing=kw.get("smoothing", 0.0))


def exact_kw(kw):
    """The statement's arguments as the fp32 numbers that the call gets."""
    return {k: (float(np.float32(v)) if isinstance(v, float) else v) for k, v in dict(dict(beta=0.1), **kw).items()}


@pytest.mark.parametrize("kw", KINDS, ids=lambda k: "-".join(map(str, k.values())))
@pytest.mark.parametrize("dtype,d,V", [("bf16", 64, 1000), ("bf16", 192, 257), ("fp32", 33, 301), ("fp32", 64, 1)])
@pytest.mark.parametrize("chunk", [None, 128])
def test_loss_and_gradients(ctx, kw, dtype, d, V, chunk):
    b = batch(333, d, V, CS, PAIRS, dtype)
    cfg, pc, kw = cfg_of(dtype), pref_cfg(kw), exact_kw(kw)
    want = oracle(b, **kw)
    got = ctx.pref_fwd(cfg, pc, *args(b), ref_logp=b["ref"])
    check_forward(b, got, want, kw, dtype)
    dH, dW = ctx.pref_bwd(cfg, *args(b)[:4], got["coef"], got["lse"], grad_scale=0.5, chunk_tokens=chunk)
    check_grads(b, dH, dW, want, 0.5, dtype)
    one, dH, dW = ctx.pref_fwd_bwd(cfg, pc, *args(b), ref_logp=b["ref"], grad_scale=-3.0, chunk_tokens=chunk)
    check_forward(b, one, want, kw, dtype)
    check_grads(b, dH, dW, want, -3.0, dtype)
    if dtype == "bf16":
        _, dH2, dW2 = ctx.pref_fwd_bwd(cfg, pc, *args(b), ref_logp=b["ref"], grad_scale=-3.0, chunk_tokens=chunk, dw_dtype=torch.bfloat16)
        check_grads(b, dH2, dW2, want, -3.0, dtype)
    base = torch.randn(V, d, device="cuda")
    acc = base.clone()
    ctx.pref_fwd_bwd(cfg, pc, *args(b), ref_logp=b["ref"], dW=acc, accumulate_dW=True, chunk_tokens=chunk)
    check_grads(b, dH / -3.0 if dtype == "fp32" else dH.float() / -3.0, acc, want, 1.0, dtype, before=f64(base))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_weights_and_no_reference(ctx, dtype):
    b = batch(333, 64, 500, CS, PAIRS, dtype, seed=2)
    b["weight"] = torch.tensor([0.5, -1.0, 0.0, 3.0, 2.0, 0.25, 1.0], device="cuda")
    b["ref"].zero_()
    want = oracle(b, weight=f64(b["weight"]), beta=float(np.float32(0.1)))
    got, dH, dW = ctx.pref_fwd_bwd(cfg_of(dtype), B.pref_cfg_default(), *args(b), pair_weight=b["weight"])
    check_forward(b, got, want, dict(beta=float(np.float32(0.1))), dtype)
    check_grads(b, dH, dW, want, 1.0, dtype)


@pytest.mark.parametrize("T,R,V,d,P", [(1, 1, 300, 64, 1), (2, 2, 5, 64, 1), (200, 3000, 300, 64, 40), (129, 2, 2000, 128, 1), (700, 700, 300, 64, 1500), (513, 3, 700, 2112, 2)])
def test_shapes(ctx, T, R, V, d, P):
    g = np.random.default_rng(T)
    cs = np.concatenate([[0], np.sort(g.integers(0, T + 1, R - 1)), [T]]).tolist()
    b = batch(T, d, V, cs, g.integers(0, R, (P, 2)).tolist(), "bf16", seed=T)
    kw = dict(beta=float(np.float32(0.1)))
    want = oracle(b, **kw)
    got, dH, dW = ctx.pref_fwd_bwd(cfg_of("bf16"), B.pref_cfg_default(), *args(b), ref_logp=b["ref"])
    check_forward(b, got, want, kw, "bf16")
    if np.abs(want["coef"]).max() > 1e-6:
        check_grads(b, dH, dW, want, 1.0, "bf16")


@pytest.mark.parametrize("dw", [torch.bfloat16, torch.float32])
def test_workspaces_of_exactly_the_size_asked_for(ctx, dw):
    """One chunk, several chunks: the call takes what its size function says (a bf16 dW of several chunks needs V d floats more)."""
    T, d, V, R = 300, 256, 20000, 4
    b = batch(T, d, V, [0, 80, 150, 230, 300], [(0, 1), (2, 3)], "bf16", seed=3)
    cfg, pc = cfg_of("bf16"), B.pref_cfg_default()
    want = oracle(b, beta=float(np.float32(0.1)))
    for chunk in (128, 256, 384, 1 << 20):
        out, dH, dW = ctx.pref_fwd_bwd(cfg, pc, *args(b), ref_logp=b["ref"], dw_dtype=dw, chunk_tokens=chunk)
        check_grads(b, dH, dW, want, 1.0, "bf16")
        dH, dW = ctx.pref_bwd(cfg, *args(b)[:4], out["coef"], out["lse"], dw_dtype=dw, chunk_tokens=chunk)
        check_grads(b, dH, dW, want, 1.0, "bf16")


def test_nothing_to_do(ctx):
    """No tokens, no pairs, no rollouts: a loss of its own, gradients of zero."""
    empty = torch.zeros(0, 2, dtype=torch.int32, device="cuda")
    for dtype in ("bf16", "fp32"):
        cfg = cfg_of(dtype)
        b = batch(100, 64, 300, [0, 50, 100], [(0, 1)], dtype)
        for case in (dict(b, pairs=empty), dict(b, cs=torch.zeros(3, dtype=torch.int64, device="cuda")),
                     dict(b, y=torch.full_like(b["y"], -1)), dict(b, cs=torch.zeros(1, dtype=torch.int64, device="cuda"), pairs=empty),
                     dict(b, H=b["H"][:0], y=b["y"][:0], cs=torch.zeros(3, dtype=torch.int64, device="cuda"), ref=b["ref"][:0])):
            got, dH, dW = ctx.pref_fwd_bwd(cfg, B.pref_cfg_default(), *args(case), ref_logp=case["ref"])
            n = len(case["pairs"])
            assert abs(got["loss"].item() - (np.log(2) if n else 0)) < 1e-7 and got["metrics"][3].item() == n
            assert not dH.any() and not dW.any() and not got["logp"].any() and not got["ratio"].any()
            two = ctx.pref_fwd(cfg, B.pref_cfg_default(), *args(case), ref_logp=case["ref"])
            dH, dW = ctx.pref_bwd(cfg, *args(case)[:4], two["coef"], two["lse"])
            assert not dH.any() and not dW.any() and torch.equal(two["loss"], got["loss"])


def test_bad_inputs_are_reported(ctx):
    own = B.Context(0)
    cfg, pc = cfg_of("bf16"), B.pref_cfg_default()
    b = batch(100, 64, 300, [0, 30, 60, 100], [(0, 1), (1, 2)], "bf16")
    want = own.pref_fwd(cfg, pc, *args(b), ref_logp=b["ref"])
    bad = dict(b, pairs=torch.tensor([[0, 1], [3, 0], [1, 2], [0, -1], [-7, 2], [2 ** 31 - 1, 0]], dtype=torch.int32, device="cuda"))
    got = own.pref_fwd(cfg, pc, *args(bad), ref_logp=b["ref"])
    assert own.last_status() == B.AERO_ST_BAD_PAIR
    assert torch.equal(got["loss"], want["loss"]) and torch.equal(got["coef"], want["coef"])
    y = b["y"].clone()
    y[:5] = torch.tensor([300, -1, 2 ** 31 - 1, -2, 0])
    same = y.clone()
    same[[0, 2, 3]] = -1
    want = own.pref_fwd(cfg, pc, *args(dict(b, y=same)), ref_logp=b["ref"])
    assert own.last_status() == 0
    got = own.pref_fwd(cfg, pc, *args(dict(b, y=y)), ref_logp=b["ref"])
    assert own.last_status() == B.AERO_ST_BAD_TARGET
    assert all(torch.equal(got[k], want[k]) for k in NAMES)
    own.pref_fwd_bwd(cfg, pc, *args(dict(b, cs=torch.tensor([0, 30, 60, 101], dtype=torch.int64, device="cuda"))), ref_logp=b["ref"])
    assert own.last_status() & B.AERO_ST_BAD_OFFSETS
    over = torch.tensor([0, 100, 0, 100, 0, 100], dtype=torch.int64, device="cuda")          # 0 .. 100 three times
    out, dH, _ = own.pref_fwd_bwd(cfg, pc, *args(dict(b, cs=over, pairs=torch.tensor([[0, 2], [4, 0]], dtype=torch.int32, device="cuda"))))
    assert own.last_status() & B.AERO_ST_BAD_OFFSETS and abs(out["loss"].item() - np.log(2)) < 1e-7 and not dH.any()
    own.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_row_that_is_no_number(ctx, dtype):
    """NaN in a row reaches its pairs and the loss; in rollouts of no pair and behind the last one nothing is read."""
    b = batch(120, 64, 300, [0, 30, 60, 90, 100], [(0, 1)], dtype)
    want = ctx.pref_fwd_bwd(cfg_of(dtype), B.pref_cfg_default(), *args(b), ref_logp=b["ref"])
    b["H"][60:], b["ref"][60:] = float("nan"), float("nan")
    got = ctx.pref_fwd_bwd(cfg_of(dtype), B.pref_cfg_default(), *args(b), ref_logp=b["ref"])
    assert all(torch.equal(got[0][k], want[0][k]) for k in NAMES) and torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])
    b["y"][7] = 5
    b["H"][7] = float("nan")
    out, dH, _ = ctx.pref_fwd_bwd(cfg_of(dtype), B.pref_cfg_default(), *args(b), ref_logp=b["ref"])
    assert torch.isnan(out["loss"]).all() and torch.isnan(out["margin"]).all() and torch.isnan(out["logp"][7])
    assert torch.isfinite(out["logp"][:7]).all() and torch.isnan(dH[7]).any()


def test_same_bits_captured_and_replayed_on_another_stream(ctx):
    b = batch(333, 128, 1000, CS, PAIRS, "bf16", seed=5)
    cfg, pc = cfg_of("bf16"), B.pref_cfg_default()
    first = ctx.pref_fwd_bwd(cfg, pc, *args(b), ref_logp=b["ref"])
    again = ctx.pref_fwd_bwd(cfg, pc, *args(b), ref_logp=b["ref"])
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    own = B.Context(0, stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out, dH, dW = own.pref_fwd_bwd(cfg, pc, *args(b), ref_logp=b["ref"])
        fwd = own.pref_fwd(cfg, pc, *args(b), ref_logp=b["ref"])
        dH2, dW2 = own.pref_bwd(cfg, *args(b)[:4], fwd["coef"], fwd["lse"])
    for _ in range(2):
        for t in (dH, dW, dH2, dW2):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
    for o, h, w in (again, (out, dH, dW)):
        assert all(torch.equal(o[k], first[0][k]) for k in NAMES) and torch.equal(h, first[1]) and torch.equal(w, first[2])
    two = ctx.pref_fwd(cfg, pc, *args(b), ref_logp=b["ref"])
    want = ctx.pref_bwd(cfg, *args(b)[:4], two["coef"], two["lse"])
    assert torch.equal(fwd["coef"], two["coef"]) and torch.equal(dH2, want[0]) and torch.equal(dW2, want[1])
    del graph
    own.close()


@pytest.mark.parametrize("d,V", [(1536, 20000), (3584, 20000)])
def test_sums_over_long_rollouts(ctx, d, V):
    """The mean error of the log-probs of a long rollout.  Cut off towards zero, the d / 16 additions of a logit of these inputs lose 1.5e-8
    of it each on average, which moves every log-prob the same way: by d / 16 1.55e-8 times the variance of the logits, 0.0004 d, which is
    9e-7 and 5e-6.  With that taken back what is left is a quarter of it at most (the mean over a logit's partial sums, a constant of
    the inputs' distribution, against the measured one) and the mean of 1000 roundings of 4e-6 at most: 2e-7."""
    T = 1000
    g = torch.Generator(device="cuda").manual_seed(7)
    W = (torch.randn(V, d, generator=g, device="cuda") * 0.02).bfloat16()
    H = torch.randn(T, d, generator=g, device="cuda").bfloat16()
    y = torch.randint(0, V, (T,), generator=g, device="cuda").int()
    z = H.double() @ W.double().T
    want = torch.log_softmax(z, 1).gather(1, y.long()[:, None])[:, 0]
    cs = torch.tensor([0, T, T], device="cuda")
    out = ctx.pref_fwd(cfg_of("bf16"), B.pref_cfg_default(), H, W, y, cs, torch.tensor([[0, 1]], dtype=torch.int32, device="cuda"))
    cut = d / 16 * 1.55e-8 * 0.0004 * d
    assert abs((out["logp"].double() - want).mean().item()) <= 0.25 * cut + 2e-7
    assert abs(out["ratio"][0].item() - want.sum().item()) <= T * (0.25 * cut + 2e-7) + 2.0 ** -24 * want.sum().abs().item()


def test_a_preference_step_together(ctx):
    """A frozen reference scored in 4 bits, the final norm, the loss on pairs, and the step that applies its gradients: run as one
    program, each part against its own statement on what the part before it gave."""
    T, d, V = 333, 128, 1000
    cfg = cfg_of("bf16")
    b = batch(T, d, V, CS, PAIRS, "bf16", seed=11)
    gamma = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    ref_w = ctx.quantize_fp4(cfg, b["W"])
    state = dict(param=b["W"], master=b["W"].float(), m=torch.zeros(V * d, dtype=torch.float8_e4m3fn, device="cuda"),
                 v=torch.zeros(V * d, dtype=torch.uint8, device="cuda"), m_scale=torch.zeros(V * d // 256, device="cuda"),
                 v_scale=torch.zeros(V * d // 256, device="cuda"), weight_decay=0.1)
    small = dict(param=gamma, master=gamma.float(), m=torch.zeros(d, device="cuda"), v=torch.zeros(d, device="cuda"))
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    losses = []
    for k in range(2):
        n = ctx.rmsnorm_fwd(cfg, b["H"], gamma)
        z = ctx.lmhead_fp4(ctx.quantize_fp4(cfg, n["h"]), ref_w, out_dtype=torch.float32)
        ref = torch.log_softmax(z, 1).gather(1, b["y"].long().clamp(min=0)[:, None])[:, 0].contiguous()
        now = dict(b, H=n["h"], ref=ref)
        want = oracle(now, beta=float(np.float32(0.1)))
        out, dH, dW = ctx.pref_fwd_bwd(cfg, B.pref_cfg_default(), *args(now), ref_logp=ref, dw_dtype=torch.bfloat16)
        check_forward(now, out, want, dict(beta=float(np.float32(0.1))), "bf16")
        check_grads(now, dH, dW, want, 1.0, "bf16")
        dx, dgamma = ctx.rmsnorm_bwd(cfg, dH, b["H"], gamma, n["rstd"])
        before = f64(state["master"])
        plan = B.AdamWPlan([dict(state, grad=dW), dict(small, grad=dgamma)])
        stats = ctx.adamw_step(B.adamw_cfg_default(lr=1e-3, max_norm=1.0), plan, step)
        norm = M.grad_norm([f64(dW), f64(dgamma)])
        assert abs(stats[0].item() - norm) <= 2.0 ** -20 * norm and step.item() == k + 1
        assert np.abs(f64(state["master"]) - before).max() <= 4e-3 and torch.isfinite(dx).all()
        assert torch.equal(state["param"], state["master"].bfloat16())
        losses.append(out["loss"].item())
    assert np.isfinite(losses).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("smoothing", [0.0, 0.25, 1.0])
def test_infinite_margins(ctx, dtype, sign, smoothing):
    """A reference that gives a token no probability at all makes its rollout's log ratio infinite.  A part of the loss whose factor is 0
    (the second one without smoothing, the first with smoothing 1) adds nothing then either; coef is the slope's limit."""
    b = batch(60, 64, 300, [0, 20, 40, 60], [(0, 1), (1, 2)], dtype, seed=8)
    b["y"][3] = 7
    b["ref"][3] = -float("inf")
    if sign < 0:
        b["pairs"] = b["pairs"].flip(1).contiguous()
    pc = B.pref_cfg_default(label_smoothing=smoothing)
    out, dH, dW = ctx.pref_fwd_bwd(cfg_of(dtype), pc, *args(b), ref_logp=b["ref"])
    two = ctx.pref_fwd(cfg_of(dtype), pc, *args(b), ref_logp=b["ref"])
    other = out["margin"][1].double().cpu().numpy()
    each, slope = M.pref_pair("logistic", other, smoothing)
    weight = smoothing if sign > 0 else 1 - smoothing                                 # of the part that is infinite
    loss = 0.5 * each if weight == 0 else float("inf")
    beta = float(np.float32(0.1))
    for got in (out, two):
        assert got["margin"][0].item() == sign * float("inf")
        assert got["loss"].item() == loss or abs(got["loss"].item() - loss) <= 2.0 ** -22 * abs(loss)
        first = 0.5 * beta * (smoothing if sign > 0 else smoothing - 1)               # d loss / d r_chosen of the pair
        want = np.array([first, 0.5 * beta * slope - first, -0.5 * beta * slope]) if sign > 0 else \
            np.array([-first, first - 0.5 * beta * slope, 0.5 * beta * slope])
        assert np.abs(f64(got["coef"]) - want).max() <= 2.0 ** -22
    assert torch.isfinite(dH.float()).all() and torch.isfinite(dW).all()


CUTS = ["early", "late", "blocks", "sparse", "whole", "tiny"]


@pytest.mark.parametrize("d", [1536, 3584])
@pytest.mark.parametrize("kind", CUTS)
def test_sums_of_other_inputs(ctx, kind, d):
    """The mean error of log-probs where the products are not alike along d: large ones at its start or end, most columns of H zero
    (one in 16, or 16 in 128) or of 1e-9 of the others, whole numbers, of which nothing is cut off.  A correction may leave a
    quarter of what the additions lose of dense inputs (test_sums_over_long_rollouts) where they lose as much, and nowhere more than
    without it; 2e-7 for the mean of 500 roundings of 4e-6 at most."""
    T, V = 500, 20000
    g = torch.Generator(device="cuda").manual_seed(d)
    W = torch.randn(V, d, generator=g, device="cuda") * (1.43 / d) ** 0.5
    H = torch.randn(T, d, generator=g, device="cuda")
    k = torch.arange(d, device="cuda")
    if kind == "whole":
        W, H = (torch.randint(-3, 4, (n, d), generator=g, device="cuda").float() / s for n, s in ((V, 128), (T, 1)))
    else:
        H *= dict(early=(k < 64) * 30.0 + 1, late=(k >= d - 64) * 30.0 + 1, blocks=(k % 128 < 16).float(), sparse=(k % 16 == 0).float(),
                  tiny=torch.where(k % 128 < 16, 1.0, 1e-9))[kind]
        H *= d ** 0.5 / H.norm(dim=1, keepdim=True)
    W, H = W.bfloat16(), H.bfloat16()
    y = torch.randint(0, V, (T,), generator=g, device="cuda").int()
    z = H.double() @ W.double().T
    want = torch.logsumexp(z, 1)
    mean_z = (torch.softmax(z, 1) * z).sum(1).mean().item()
    one = torch.ones(1, device="cuda")
    plain = ctx.distill_fwd(cfg_of("bf16"), H, W, y[:, None].contiguous(), torch.zeros(T, 1, device="cuda"), torch.tensor([0, T], device="cuda"),
                            one, one.to(torch.uint8))["lse"]
    out = ctx.pref_fwd(cfg_of("bf16"), B.pref_cfg_default(), H, W, y, torch.tensor([0, T, T], device="cuda"),
                       torch.tensor([[0, 1]], dtype=torch.int32, device="cuda"))
    off, without = ((x.double() - want).mean().item() for x in (out["lse"], plain))
    dense = 0.25 * d / 16 * 1.55e-8 * mean_z if kind in ("early", "late") else abs(without)
    assert abs(off) <= dense + 2e-7, (off, without)


def test_a_policy_against_itself(ctx):
    """Log-probs of the same weights as reference: margins of zero where they come from this loss's own forward; from aero_logprob_fwd,
    whose logits keep what the tensor cores' additions cut off, margins of no more than both calls' errors in the log-probs."""
    T, d, V = 700, 1536, 5000
    cs = [0, 300, 310, 500, 700]
    b = batch(T, d, V, cs, [(0, 1), (2, 3), (3, 1)], "bf16", seed=12)
    cfg, pc = cfg_of("bf16"), B.pref_cfg_default()
    first = ctx.pref_fwd(cfg, pc, *args(b))
    again = ctx.pref_fwd(cfg, pc, *args(b), ref_logp=first["logp"])
    assert not again["margin"].any() and not again["ratio"].any() and abs(again["loss"].item() - np.log(2)) < 1e-7
    S = float((b["H"].float().abs() @ b["W"].float().abs().T).max())
    tol = (d / 16 + 2) * 2.0 ** -23 * S + (V / 32 + 64) * 2.0 ** -24 + 2.0 ** -23 * first["logp"].abs().max().item()
    n = np.array([(b["y"][x:z] >= 0).sum().item() for x, z in zip(cs, cs[1:])])
    one, dH, dW = ctx.pref_fwd_bwd(cfg, pc, *args(b), ref_logp=first["logp"])
    assert (np.abs(f64(one["ratio"])) <= 2 * n * tol).all()
    other = ctx.logprob_fwd(cfg, b["H"], b["W"], b["y"].clamp(min=0))["logp"]
    got = ctx.pref_fwd(cfg, pc, *args(b), ref_logp=other)
    assert (np.abs(f64(got["ratio"])) <= 2 * n * tol).all()

"""GPU tests of the AdamW step (aero_adamw_step, aero_adamw_states) against the fp64 statement, applied to the state that the
device held before each step.

Tolerances.  u = 2^-24.  m is two products and a sum of values that carry the clipped gradient's two roundings: at most 5 u of
|beta1 m| + |(1 - beta1) g'|.  v has one more product of those: 8 u of its (positive) terms.  The step divides m c1 by
sqrt(v c2) + eps: m's 5, the rate's 3, half of v's 8, the root, the sum and the quotient: below 16 u of the step, but where m's two
terms cancel 16 u of what they would make; p adds three roundings of itself.  An output in bf16 is off by 2^-8 of itself besides.
8-bit states: a code is the nearest value of its table to the state over the block's scale, where the quotient carries 4 u (and
the root of v 5): compared through its distance to the nearest value, with 2^-20 of the value to spare."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import pref_step as M
from paper_2602_14338_b200 import binding as B

pytestmark = pytest.mark.gpu

U, HALF16 = 2.0 ** -24, 2.0 ** -8
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(0)
    yield c
    assert c.last_status() == 0
    c.close()


def f64(t):
    return t.double().cpu().numpy()


def shifted(n, dtype, shift):
    return torch.zeros(n + shift, dtype=dtype, device="cuda")[shift:]


def make(sizes, param, grad, bits, master, seed, shift=0):
    g = torch.Generator().manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        t = dict(param=shifted(n, DT[param], shift), grad=shifted(n, DT[grad], shift), weight_decay=0.1 * (i % 2), lr_scale=1.0 + i % 3)
        p = torch.randn(n, generator=g) * 0.1
        t["param"].copy_(p)
        if master:
            t["master"] = shifted(n, torch.float32, shift)
            t["master"].copy_(p)
        t["grad"].copy_(torch.randn(n, generator=g) * 10.0 ** torch.randint(-4, 2, (n,), generator=g))
        if bits == 32:
            t["m"], t["v"] = shifted(n, torch.float32, shift), shifted(n, torch.float32, shift)
        else:
            t["m"], t["v"] = shifted(n, torch.float8_e4m3fn, shift), shifted(n, torch.uint8, shift)
            t["m_scale"], t["v_scale"] = (torch.zeros((n + 255) // 256, device="cuda") for _ in range(2))
        out.append(t)
    return out


def states(t):
    """m and v of one tensor in 64 bits, decoded here."""
    if t["m"].dtype == torch.float32:
        return f64(t["m"]), f64(t["v"])
    n = t["m"].numel()
    ms, vs = (np.repeat(f64(t[k]), 256)[:n] for k in ("m_scale", "v_scale"))
    return f64(t["m"]) * ms, (M.E4M4[t["v"].cpu().numpy()] * vs) ** 2


def check_codes(t, m, v):
    """The stored states of tensor t against the fp64 ones m, v."""
    n = len(m)
    ms, vs = M.state_scales(m, v)
    assert np.all(np.abs(f64(t["m_scale"]) - ms) <= 8 * U * ms) and np.all(np.abs(f64(t["v_scale"]) - vs) <= 8 * U * vs)
    y = m / np.repeat(ms, 256)[:n]
    off = np.abs(f64(t["m"]) - y)
    assert np.all(off <= M.nearest(np.abs(y), M.E4M3) + 2.0 ** -20 * np.abs(y))
    r = np.sqrt(v) / np.repeat(vs, 256)[:n]
    code = t["v"].cpu().numpy()
    off = np.abs(M.E4M4[code] - r)
    small = r < M.E4M4[1]                                            # not zero: code 1
    assert np.all((off <= M.nearest(r, M.E4M4) + 2.0 ** -20 * r) | (small & (code == 1)))
    assert np.all(code[(r > 0)] > 0) and np.all(code[r == 0] == 0)


def step_and_check(ctx, tensors, step, **kw):
    ac = B.adamw_cfg_default(**kw)
    before = [(f64(t["master"] if "master" in t else t["param"]), *states(t)) for t in tensors]
    t_before = int(step.item())
    stats = ctx.adamw_step(ac, B.AdamWPlan(tensors), step).cpu().numpy()
    norm = M.grad_norm([f64(t["grad"]) for t in tensors], ac.grad_scale)
    clip = M.clip_of(norm, ac.max_norm)
    if ac.max_norm > 0 or ac.skip_nonfinite:
        assert abs(stats[0] - norm) <= 2.0 ** -20 * norm
    assert abs(stats[1] - clip) <= 2.0 ** -20 and stats[2] == 0 and stats[3] == t_before + 1 == step.item()
    for t, (p, m, v) in zip(tensors, before):
        lr = np.float64(np.float32(ac.lr)) * t["lr_scale"]
        wd = np.float64(np.float32(t["weight_decay"]))
        eps = np.float64(np.float32(ac.eps))
        factor = clip * np.float64(np.float32(ac.grad_scale))
        p1, m1, v1 = M.adamw(p, f64(t["grad"]), m, v, t_before + 1, lr, ac.beta1, ac.beta2, eps, wd, factor)
        g = np.abs(f64(t["grad"]) * factor)
        terms = ac.beta1 * np.abs(m) + (1 - ac.beta1) * g
        root = np.sqrt(v1 / (1 - ac.beta2 ** (t_before + 1))) + eps
        size = lr * terms / (1 - ac.beta1 ** (t_before + 1)) / np.where(root > 0, root, 1)
        tol = 16 * U * size + 3 * U * (np.abs(p) + size)
        got = f64(t["master"] if "master" in t else t["param"])
        off = np.abs(got - p1)
        if t["param"].dtype == torch.bfloat16 and "master" not in t:
            tol = tol + HALF16 * np.abs(p1) + tol
        assert np.all(off <= tol), (off / np.maximum(tol, 1e-300)).max()
        if "master" in t:
            assert torch.equal(t["param"], t["master"].bfloat16())
        if t["m"].dtype == torch.float32:
            assert np.all(np.abs(f64(t["m"]) - m1) <= 5 * U * terms + 2.0 ** -149)
            assert np.all(np.abs(f64(t["v"]) - v1) <= 8 * U * v1 + 2.0 ** -149)
        else:
            check_codes(t, m1, v1)


SIZES = [[1], [255, 256, 257], [5000, 3, 1536, 2048], [0, 7, 0, 70000, 0]]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param,master,grad", [("fp32", False, "fp32"), ("bf16", True, "bf16"), ("bf16", False, "fp32"),
                                               ("fp32", False, "bf16")])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("shift", [0, 1])
def test_steps(ctx, bits, param, master, grad, sizes, shift):
    tensors = make(sizes, param, grad, bits, master, 1, shift)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    g = torch.Generator().manual_seed(9)
    for k in range(3):
        step_and_check(ctx, tensors, step, lr=1e-2, beta2=0.99, max_norm=(0.0, 1.0, 1e9)[k], grad_scale=(1.0, 0.25, -2.0)[k])
        for t in tensors:
            t["grad"].copy_(torch.randn(t["grad"].numel(), generator=g))


def test_more_tensors_than_a_launch_takes(ctx):
    tensors = make([1 + 37 * i % 900 for i in range(300)], "bf16", "bf16", 8, True, 2)
    step = torch.full((1,), 1000, dtype=torch.int64, device="cuda")
    step_and_check(ctx, tensors, step, lr=1e-3, max_norm=0.5)
    step_and_check(ctx, tensors, step, lr=1e-3, max_norm=0.5)


def test_no_tensor(ctx):
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    stats = ctx.adamw_step(B.adamw_cfg_default(max_norm=1.0), B.AdamWPlan([]), step)
    assert stats.tolist() == [0.0, 1.0, 0.0, 1.0] and step.item() == 1


@pytest.mark.parametrize("size", [1e-25, 1e-42, 1e25])
def test_norm_of_tiny_and_huge_gradients(ctx, size):
    tensors = make([3000, 5], "fp32", "fp32", 32, False, 3)
    for t in tensors:
        t["grad"].copy_(torch.randn(t["grad"].numel(), generator=torch.Generator().manual_seed(4)).double() * size)
    norm = M.grad_norm([f64(t["grad"]) for t in tensors])
    stats = ctx.adamw_step(B.adamw_cfg_default(max_norm=1.0), B.AdamWPlan(tensors), torch.zeros(1, dtype=torch.int64, device="cuda"))
    assert abs(stats[0].item() - norm) <= 2.0 ** -20 * norm + 2.0 ** -149


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_nonfinite_gradient(ctx, bits, bad):
    tensors = make([600, 40], "bf16", "fp32", bits, True, 5)
    step = torch.full((1,), 7, dtype=torch.int64, device="cuda")
    step_and_check(ctx, tensors, step, lr=1e-3)
    tensors[0]["grad"][300] = bad
    plan = B.AdamWPlan(tensors)
    held = [{k: x.clone() for k, x in t.items() if torch.is_tensor(x)} for t in tensors]
    stats = ctx.adamw_step(B.adamw_cfg_default(skip_nonfinite=1), plan, step)
    assert stats[2].item() == 1 and step.item() == 8
    for t, h in zip(tensors, held):
        for k, x in h.items():
            assert torch.equal(t[k].view(torch.uint8), x.view(torch.uint8)), k
    stats = ctx.adamw_step(B.adamw_cfg_default(), plan, step)
    assert stats[2].item() == 0 and step.item() == 9
    assert not torch.isfinite(tensors[0]["master"][300]) and torch.isfinite(tensors[1]["master"]).all()
    m, v = ctx.adamw_states(plan, out_dtype=torch.float32)
    nan = torch.zeros(600, dtype=torch.bool, device="cuda")
    nan[300] = True
    if bits == 8:
        nan[256:512] = True                                        # the whole block
        assert torch.equal(torch.isnan(m[0]), nan) and torch.equal(torch.isnan(v[0]), nan)
    else:
        assert torch.equal(~torch.isfinite(m[0]), nan) and torch.equal(~torch.isfinite(v[0]), nan)
    assert torch.isfinite(m[1]).all() and torch.isfinite(v[1]).all()


def test_norm_that_is_no_number_without_skip(ctx):
    """max_norm with an infinite norm and no skip: the clip is 0 and an infinite gradient becomes NaN, nothing faults."""
    tensors = make([10], "fp32", "fp32", 32, False, 6)
    tensors[0]["grad"][3] = float("inf")
    stats = ctx.adamw_step(B.adamw_cfg_default(max_norm=1.0), B.AdamWPlan(tensors), torch.zeros(1, dtype=torch.int64, device="cuda"))
    assert stats[0].item() == float("inf") and stats[1].item() == 0
    assert torch.isnan(tensors[0]["param"]).sum().item() == 1


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shift", [0, 3])
def test_states_as_numbers(ctx, bits, out, shift):
    tensors = make([700, 0, 256, 1], "fp32", "fp32", bits, False, 8, shift)
    ctx.adamw_step(B.adamw_cfg_default(), B.AdamWPlan(tensors), torch.zeros(1, dtype=torch.int64, device="cuda"))
    plan = B.AdamWPlan(tensors)
    ms, vs = ctx.adamw_states(plan, out_dtype=out)
    half = HALF16 if out == torch.bfloat16 else U
    for t, m, v in zip(tensors, ms, vs):
        em, ev = states(t)
        assert np.all(np.abs(f64(m) - em) <= (half + 2 * U) * np.abs(em))
        assert np.all(np.abs(f64(v) - ev) <= (half + 4 * U) * ev + 2.0 ** -149)
    only = (C.c_void_p * 4)(*[x.data_ptr() for x in vs])             # one of the two alone
    want = [v.clone() for v in vs]
    for v in vs:
        v.zero_()
    assert ctx.lib.aero_adamw_states(ctx.h, 4, plan.array, B.AERO_BF16 if out == torch.bfloat16 else B.AERO_FP32, None, only) == 0
    assert all(torch.equal(a, b) for a, b in zip(vs, want))


def test_captured_and_replayed(ctx):
    """The step counts on and the learning rate is read anew when a captured call is replayed."""
    run, ref = make([5000, 300], "bf16", "fp32", 8, True, 11), make([5000, 300], "bf16", "fp32", 8, True, 11)
    steps = [torch.zeros(1, dtype=torch.int64, device="cuda") for _ in range(2)]
    lr = torch.tensor([1e-2], device="cuda")
    ac = B.adamw_cfg_default(max_norm=1.0)
    plan = B.AdamWPlan(run)
    stream = torch.cuda.Stream()
    own = B.Context(0, stream)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        stats = own.adamw_step(ac, plan, steps[0], lr=lr)
    for k in range(3):
        lr.fill_(1e-2 / (k + 1))
        graph.replay()
        torch.cuda.synchronize()
        want = ctx.adamw_step(B.adamw_cfg_default(max_norm=1.0, lr=lr.item()), B.AdamWPlan(ref), steps[1])
        assert torch.equal(stats, want) and steps[0].item() == steps[1].item() == k + 1
        for a, b in zip(run, ref):
            for name in ("param", "master", "m", "v", "m_scale", "v_scale"):
                assert torch.equal(a[name].view(torch.uint8), b[name].view(torch.uint8)), name
    del graph
    own.close()


def test_beyond_32_bit_offsets(ctx):
    n = 2 ** 31 + 300
    t = dict(param=torch.zeros(n, dtype=torch.bfloat16, device="cuda"), grad=torch.zeros(n, dtype=torch.bfloat16, device="cuda"),
             m=torch.zeros(n, dtype=torch.float8_e4m3fn, device="cuda"), v=torch.zeros(n, dtype=torch.uint8, device="cuda"))
    t["m_scale"], t["v_scale"] = (torch.zeros((n + 255) // 256, device="cuda") for _ in range(2))
    tail = 5000
    small = {k: x[-tail:].clone() for k, x in t.items() if "scale" not in k}
    small["param"].normal_()
    small["grad"].normal_()
    t["param"][-tail:], t["grad"][-tail:] = small["param"], small["grad"]
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    stats = ctx.adamw_step(B.adamw_cfg_default(max_norm=1.0, lr=0.1), B.AdamWPlan([t]), step).cpu().numpy()
    norm = M.grad_norm([f64(small["grad"])])
    assert abs(stats[0] - norm) <= 2.0 ** -20 * norm
    p1, m1, v1 = M.adamw(f64(small["param"]), f64(small["grad"]), 0 * f64(small["param"]), 0 * f64(small["param"]), 1,
                         np.float64(np.float32(0.1)), 0.9, 0.999, np.float64(np.float32(1e-8)), 0.0, M.clip_of(norm, 1.0))
    got = f64(t["param"][-tail:])
    assert np.all(np.abs(got - p1) <= HALF16 * np.abs(p1) + 40 * U * (np.abs(p1) + 0.2))
    assert torch.count_nonzero(t["param"][:2 ** 31 - 8000]).item() == 0
    ms = np.repeat(f64(t["m_scale"]), 256)[n - tail:n]
    assert np.all(np.abs(f64(t["m"][-tail:]) * ms - m1) <= 2.0 ** -4 * np.abs(m1) + 2.0 ** -9 * ms)


def test_roots_over_all_values(ctx):
    """A block's scale is the root of its largest v times 1 / 496, so its bits tell whether the root is the correctly rounded one.  With
    beta2 = 1/2 and no gradient v is half the square of the decoded root, whose scale takes every fifth fp32 pattern of two binades
    and some of every exponent (the values of a block are all within the range of the fast form, or none is)."""
    g = torch.cat([torch.arange(0x3f800000, 0x40800000, 5, dtype=torch.int32).view(torch.float32),
                   torch.arange(1, 0x7f000000, 99991, dtype=torch.int32).view(torch.float32).clamp(max=1e15)]).cuda()
    n = g.numel()
    t = dict(param=torch.zeros(n * 256, dtype=torch.bfloat16, device="cuda"), grad=torch.zeros(n * 256, dtype=torch.bfloat16, device="cuda"),
             m=torch.zeros(n * 256, dtype=torch.float8_e4m3fn, device="cuda"), v=torch.zeros(n * 256, dtype=torch.uint8, device="cuda"),
             m_scale=torch.zeros(n, device="cuda"), v_scale=g.clone())
    t["v"].view(n, 256)[:, 0], t["v"].view(n, 256)[:, 1:] = 176, 160          # 16 2^(11 - 11) = 16, and 8
    ctx.adamw_step(B.adamw_cfg_default(beta2=0.5, lr=0.0), B.AdamWPlan([t]), torch.zeros(1, dtype=torch.int64, device="cuda"))
    v = (16 * g) * (16 * g) * 0.5
    want = torch.sqrt(v).clamp(min=2.0 ** -100) * torch.tensor(1.0 / 496.0, device="cuda")
    assert torch.equal(t["v_scale"], want)


# Chunks are 2048 elements of one tensor; up to 1184 of them in 128 tensors of one kind of states are summed by the step's blocks.
JOINED = {"one": ([1], 2), "limit": ([1184 * 2048], 2), "beyond": ([1184 * 2048 + 1], 3),
          "limit, many": ([9 * 2048] * 127 + [41 * 2048 - 5], 2), "empty ones": ([0, 700, 0, 2049] + [0] * 140, 2),
          "tensors": ([40] * 129, 5)}


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("name", JOINED)
def test_norm_summed_by_the_step(ctx, name, bits):
    """Two or three launches leave the same bits: with skip_nonfinite the step has a launch between norm and step.  The gradients
    are whole numbers below 2^11, so that the sum of their squares is the same in every order."""
    sizes, launches = JOINED[name]
    one, two = make(sizes, "bf16", "fp32", bits, True, 21), make(sizes, "bf16", "fp32", bits, True, 21)
    for a, b in zip(one, two):
        a["grad"].copy_(torch.randint(-1000, 1001, (a["grad"].numel(),), generator=torch.Generator().manual_seed(22)).float())
        b["grad"].copy_(a["grad"])
    steps = [torch.full((1,), 3, dtype=torch.int64, device="cuda") for _ in range(2)]
    for k in range(2):
        n = ctx.launch_count()
        got = ctx.adamw_step(B.adamw_cfg_default(max_norm=0.7, grad_scale=0.25), B.AdamWPlan(one), steps[0])
        assert ctx.launch_count() - n == launches
        want = ctx.adamw_step(B.adamw_cfg_default(max_norm=0.7, grad_scale=0.25, skip_nonfinite=1), B.AdamWPlan(two), steps[1])
        assert torch.equal(got, want) and steps[0].item() == steps[1].item() == 4 + k
    for a, b in zip(one, two):
        for key in a:
            if torch.is_tensor(a[key]):
                assert torch.equal(a[key].view(torch.uint8), b[key].view(torch.uint8)), key


def test_both_kinds_of_states_in_a_small_call(ctx):
    tensors = make([700, 30], "fp32", "fp32", 32, False, 23) + make([900], "bf16", "bf16", 8, True, 24)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    step_and_check(ctx, tensors, step, lr=1e-3, max_norm=0.5)
    step_and_check(ctx, tensors, step, lr=1e-3, max_norm=0.5)


@pytest.mark.parametrize("n", [10, 1184 * 2048 + 1])
def test_nan_gradient_without_skip(ctx, n):
    """A norm that is NaN makes the clip and so every element NaN, in calls of either number of launches."""
    tensors = make([n], "fp32", "fp32", 32, False, 25)
    tensors[0]["grad"][3] = float("nan")
    stats = ctx.adamw_step(B.adamw_cfg_default(max_norm=1.0), B.AdamWPlan(tensors), torch.zeros(1, dtype=torch.int64, device="cuda"))
    assert torch.isnan(stats[:2]).all() and stats[2:].tolist() == [0.0, 1.0]
    assert torch.isnan(tensors[0]["param"]).all()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("behind", [1, 5, 200])
def test_empty_tensors_behind_a_full_launch(ctx, bits, behind):
    """As many tensors as a launch takes, and empty ones behind them: both launches of the call run over the same tensors."""
    sizes = [40] * 128 + [0] * behind
    one, two = make(sizes, "bf16", "fp32", bits, True, 31), make(sizes, "bf16", "fp32", bits, True, 31)
    for a, b in zip(one, two):
        a["grad"].copy_(torch.randint(-1000, 1001, (a["grad"].numel(),), generator=torch.Generator().manual_seed(32)).float())
        b["grad"].copy_(a["grad"])
    steps = [torch.full((1,), 3, dtype=torch.int64, device="cuda") for _ in range(2)]
    n = ctx.launch_count()
    got = ctx.adamw_step(B.adamw_cfg_default(max_norm=0.7), B.AdamWPlan(one), steps[0])
    assert ctx.launch_count() - n == 2
    want = ctx.adamw_step(B.adamw_cfg_default(max_norm=0.7, skip_nonfinite=1), B.AdamWPlan(two), steps[1])
    assert torch.equal(got, want) and steps[0].item() == steps[1].item() == 4
    for a, b in zip(one, two):
        for key in a:
            if torch.is_tensor(a[key]):
                assert torch.equal(a[key].view(torch.uint8), b[key].view(torch.uint8)), key


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("decay", [0.01, 0.1])
def test_weight_decay_at_small_learning_rates(ctx, bits, decay):
    """lr weight_decay of 1e-8 and 1e-7, below what 1 - lr weight_decay can hold in fp32: the mean of many masters still falls by
    it.  A step's rounding of p in [0.5, 1) is 2^-25 at most, to either side as the step's other part (lr times a number that differs
    from element to element) decides: over 100 steps of 2^18 elements its mean has a deviation below 2^-25 10 / 512, 6e-10; the step
    itself is off by 16 u of lr, 1e-10 in all.  What is looked for is 7e-7 and more; 2 % of it is allowed."""
    n, steps, lr = 2 ** 18, 100, float(np.float32(1e-6))
    wd = float(np.float32(decay))
    g = torch.Generator(device="cuda").manual_seed(41)
    t = dict(param=torch.zeros(n, dtype=torch.bfloat16, device="cuda"), grad=torch.zeros(n, device="cuda"), weight_decay=decay,
             master=0.5 + 0.5 * torch.rand(n, generator=g, device="cuda"))
    if bits == 32:
        t["m"], t["v"] = torch.randn(n, generator=g, device="cuda") * 0.1, 0.5 + torch.rand(n, generator=g, device="cuda")
    else:
        t["m"] = (torch.randn(n, generator=g, device="cuda") * 40).to(torch.float8_e4m3fn)
        t["v"] = torch.randint(160, 192, (n,), generator=g, device="cuda").to(torch.uint8)
        t["m_scale"], t["v_scale"] = torch.full((n // 256,), 1 / 400, device="cuda"), torch.full((n // 256,), 1 / 20, device="cuda")
    step = torch.full((1,), 1000, dtype=torch.int64, device="cuda")
    plan, ac = B.AdamWPlan([t]), B.adamw_cfg_default(lr=lr, beta2=0.99)
    eps = float(np.float32(1e-8))
    want = t["master"].double()
    for k in range(1001, 1001 + steps):
        t["grad"].copy_(torch.randn(n, generator=g, device="cuda"))
        if bits == 32:
            m, v = t["m"].double(), t["v"].double()
        else:
            each = lambda s: s.double().repeat_interleave(256)  # noqa: E731
            m = t["m"].double() * each(t["m_scale"])
            v = (torch.from_numpy(M.E4M4).cuda()[t["v"].long()] * each(t["v_scale"])) ** 2
        m = 0.9 * m + (1 - 0.9) * t["grad"].double()
        v = 0.99 * v + (1 - 0.99) * t["grad"].double() ** 2
        want = (1 - lr * wd) * want - lr * (m / (1 - 0.9 ** k)) / ((v / (1 - 0.99 ** k)).sqrt() + eps)
        ctx.adamw_step(ac, plan, step)
    off = (t["master"].double() - want).mean().item()
    assert abs(off) <= 0.02 * steps * lr * wd * 0.75, off / (steps * lr * wd * 0.75)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("decay", [0.0, 0.1])
def test_infinite_parameters_stay(ctx, bits, decay):
    """A parameter of -inf (a logit's bias that masks a token) stays what it is, with decay and without; so does a NaN."""
    tensors = make([600, 1], "fp32", "fp32", bits, False, 42)
    for t in tensors:
        t["weight_decay"] = decay
    tensors[0]["param"][[3, 300]] = torch.tensor([float("-inf"), float("inf")], device="cuda")
    tensors[0]["param"][400] = float("nan")
    tensors[1]["param"][0] = float("-inf")
    ctx.adamw_step(B.adamw_cfg_default(lr=1e-2), B.AdamWPlan(tensors), torch.zeros(1, dtype=torch.int64, device="cuda"))
    p = tensors[0]["param"]
    assert p[3].item() == float("-inf") and p[300].item() == float("inf") and tensors[1]["param"].item() == float("-inf")
    bad = ~torch.isfinite(p)
    assert torch.isnan(p[400]) and bad.sum().item() == 3
    tensors[1]["grad"][0] = float("nan")
    ctx.adamw_step(B.adamw_cfg_default(lr=1e-2), B.AdamWPlan(tensors), torch.ones(1, dtype=torch.int64, device="cuda"))
    assert torch.isnan(tensors[1]["param"][0]) and p[3].item() == float("-inf")


def test_plan_of_overlapping_tensors():
    """Slices that share elements, a gradient that is written or shares elements with what is: refused; neighbours and shared gradients are not."""
    f = lambda n: torch.zeros(n, device="cuda")  # noqa: E731
    base, grads = f(100), f(100)
    t = lambda p, g, m=None, **over: dict(param=p, grad=g, m=m if m is not None else f(p.numel()), v=f(p.numel()), **over)  # noqa: E731
    B.AdamWPlan([t(base[:50], grads[:50]), t(base[50:], grads[:50])])
    for bad in ([t(base[:51], grads[:51]), t(base[50:], grads[50:])],                 # slices with an element in common
                [t(base[:50], base[50:])] + [t(base[99:], grads[:1])],                # a gradient with an element that is a parameter's
                [t(base[:50], base[:50])],                                            # a gradient that is its parameter
                [t(base[:50], grads[:50], m=base[25:75])],                            # a state over the parameter
                [t(base[:50], grads[:50], m=grads[50:]), t(base[50:], grads[50:])]):  # a state that is another tensor's gradient
        with pytest.raises(B.AeroError, match="overlap|twice"):
            B.AdamWPlan(bad)


ROOTS = [(1.9692776203155518, 0.1, 1.4792181253433228), (3.7277493476867676, 0.5, 2.730475902557373)]



@pytest.mark.parametrize("v,beta2,grad", ROOTS)
def test_roots_of_the_special_values(ctx, v, beta2, grad):
    """The two mantissas whose root depends on which of the reciprocal roots within the documented bound the instruction gives
    (tests/test_adamw_roots.py: no other does), at every power of four of the fast form's range: v is (1 - beta2) grad^2 of a first step."""
    powers = torch.arange(-49, 50, device="cuda").double()
    g = (grad * torch.exp2(powers)).float()
    n = g.numel()
    t = dict(param=torch.zeros(n * 256, device="cuda"), grad=g.repeat_interleave(256), m=torch.zeros(n * 256, dtype=torch.float8_e4m3fn, device="cuda"),
             v=torch.zeros(n * 256, dtype=torch.uint8, device="cuda"), m_scale=torch.zeros(n, device="cuda"), v_scale=torch.zeros(n, device="cuda"))
    rest = float(np.float32(1 - beta2))
    values = ((rest * g.double()).float().double() * g.double()).float()
    assert torch.equal(values, (v * torch.exp2(2 * powers)).float())
    ctx.adamw_step(B.adamw_cfg_default(beta2=beta2, lr=0.0), B.AdamWPlan([t]), torch.zeros(1, dtype=torch.int64, device="cuda"))
    root = torch.sqrt(values.double()).float()                        # (53 bits are enough to round the root of 24 once)
    want = root.clamp(min=2.0 ** -100) * torch.tensor(1.0 / 496.0, device="cuda")
    other = torch.nextafter(root, torch.full_like(root, float("inf"))) * torch.tensor(1.0 / 496.0, device="cuda")
    assert torch.all(want != other) and torch.equal(t["v_scale"], want)

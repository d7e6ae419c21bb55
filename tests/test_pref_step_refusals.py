"""Calls of the operators of a preference-training step that are refused, before any device call: the error code of each argument
error.  CPU only.  The context handed to the C calls is a block of zeros, which is all that the argument checks look at; no
call here gets past them."""
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


def adamw_tensor(**over):
    t = dict(n=1000, param=P, grad=P, master=None, m=P, v=P, m_scale=P, v_scale=P, param_dtype=B.AERO_BF16, grad_dtype=B.AERO_FP32,
             state_bits=8, weight_decay=0.0, lr_scale=1.0)
    t.update(over)
    return B.AeroAdamWTensor(**t)


def test_adamw_refusals(lib, fake):
    need = lib.aero_adamw_workspace_bytes(1)
    assert need > 0 and lib.aero_adamw_workspace_bytes(-1) == 0 and lib.aero_adamw_workspace_bytes(0) >= 256

    def step(ctx=fake, ac=None, n=1, t=None, stp=P, ws=P, wsb=need, **over):
        ac = ac if ac is not None else B.adamw_cfg_default()
        t = (B.AeroAdamWTensor * 1)(adamw_tensor(**over)) if t is None else t
        return lib.aero_adamw_step(ctx, C.byref(ac), n, t, stp, None, None, ws, wsb)

    assert step(ctx=None) == INVALID and step(n=-1) == INVALID and step(stp=None) == INVALID and step(ws=None) == INVALID
    assert step(t=C.POINTER(B.AeroAdamWTensor)()) == INVALID
    assert step(ws=P + 16) == INVALID and step(wsb=need - 1) == WORKSPACE
    for name in ("param", "grad", "m", "v", "m_scale", "v_scale"):
        assert step(**{name: None}) == INVALID, name
    for name, off in (("param", 1), ("grad", 2), ("m_scale", 2), ("v_scale", 1)):
        assert step(**{name: P + off}) == INVALID, name
    assert step(state_bits=32, m=P + 2) == INVALID and step(state_bits=32, v=P + 1) == INVALID
    assert step(master=P + 2) == INVALID and step(master=P, param_dtype=B.AERO_FP32) == INVALID
    assert step(n=1, t=(B.AeroAdamWTensor * 1)(adamw_tensor(n=-1))) == INVALID
    assert step(param_dtype=2) == UNSUPPORTED and step(grad_dtype=-1) == UNSUPPORTED and step(state_bits=16) == UNSUPPORTED
    nan = float("nan")
    assert step(weight_decay=-0.1) == INVALID and step(weight_decay=nan) == INVALID and step(lr_scale=-1.0) == INVALID
    for name, bad in (("lr", -1.0), ("lr", nan), ("beta1", 1.0), ("beta1", -0.1), ("beta2", 1.0), ("beta2", nan), ("eps", -1e-8),
                      ("eps", nan), ("max_norm", float("inf")), ("max_norm", nan), ("grad_scale", nan), ("grad_scale", float("inf"))):
        assert step(ac=B.adamw_cfg_default(**{name: bad})) == INVALID, name

    def states(ctx=fake, n=1, out=B.AERO_BF16, m=P, v=P, **over):
        t = (B.AeroAdamWTensor * 1)(adamw_tensor(**over))
        array = lambda p: None if p is None else (C.c_void_p * 1)(p or None)  # noqa: E731
        return lib.aero_adamw_states(ctx, n, t, out, array(m), array(v))

    assert states(ctx=None) == INVALID and states(n=-1) == INVALID and states(out=5) == UNSUPPORTED
    assert states(m=None, v=None) == INVALID and states(m=0) == INVALID and states(m=P + 1) == INVALID
    assert states(v=P + 2, out=B.AERO_FP32) == INVALID and states(m_scale=None) == INVALID and states(state_bits=4) == UNSUPPORTED


def test_fp4_refusals(lib, fake):
    assert lib.aero_fp4_code_bytes(129, 288) == 2 * 2 * 128 * 128 and lib.aero_fp4_scale_bytes(129, 288, 16) == 2 * 2 * 2048
    assert lib.aero_fp4_scale_bytes(1, 32, 32) == 1024 and lib.aero_fp4_scale_bytes(1, 32, 8) == 0
    assert lib.aero_fp4_code_bytes(-1, 32) == 0 and lib.aero_fp4_code_bytes(0, 32) == 0

    def quant(ctx=fake, c=None, T=4, d=64, block=16, x=P, codes=P, scales=P, row=P):
        return lib.aero_quantize_fp4(ctx, c or cfg(), T, d, block, x, codes, scales, row)

    def values(ctx=fake, T=4, d=64, block=16, codes=P, scales=P, row=P, dtype=B.AERO_BF16, out=P):
        return lib.aero_dequantize_fp4(ctx, T, d, block, codes, scales, row, dtype, out)

    def product(ctx=fake, T=4, d=64, V=10, block=16, h=P, hs=P, hr=P, w=P, ws=P, wr=P, dtype=B.AERO_BF16, out=P):
        return lib.aero_lmhead_fp4(ctx, T, d, V, block, h, hs, hr, w, ws, wr, dtype, out)

    for call in (quant, values, product):
        assert call(ctx=None) == INVALID and call(T=-1) == INVALID and call(d=0) == INVALID
        assert call(d=48) == UNSUPPORTED and call(d=65568) == UNSUPPORTED and call(T=(1 << 30) + 1) == UNSUPPORTED
        assert call(block=64) == UNSUPPORTED and call(block=0) == UNSUPPORTED
        assert call(block=32) == INVALID                                    # no row scales there
    for name in ("x", "codes", "scales", "row"):
        assert quant(**{name: None}) == INVALID, name
    for name in ("x", "codes", "scales"):
        assert quant(**{name: P + 8}) == INVALID, name
    assert quant(row=P + 2) == INVALID and quant(c=cfg(5)) == UNSUPPORTED
    for name in ("codes", "scales", "row", "out"):
        assert values(**{name: None}) == INVALID and values(**{name: P + 2}) == INVALID, name
    assert values(dtype=3) == UNSUPPORTED and product(dtype=3) == UNSUPPORTED
    for name in ("h", "hs", "hr", "w", "ws", "wr", "out"):
        assert product(**{name: None}) == INVALID and product(**{name: P + 1}) == INVALID, name
    assert product(V=0) == INVALID and product(V=(1 << 30) + 1) == UNSUPPORTED and product(V=1 << 30, d=1024) == UNSUPPORTED
    assert product(dtype=B.AERO_FP32, out=P + 2) == INVALID


def test_pref_refusals(lib, fake):
    fwd_need = lib.aero_pref_fwd_workspace_bytes(40, 64, 10, 3, 4)
    both_need = lib.aero_pref_fwd_bwd_workspace_bytes(40, 64, 10, 3, 4, 128, B.AERO_FP32)
    bwd_need = lib.aero_pref_bwd_workspace_bytes(40, 64, 10, 3, 128, B.AERO_FP32)
    assert 0 < fwd_need <= both_need and 0 < bwd_need <= both_need
    assert lib.aero_pref_fwd_workspace_bytes(-1, 64, 10, 3, 4) == 0 and lib.aero_pref_fwd_workspace_bytes(40, 64, 10, 3, -1) == 0

    def fwd(ctx=fake, c=None, pc=None, T=40, d=64, V=10, R=3, n=4, H=P, W=P, y=P, ref=P, cs=P, pairs=P, pw=None, logp=P, lse=P, ratio=P,
            margin=P, coef=P, loss=P, ws=P, wsb=fwd_need):
        pc = C.byref(pc if pc is not None else B.pref_cfg_default())
        return lib.aero_pref_fwd(ctx, c or cfg(), pc, T, d, V, R, n, H, W, y, ref, cs, pairs, pw, logp, lse, ratio, margin, coef, loss, None,
                                 ws, wsb)

    def both(ctx=fake, c=None, pc=None, T=40, d=64, V=10, R=3, n=4, H=P, W=P, y=P, ref=P, cs=P, pairs=P, pw=None, logp=P, lse=P, ratio=P,
             margin=P, coef=P, loss=P, dH=P, dW=P, dt=B.AERO_FP32, acc=0, ws=P, wsb=both_need):
        pc = C.byref(pc if pc is not None else B.pref_cfg_default())
        return lib.aero_pref_fwd_bwd(ctx, c or cfg(), pc, T, d, V, R, n, H, W, y, ref, cs, pairs, pw, logp, lse, ratio, margin, coef, loss,
                                     None, 1.0, dH, dW, dt, acc, ws, wsb)

    def bwd(ctx=fake, c=None, T=40, d=64, V=10, R=3, H=P, W=P, y=P, cs=P, coef=P, lse=P, dH=P, dW=P, dt=B.AERO_FP32, acc=0, ws=P,
            wsb=bwd_need):
        return lib.aero_pref_bwd(ctx, c or cfg(), T, d, V, R, H, W, y, cs, coef, lse, 1.0, dH, dW, dt, acc, ws, wsb)

    for call in (fwd, both, bwd):
        for name in ("ctx", "H", "W", "y", "cs", "lse", "coef", "ws"):
            assert call(**{name: None}) == INVALID, name
        assert call(T=-1) == INVALID and call(T=1 << 31) == INVALID and call(d=0) == INVALID and call(V=0) == INVALID and call(R=-1) == INVALID
        assert call(d=65) == UNSUPPORTED and call(c=cfg(9)) == UNSUPPORTED and call(d=1088, c=cfg(B.AERO_FP32)) == UNSUPPORTED
        assert call(H=P + 8) == INVALID and call(W=P + 2) == INVALID and call(ws=P + 16) == INVALID
        assert call(wsb=255) == WORKSPACE
    assert fwd(wsb=fwd_need // 2) == WORKSPACE and both(wsb=both_need // 64) == WORKSPACE and bwd(wsb=bwd_need // 64) == WORKSPACE
    for call in (fwd, both):
        for name in ("pairs", "logp", "ratio", "margin", "loss"):
            assert call(**{name: None}) == INVALID, name
        assert call(n=-1) == INVALID and call(pairs=P + 4) == INVALID and call(pc=B.pref_cfg_default(kind=3)) == UNSUPPORTED
        for name, bad in (("beta", float("nan")), ("beta", float("inf")), ("margin", float("nan")), ("label_smoothing", -0.1),
                          ("label_smoothing", 1.1), ("label_smoothing", float("nan"))):
            assert call(pc=B.pref_cfg_default(**{name: bad})) == INVALID, name
    for call in (both, bwd):
        assert call(dH=None) == INVALID and call(dW=None) == INVALID and call(dH=P + 8) == INVALID and call(dW=P + 4) == INVALID
        assert call(dt=4) == UNSUPPORTED and call(dt=B.AERO_BF16, acc=1) == INVALID
        assert call(dt=B.AERO_BF16, c=cfg(B.AERO_FP32)) == UNSUPPORTED


@pytest.mark.parametrize("rows,cols", [(0, 32), (1, 32), (128, 256), (129, 288), (1000, 65536)])
@pytest.mark.parametrize("block", [16, 32])
def test_buffers_of_fp4_rows_have_the_sizes_of_the_library(lib, rows, cols, block):
    r = B.Fp4Rows(rows, cols, block, device="meta")
    assert r.codes.numel() == lib.aero_fp4_code_bytes(rows, cols) and r.scales.numel() == lib.aero_fp4_scale_bytes(rows, cols, block)
    assert (r.row_scale is None) if block == 32 else r.row_scale.numel() == rows


def test_binding_refusals():
    for bad in (dict(rows=4, cols=48), dict(rows=4, cols=64, block=8), dict(rows=-1, cols=64)):
        with pytest.raises(B.AeroError):
            B.Fp4Rows(**bad, device="meta")
    with pytest.raises(B.AeroError):
        B.Fp4Rows(4, 64, 16, codes=torch.zeros(7, dtype=torch.uint8))
    n = torch.zeros(8)
    for bad in (dict(param=n, grad=n, m=n, v=n), dict(param=n, grad=n, m=n, v=n, lr=1.0)):          # host tensors, an unknown key
        with pytest.raises(B.AeroError):
            B.AdamWPlan([bad])


@pytest.mark.parametrize("missing", ["param", "grad", "m", "v"])
def test_adamw_plan_with_a_tensor_missing(missing):
    t = {k: torch.zeros(4) for k in ("param", "grad", "m", "v") if k != missing}
    with pytest.raises(B.AeroError, match=missing):
        B.AdamWPlan([t])


@pytest.mark.parametrize("block", [16, 32])
def test_fp4_rows_of_a_part_of_the_buffers(block):
    """Buffers are given all together or not at all: one that is missing would be filled with whatever the memory holds."""
    r = B.Fp4Rows(4, 64, block, device="meta")
    parts = dict(codes=r.codes, scales=r.scales)
    if block == 16:
        parts["row_scale"] = r.row_scale
    for name in parts:
        some = {k: x for k, x in parts.items() if k != name}
        with pytest.raises(B.AeroError, match=f"without {name}"):
            B.Fp4Rows(4, 64, block, device="meta", **some)


def test_adamw_plan_arrays_that_share_memory():
    """Ranges [first, end) of addresses: those that are written touch no other, those that are read may share."""
    def check(written, read):
        B.AdamWPlan._check_apart(written + read)

    a, b, c = (100, 200, 0, "param"), (200, 240, 0, "m"), (240, 300, 1, "v")
    check([a, b, c], [(300, 400, 0, "grad"), (300, 400, 1, "grad"), (350, 360, 2, "grad"), (0, 100, 3, "grad")])
    check([], [])
    check([a], [(100, 100, 1, "grad"), (150, 150, 1, "grad")])                        # nothing in them
    for written, read in (([a, (199, 201, 1, "param")], []), ([a, a], []), ([a, (100, 300, 1, "v"), c], []), ([a], [(150, 160, 0, "grad")]),
                          ([a, b], [(0, 101, 0, "grad")]), ([a, b], [(239, 900, 0, "grad")]), ([(0, 1000, 0, "param"), (10, 20, 1, "m")], []),
                          ([a, c], [(0, 1000, 0, "grad"), (500, 600, 1, "grad")]), ([c], [(0, 1000, 0, "grad"), (20, 30, 1, "grad")])):
        with pytest.raises(B.AeroError, match="overlap"):
            check(written, read)


def test_more_pairs_or_rollouts_than_the_indexes_hold(lib, fake):
    """Steps past the last of 2^31 - 1 would wrap; 2^30 is the limit of both.  (The call ends before the sizes are followed anywhere.)"""
    pc, big = C.byref(B.pref_cfg_default()), (1 << 30) + 1
    for R, pairs in ((big, 4), (3, big), (2 ** 31 - 1, 2 ** 31 - 1)):
        assert lib.aero_pref_fwd(fake, cfg(), pc, 40, 64, 10, R, pairs, P, P, P, P, P, P, None, P, P, P, P, P, P, None, P, 1 << 62) == UNSUPPORTED
        assert lib.aero_pref_fwd_bwd(fake, cfg(), pc, 40, 64, 10, R, pairs, P, P, P, P, P, P, None, P, P, P, P, P, P, None, 1.0, P, P,
                                     B.AERO_FP32, 0, P, 1 << 62) == UNSUPPORTED
    assert lib.aero_pref_bwd(fake, cfg(), 40, 64, 10, big, P, P, P, P, P, P, 1.0, P, P, B.AERO_FP32, 0, P, 1 << 62) == UNSUPPORTED

"""GPU tests of distillation from a teacher's top logits (aero_distill_fwd / _bwd / _fwd_bwd) against the
fp64 statement.

Tolerances, for one row with S = max_v sum_k |h_k w_vk|:
  a logit        (d/8 + 8) 2^-23 S: fp32 accumulation in steps of 16 products, twice for the order of the adds
  log-sum-exp    the logits' error, (V/32 + 64) 2^-24 for the running sum, 2^-20 |lse| for the logarithms
  kl             Q (lse + logit), 2^-18 sum q (|log q| + |log p|) for exp and log of the list
  dz             2^-8 |dz| (rounded to bf16; fp32 path: none) and, one-call step, 2^-8 Q p w (its p~ was too),
                 (Q p + q) w (lse + logit + 2^-17)
                 and Q w 2^-67: p~ = exp(z - c) with c at most 40 above the largest of the row's first logits
                 leaves bf16's range (2^-126 = e^-87) for z 47 below them, that is p below e^-47 < 2^-67
                 (fp32 path: below 2^-126)
  dH, dW         the dz errors through |W|, |H|; 2^-14 of the magnitudes for accumulation; the rounding of the
                 output."""
import numpy as np
import pytest
import torch

from oracle import model_ends as M
from paper_2602_14338_b200 import binding as B
from tests import aero_testlib as TL

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.Context(0)
    yield c
    assert c.last_status() == 0
    c.close()


class Case:
    def __init__(self, T, d, V, K, dtype="bf16", R=None, seed=0, lean=True, teacher_lse=False, drop=True, spread=2.5):
        rng = np.random.default_rng(1000 * seed + T + d + V + K)
        dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.dtype, self.T, self.d, self.V, self.K = dtype, T, d, V, K
        W = torch.from_numpy(rng.standard_normal((V, d)) * 0.05).to(dt)
        ids = rng.integers(0, V, (T, K))
        H = torch.from_numpy(rng.standard_normal((T, d)))
        if lean and T:
            s = rng.choice([0.0, 4.0, 8.0, 14.0], T)       # from a flat row to one the student is sure of
            lead = W[torch.from_numpy(ids[:, 0])].double()
            H = 0.5 * H + torch.from_numpy(s)[:, None] * lead / lead.square().sum(1, keepdim=True)
        self.Ht, self.Wt = H.to(dt), W
        logits = rng.standard_normal((T, K)) * spread + 11.0
        if T >= 6:
            ids[1, K // 2:] = M.NO_TOKEN                   # a shorter list
            ids[2] = M.NO_TOKEN                            # an empty one
            logits[2] = np.nan                             # (its logits are not read)
            logits[3, :] = -np.inf                         # present, without weight
            ids[4] = ids[4, 0]                             # one token in every place
            logits[5, K // 2:] = -np.inf
        self.ids, self.logits = ids.astype(np.int32), logits.astype(np.float32)
        self.tlse = (np.log(np.exp(np.where(np.isfinite(logits), logits, -80)).sum(1)) + 0.3).astype(np.float32) if teacher_lse else None
        R = R if R is not None else max(1, min(T // 5, 9))
        cut = np.sort(rng.choice(np.arange(1, T), R - 1, replace=False)) if R > 1 else np.array([], int)
        self.cs = np.concatenate([[0], cut, [T]]).astype(np.int64)
        self.keep = np.ones(R, np.uint8)
        if drop and R > 2:
            self.keep[1::3] = 0
        self.w = (rng.random(R) * self.keep / max(T, 1)).astype(np.float32)

    def device(self):
        t = lambda a: None if a is None else torch.from_numpy(a).cuda()
        return dict(H=self.Ht.cuda(), W=self.Wt.cuda(), ids=t(self.ids), logits=t(self.logits), cs=t(self.cs), w=t(self.w),
                    keep=t(self.keep)), t(self.tlse)

    @property
    def cfg(self):
        return B.cfg_default(dtype=B.AERO_BF16 if self.dtype == "bf16" else B.AERO_FP32)

    def reference(self, grad_scale=1.0):
        H, W = self.Ht.double().numpy(), self.Wt.double().numpy()
        r = M.distill(H, W, self.ids, self.logits, self.cs, self.w, self.keep, self.tlse, grad_scale)
        S = (np.abs(H) @ np.abs(W).T).max(axis=1) if self.T else np.zeros(0)
        tz = (self.d / 8 + 8) * 2.0 ** -23 * S
        r["t_lse"] = tz + (self.V / 32 + 64) * 2.0 ** -24 + 2.0 ** -20 * np.abs(r["lse"])
        with np.errstate(invalid="ignore"):
            sizes = np.where(r["q"] > 0, r["q"] * (np.abs(r["lq"]) + np.abs(r["lp"])), 0).sum(axis=1)
        r["t_kl"] = r["Q"] * (r["t_lse"] + tz) + 2.0 ** -18 * sizes + 1e-12
        both = r["Q"][:, None] * np.exp(r["z"] - (r["z"].max(1) if self.T else np.zeros(0))[:, None]
                                        - np.log(np.exp(r["z"] - r["z"].max(1)[:, None]).sum(1))[:, None])
        soft = both * (abs(grad_scale) * r["wt"])[:, None]
        for t in range(self.T):
            np.add.at(both[t], np.where(r["there"][t], self.ids[t], 0), r["q"][t])
        both *= (abs(grad_scale) * r["wt"])[:, None]
        half = 2.0 ** -8 if self.dtype == "bf16" else 0.0
        edz = half * (np.abs(r["dz"]) + soft) + both * (r["t_lse"] + tz + 2.0 ** -17)[:, None]
        edz += (abs(grad_scale) * r["wt"] * r["Q"])[:, None] * (2.0 ** -67 if self.dtype == "bf16" else 2.0 ** -126)
        r["t_dH"] = edz @ np.abs(W) + 2.0 ** -14 * (np.abs(r["dz"]) @ np.abs(W)) + half * np.abs(r["dH"])
        r["t_dW"] = edz.T @ np.abs(H) + 2.0 ** -14 * (np.abs(r["dz"]).T @ np.abs(H))
        return r


def close(got, want, tol, what):
    got = got.double().cpu().numpy() if torch.is_tensor(got) else got
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} values, worst {np.nanmax(np.abs(got - want) / np.maximum(tol, 1e-300)):.3g} of the bound"


def check_forward(case, out, r):
    close(out["lse"], r["lse"], r["t_lse"], "lse")
    close(out["kl"], r["kl"], r["t_kl"], "kl")
    loss = float(out["loss"])
    assert abs(loss - r["loss"]) <= (r["wt"] * r["t_kl"]).sum() + 2.0 ** -22 * (r["wt"] * np.abs(r["kl"])).sum() + 1e-12
    kept = max(int(r["kept"].sum()), 1)
    met = out["metrics"].cpu().numpy()
    assert met[3] == r["kept"].sum()
    assert met[0] == pytest.approx((r["kept"] & (r["Q"] == 0)).sum() / kept, abs=1e-6)
    assert met[1] == pytest.approx(r["kl"].sum() / kept, rel=1e-3, abs=1e-5)
    assert met[2] == pytest.approx((r["mass"] * r["kept"]).sum() / kept, rel=1e-3, abs=1e-5)


def check_grads(case, dH, dW, r, dw_half=0.0, base=0.0):
    close(dH, r["dH"], r["t_dH"], "dH")
    close(dW, r["dW"] + base, r["t_dW"] + dw_half * np.abs(r["dW"]) + 2.0 ** -22 * np.abs(base), "dW")
    dropped = torch.from_numpy(~r["kept"]).cuda()
    assert not dH[dropped].any()


BF16 = [dict(T=1, d=64, V=1, K=1), dict(T=1, d=64, V=100, K=3), dict(T=7, d=64, V=65, K=1), dict(T=130, d=128, V=300, K=8),
        dict(T=300, d=192, V=1000, K=33, teacher_lse=True), dict(T=700, d=256, V=2049, K=64), dict(T=257, d=1536, V=700, K=256),
        dict(T=64, d=3584, V=1500, K=5, teacher_lse=True), dict(T=1000, d=64, V=4096, K=20, R=60),
        dict(T=700, d=64, V=300, K=3, R=700), dict(T=20000, d=64, V=100, K=2, R=5000),
        # chunks of one to three token tiles, several units per worker of the dW product, on CTAs and on pairs of them
        dict(T=100, d=64, V=60000, K=4, R=1), dict(T=250, d=320, V=24000, K=4, R=1), dict(T=100, d=2112, V=8000, K=4, R=1),
        dict(T=250, d=2112, V=8000, K=4, R=1), dict(T=380, d=2112, V=8000, K=4, R=1)]
FP32 = [dict(T=1, d=1, V=1, K=1), dict(T=3, d=57, V=100, K=3), dict(T=60, d=64, V=300, K=8, teacher_lse=True),
        dict(T=200, d=96, V=700, K=40), dict(T=41, d=129, V=77, K=70), dict(T=33, d=1024, V=100, K=6)]


@pytest.mark.parametrize("kw", [dict(k, dtype="bf16") for k in BF16] + [dict(k, dtype="fp32") for k in FP32])
def test_forward_backward_and_one_call(ctx, kw):
    case = Case(**kw)
    dv, tl = case.device()
    r = case.reference(grad_scale=1.5)
    out = ctx.distill_fwd(case.cfg, **dv, teacher_lse=tl)
    check_forward(case, out, r)
    dH, dW = ctx.distill_bwd(case.cfg, **dv, lse=out["lse"], teacher_lse=tl, grad_scale=1.5)
    check_grads(case, dH, dW, r)
    out2, dH2, dW2 = ctx.distill_fwd_bwd(case.cfg, **dv, teacher_lse=tl, grad_scale=1.5)
    check_forward(case, out2, r)
    check_grads(case, dH2, dW2, r)
    # the same bits again
    out3, dH3, dW3 = ctx.distill_fwd_bwd(case.cfg, **dv, teacher_lse=tl, grad_scale=1.5)
    for a, b in ((out2["lse"], out3["lse"]), (out2["kl"], out3["kl"]), (out2["loss"], out3["loss"]), (dH2, dH3), (dW2, dW3)):
        assert torch.equal(a, b)
    # added to what is there
    base = torch.randn(case.V, case.d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)) * 1e-2
    b64 = base.double().cpu().numpy()
    _, _, acc = ctx.distill_fwd_bwd(case.cfg, **dv, teacher_lse=tl, grad_scale=1.5, dW=base.clone(), accumulate_dW=True)
    check_grads(case, dH2, acc, r, base=b64)
    _, acc = ctx.distill_bwd(case.cfg, **dv, lse=out["lse"], teacher_lse=tl, grad_scale=1.5, dW=base.clone(), accumulate_dW=True)
    check_grads(case, dH2, acc, r, base=b64)
    assert ctx.last_status() == 0


@pytest.mark.parametrize("tuning", [dict(vsplit=2), dict(vsplit=4), dict(rowscale=0), dict(gemm_pairs=1), dict(gemm_pairs=0, vsplit=2, rowscale=0)])
def test_every_schedule_of_stage_b(ctx, tuning):
    case = Case(T=500, d=256, V=3000, K=17, R=11)
    dv, tl = case.device()
    r = case.reference()
    ctx.set_tuning(**tuning)
    try:
        out, dH, dW = ctx.distill_fwd_bwd(case.cfg, **dv)
        fwd = ctx.distill_fwd(case.cfg, **dv)
        dH2, dW2 = ctx.distill_bwd(case.cfg, **dv, lse=fwd["lse"])
    finally:
        ctx.set_tuning()
    check_forward(case, out, r)
    check_forward(case, fwd, r)
    check_grads(case, dH, dW, r)
    check_grads(case, dH2, dW2, r)
    assert ctx.last_status() == 0


@pytest.mark.parametrize("chunk_tokens", [128, 256, None])
def test_chunks_and_dw_types(ctx, chunk_tokens):
    case = Case(T=900, d=128, V=1111, K=9, R=13)
    dv, _ = case.device()
    r = case.reference()
    lse = ctx.distill_fwd(case.cfg, **dv)["lse"]
    for dt, half in ((torch.float32, 0.0), (torch.bfloat16, 2.0 ** -8)):
        _, dH, dW = ctx.distill_fwd_bwd(case.cfg, **dv, dw_dtype=dt, chunk_tokens=chunk_tokens)
        assert dW.dtype == dt
        check_grads(case, dH, dW, r, half)
        dH, dW = ctx.distill_bwd(case.cfg, **dv, lse=lse, dw_dtype=dt, chunk_tokens=chunk_tokens)
        check_grads(case, dH, dW, r, half)
    assert ctx.last_status() == 0


def test_more_rows_than_one_wave_over_many_vocabulary_tiles(ctx):
    """More than 148 tiles of rows: no planned splits beyond stage (b)'s (8 at most, over nine vocabulary tiles), no split of dH; in
    one chunk and in two, whose bf16 dW has its sums in the workspace."""
    case = Case(T=19500, d=64, V=2300, K=3, R=40)
    dv, _ = case.device()
    r = case.reference()
    fwd = ctx.distill_fwd(case.cfg, **dv)
    check_forward(case, fwd, r)
    for chunk_tokens in (None, 148 * 64):
        for dt, half in ((torch.float32, 0.0), (torch.bfloat16, 2.0 ** -8)):
            out, dH, dW = ctx.distill_fwd_bwd(case.cfg, **dv, dw_dtype=dt, chunk_tokens=chunk_tokens)
            check_forward(case, out, r)
            check_grads(case, dH, dW, r, half)
            dH, dW = ctx.distill_bwd(case.cfg, **dv, lse=fwd["lse"], dw_dtype=dt, chunk_tokens=chunk_tokens)
            check_grads(case, dH, dW, r, half)
    assert ctx.last_status() == 0


@pytest.mark.parametrize("T,d,V", [(100, 256, 3000), (300, 2112, 700), (129, 3584, 290)])
def test_bf16_dw_of_a_few_rows_needs_no_room_for_sums(ctx, T, d, V):
    """One chunk whose block is smaller than an fp32 dW would be; single CTAs and CTA pairs, vocabularies that end inside
    a 128-row tile and inside one of its 32-row pieces."""
    case = Case(T=T, d=d, V=V, K=9, R=1)
    dv, _ = case.device()
    r = case.reference()
    _, dH, dW = ctx.distill_fwd_bwd(case.cfg, **dv, dw_dtype=torch.bfloat16)
    check_grads(case, dH, dW, r, 2.0 ** -8)
    lse = ctx.distill_fwd(case.cfg, **dv)["lse"]
    dH, dW = ctx.distill_bwd(case.cfg, **dv, lse=lse, dw_dtype=torch.bfloat16)
    check_grads(case, dH, dW, r, 2.0 ** -8)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_nothing_kept_and_no_rows(ctx, dtype):
    case = Case(T=200, d=64, V=300, K=4, R=3, dtype=dtype)
    case.keep[:] = 0
    dv, _ = case.device()
    full = lambda *s, dt=torch.float32: torch.full(s, 7.0, dtype=dt, device="cuda")
    types = (torch.float32, torch.bfloat16) if dtype == "bf16" else (torch.float32,)
    for dt in types:
        out, dH, dW = ctx.distill_fwd_bwd(case.cfg, **dv, dW=full(300, 64, dt=dt), dw_dtype=dt,
                                          dH=full(200, 64, dt=case.Ht.dtype))
        assert not dH.any() and not dW.any() and float(out["loss"]) == 0 and not out["kl"].any() and not out["lse"].any()
        dH, dW = ctx.distill_bwd(case.cfg, **dv, lse=out["lse"], dW=full(300, 64, dt=dt), dw_dtype=dt, dH=full(200, 64, dt=case.Ht.dtype))
        assert not dH.any() and not dW.any()
    # no rows at all
    dv.update(H=dv["H"][:0], ids=dv["ids"][:0], logits=dv["logits"][:0], cs=torch.zeros(1, dtype=torch.int64, device="cuda"),
              w=dv["w"][:0], keep=dv["keep"][:0])
    out, dH, dW = ctx.distill_fwd_bwd(case.cfg, **dv, dW=full(300, 64))
    assert dH.shape == (0, 64) and not dW.any() and float(out["loss"]) == 0
    # rows, but no rollout owns them
    dv.update(H=torch.zeros(5, 64, dtype=case.Ht.dtype, device="cuda"), ids=torch.zeros(5, 4, dtype=torch.int32, device="cuda"),
              logits=torch.zeros(5, 4, device="cuda"))
    out, dH, dW = ctx.distill_fwd_bwd(case.cfg, **dv, dW=full(300, 64), dH=full(5, 64, dt=case.Ht.dtype))
    assert not dH.any() and not dW.any() and float(out["loss"]) == 0 and not out["kl"].any() and not out["lse"].any()
    assert ctx.last_status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_of_dropped_rollouts_are_not_looked_at(ctx, dtype):
    """NaN and infinities in the hidden states, lists and logits of dropped rollouts change nothing."""
    case = Case(T=330, d=64, V=500, K=5, dtype=dtype, R=7)
    assert not case.keep.all()
    dv, _ = case.device()
    want = ctx.distill_fwd_bwd(case.cfg, **dv)
    fwd = ctx.distill_fwd(case.cfg, **dv)
    wb = ctx.distill_bwd(case.cfg, **dv, lse=fwd["lse"])
    owner = np.searchsorted(case.cs, np.arange(case.T), side="right") - 1
    gone = torch.from_numpy(case.keep[owner] == 0).cuda()
    dv["H"][gone] = float("nan")
    dv["H"][gone, 3] = float("inf")
    dv["logits"][gone] = float("nan")
    dv["ids"][gone, 0] = 10 ** 6
    got = ctx.distill_fwd_bwd(case.cfg, **dv)
    gb = ctx.distill_bwd(case.cfg, **dv, lse=fwd["lse"])
    assert torch.equal(got[0]["kl"], want[0]["kl"]) and torch.equal(got[0]["loss"], want[0]["loss"])
    for a, b in ((got[1], want[1]), (got[2], want[2]), (gb[0], wb[0]), (gb[1], wb[1])):
        assert torch.equal(a, b)
    assert torch.equal(ctx.distill_fwd(case.cfg, **dv)["kl"], fwd["kl"])
    assert ctx.last_status() == 0


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("where", ["one column", "a split of columns", "all but the listed ones"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_logit_that_is_no_number_shows_in_every_output(ctx, dtype, where, bad):
    """Rows of W that nobody lists hold NaN or infinities: the log-sum-exp of every kept row, the loss and the gradients are then
    no numbers either, wherever in the vocabulary these rows are."""
    V = 3000 if dtype == "bf16" else 300
    case = Case(T=150, d=64, V=V, K=5, dtype=dtype, R=4)
    hit = {"one column": slice(V - 60, V - 59), "a split of columns": slice(V // 3, V // 3 + V // 4), "all but the listed ones": slice(20, V)}[where]
    case.ids = np.where(case.ids >= 0, case.ids % 20, case.ids).astype(np.int32)
    dv, _ = case.device()
    dv["W"][hit] = bad
    kept = torch.from_numpy(case.keep[np.searchsorted(case.cs, np.arange(case.T), side="right") - 1] != 0).cuda()
    fwd = ctx.distill_fwd(case.cfg, **dv)
    out, dH, dW = ctx.distill_fwd_bwd(case.cfg, **dv)
    dH2, dW2 = ctx.distill_bwd(case.cfg, **dv, lse=fwd["lse"])
    for o in (fwd, out):
        assert not torch.isfinite(o["lse"][kept]).any() and not o["lse"][~kept].any()
        assert not torch.isfinite(o["loss"]).any()
    for h, w in ((dH, dW), (dH2, dW2)):
        assert not torch.isfinite(h[0]).any() and not h[~kept].any()      # (row 0 has a full list)
        assert not torch.isfinite(w[hit]).all(dim=1).any()
    assert ctx.last_status() & ~B.AERO_ST_RANGE == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_that_no_rollout_owns(ctx, dtype):
    """Rows before the first offset and behind the last one come out as zeros."""
    case = Case(T=290, d=64, V=400, K=5, dtype=dtype, R=4, drop=False)
    dv, _ = case.device()
    pad = lambda a, fill: torch.cat([torch.full_like(a[:7], fill), a, torch.full_like(a[:50], fill)])
    padded = dict(dv, H=pad(dv["H"], 1.0), ids=pad(dv["ids"], 3), logits=pad(dv["logits"], 1.0), cs=dv["cs"] + 7)
    full = torch.full((347, 64), 9.0, dtype=case.Ht.dtype, device="cuda")
    out = {k: torch.full((347,), 9.0, device="cuda") for k in ("lse", "kl")}
    want, wH, wW = ctx.distill_fwd_bwd(case.cfg, **dv)
    got, gH, gW = ctx.distill_fwd_bwd(case.cfg, **padded, dH=full, out=out)
    r = case.reference()
    check_grads(case, gH[7:297], gW, r)
    close(got["kl"][7:297], r["kl"], r["t_kl"], "kl")
    assert torch.equal(got["loss"], want["loss"]) or abs(float(got["loss"] - want["loss"])) <= 1e-5 * abs(float(want["loss"]))
    for a in (got["lse"], got["kl"], gH):
        assert not a[:7].any() and not a[297:].any()
    assert ctx.last_status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_bad_ids_raise_the_status_bit_and_count_as_empty(ctx, dtype):
    case = Case(T=150, d=64, V=200, K=5, dtype=dtype, R=4)
    dv, _ = case.device()
    good = dv["ids"].clone()
    kept = int(case.cs[2])                          # first row of the third rollout (kept)
    good[kept, 1] = M.NO_TOKEN
    good[0, 0] = M.NO_TOKEN
    want, wH, wW = ctx.distill_fwd_bwd(case.cfg, **dict(dv, ids=good))
    assert ctx.last_status() == 0
    bad = good.clone()
    bad[kept, 1] = 200
    bad[0, 0] = -7
    got, gH, gW = ctx.distill_fwd_bwd(case.cfg, **dict(dv, ids=bad))
    assert ctx.last_status() == B.AERO_ST_BAD_TARGET
    assert torch.equal(got["kl"], want["kl"]) and torch.equal(gH, wH) and torch.equal(gW, wW)


@pytest.mark.parametrize("rowscale", [1, 0])
@pytest.mark.parametrize("kind", ["one far logit", "many high logits"])
def test_rows_beyond_the_range_of_the_stored_exponentials(ctx, kind, rowscale):
    """One logit 130 above the row's first 32 ones (more than bf16 holds of exp(z - c)), and thousands of logits 118
    above them (each in range, their sum not): such rows are redone."""
    case = Case(T=300, d=64, V=6000, K=6, R=3, drop=False, lean=False)
    W = torch.randn(6000, 64, generator=torch.Generator().manual_seed(3)) * 0.02
    H = torch.randn(300, 64, generator=torch.Generator().manual_seed(4))
    H[:, 0] = 0.0
    rows = torch.arange(5, 300, 7)
    H[rows, 0] = 10.0
    if kind == "one far logit":
        W[4000, 0] = 13.0
        case.ids[::2, 1] = 4000
    else:
        W[1000:5500, 0] = 11.8
    case.Ht, case.Wt = H.to(torch.bfloat16), W.to(torch.bfloat16)
    dv, _ = case.device()
    r = case.reference()
    ctx.set_tuning(rowscale=rowscale)
    try:
        out, dH, dW = ctx.distill_fwd_bwd(case.cfg, **dv)
    finally:
        ctx.set_tuning()
    assert ctx.last_status() == 0
    check_forward(case, out, r)
    check_grads(case, dH, dW, r)


def test_rows_out_of_range_in_many_splits_are_listed_once(ctx):
    """64 rows with a logit 130 above the first ones in every vocabulary tile of 235, over which a small call spreads
    dozens of splits: 64 rows to redo, not that many for every split (the list holds 1024)."""
    case = Case(T=64, d=64, V=60000, K=6, R=2, drop=False, lean=False)
    W = torch.randn(60000, 64, generator=torch.Generator().manual_seed(3)) * 0.02
    H = torch.randn(64, 64, generator=torch.Generator().manual_seed(4))
    H[:, 0] = 10.0
    W[:, 0] = 0.0
    W[100::256, 0] = 13.0
    case.ids[::2, 1] = 100 + 256 * 7
    case.Ht, case.Wt = H.to(torch.bfloat16), W.to(torch.bfloat16)
    dv, _ = case.device()
    r = case.reference()
    out, dH, dW = ctx.distill_fwd_bwd(case.cfg, **dv)
    assert ctx.last_status() == 0
    check_forward(case, out, r)
    check_grads(case, dH, dW, r)


def test_gradient_rows_of_a_sure_student(ctx):
    """Rows whose listed token has probability near one on both sides: p - q keeps the accuracy of the log-probs."""
    case = Case(T=256, d=256, V=4096, K=4, R=2, drop=False, lean=False, spread=0.0)
    lead = case.Wt[torch.from_numpy(case.ids[:, 0]).long()].double()
    strength = torch.tensor([15.0, 18.0, 21.0, 24.0], dtype=torch.float64).repeat(64)[:, None]
    case.Ht = (0.05 * torch.randn(256, 256, generator=torch.Generator().manual_seed(1), dtype=torch.float64)
               + strength * lead / lead.square().sum(1, keepdim=True)).to(torch.bfloat16)
    case.logits[:, 0] = 25.0
    dv, _ = case.device()
    r = case.reference()
    assert np.median(np.exp(r["lp"][6:, 0])) > 0.99
    out, dH, dW = ctx.distill_fwd_bwd(case.cfg, **dv)
    check_forward(case, out, r)
    check_grads(case, dH, dW, r)


class SureCase(Case):
    """Rows that leave between 1e-5 and 1e-8 of the probability to all other tokens, on the student's side and on the
    teacher's.  Every row lists token Y, alone or with two others; Y alone has a weight in column 2 of W, which H does not use, so
    dH[t, 2] is Y's entry of row t and nothing else.

    The entry is w (q_o p - q (1 - p)), q_o the weight of the other listed tokens.  Its two terms may be off by 2^-17 (exp,
    log) plus the errors of the logits and of the log-sum-exp without Y, as listed at the head of this file; the entry and dH
    are rounded once each."""
    Y = 1234

    def __init__(self, K, dtype, last=False):
        super().__init__(T=96, d=64, V=4096, K=K, dtype=dtype, R=1, drop=False, lean=False)
        g = torch.Generator().manual_seed(5)
        dt = self.Ht.dtype
        W = torch.randn(4096, 64, generator=g) * 0.02
        H = torch.randn(96, 64, generator=g)
        W[:, 1:3], H[:, 1:3] = 0.0, 0.0
        W[self.Y] = 0.0
        W[self.Y, 1:3] = 1.0
        H[:, 1] = torch.linspace(19.0, 27.0, 96)
        self.Ht, self.Wt = H.to(dt), W.to(dt)
        self.ids[:] = np.array([self.Y, 17, 3000])[:K]
        self.logits[:] = np.array([25.0, 6.0, 3.0])[:K]
        if last:                                           # Y in the last place
            self.ids, self.logits = self.ids[:, ::-1].copy(), self.logits[:, ::-1].copy()
        self.at = K - 1 if last else 0
        self.w[:] = 1.0 / 96

    def check(self, dH, more=0.0):
        r = self.reference()
        q, q_o = r["q"][:, self.at], np.delete(r["q"], self.at, axis=1).sum(axis=1)
        p = np.exp(r["lp"][:, self.at])
        left = np.exp(np.logaddexp.reduce(np.delete(r["z"], self.Y, axis=1), axis=1) - r["lse"])      # 1 - p
        assert 5e-9 < left.min() < 2e-8 and 5e-6 < left.max() < 5e-5
        S = (np.abs(self.Ht.double().numpy()) @ np.abs(self.Wt.double().numpy()).T).max(axis=1)
        rel = 2 * (self.d / 8 + 8) * 2.0 ** -23 * S + (self.V / 32 + 64) * 2.0 ** -24 + 2.0 ** -17
        half = 2 * 2.0 ** -8 if self.dtype == "bf16" else 2.0 ** -22
        want = r["wt"] * (q_o * p - q * left)
        close(dH[:, 2], want, half * np.abs(want) + (rel + more) * r["wt"] * (q_o * p + q * left), "entry of the sure token")


@pytest.mark.parametrize("K", [1, 3])
def test_entry_of_a_token_that_both_are_sure_of(ctx, K):
    case = SureCase(K, "bf16")
    dv, _ = case.device()
    _, dH, _ = ctx.distill_fwd_bwd(case.cfg, **dv)
    case.check(dH)
    assert ctx.last_status() == 0


@pytest.mark.parametrize("K,dtype", [(1, "bf16"), (3, "bf16"), (1, "fp32"), (3, "fp32")])
def test_entry_of_a_sure_token_from_the_rounded_lse(ctx, K, dtype):
    """The backward alone gets lse rounded to 2^-20, far above 1 - p; and both forms in fp32.  For bf16 rows it makes 1 - p of the
    other columns' dz, which are rounded to bf16."""
    case, more = SureCase(K, dtype), 2.0 ** -8 if dtype == "bf16" else 0.0
    dv, _ = case.device()
    out, dH, _ = ctx.distill_fwd_bwd(case.cfg, **dv)
    case.check(dH)
    dH, _ = ctx.distill_bwd(case.cfg, **dv, lse=out["lse"])
    case.check(dH, more)
    # an lse that is as far off as rounding can make it stands in all terms alike and changes 1 - p by as much, relative
    dH, _ = ctx.distill_bwd(case.cfg, **dv, lse=out["lse"] * (1 + 2.0 ** -23))
    case.check(dH, more)
    assert ctx.last_status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_entry_of_a_sure_token_that_is_not_listed_first(ctx, dtype):
    """The teacher's list need not be sorted."""
    case, more = SureCase(3, dtype, last=True), 2.0 ** -8 if dtype == "bf16" else 0.0
    dv, _ = case.device()
    out, dH, _ = ctx.distill_fwd_bwd(case.cfg, **dv)
    case.check(dH)
    dH, _ = ctx.distill_bwd(case.cfg, **dv, lse=out["lse"])
    case.check(dH, more)
    assert ctx.last_status() == 0


def test_captured_and_replayed(ctx):
    side = torch.cuda.Stream()
    c = B.Context(0, stream=side)
    case = Case(T=200, d=128, V=900, K=7, R=4)
    dv, _ = case.device()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        c.distill_fwd_bwd(case.cfg, **dv)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        out, dH, dW = c.distill_fwd_bwd(case.cfg, **dv)
    for seed in (5, 6):
        other = Case(T=200, d=128, V=900, K=7, R=4, seed=seed)
        ov, _ = other.device()
        for k in ("H", "W", "ids", "logits", "w"):
            dv[k].copy_(ov[k])
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        want, wH, wW = ctx.distill_fwd_bwd(case.cfg, **dv)
        assert torch.equal(out["kl"], want["kl"]) and torch.equal(out["loss"], want["loss"])
        assert torch.equal(dH, wH) and torch.equal(dW, wW)
    assert c.last_status() == 0
    del g
    c.close()


def test_separate_calls_captured_and_replayed(ctx):
    """The forward and the backward of its lse in one graph, with rows the student is sure of, replayed on other contents."""
    side = torch.cuda.Stream()
    c = B.Context(0, stream=side)
    case = SureCase(3, "bf16")
    dv, _ = case.device()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        lse = c.distill_fwd(case.cfg, **dv)["lse"]
        c.distill_bwd(case.cfg, **dv, lse=lse)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        out = c.distill_fwd(case.cfg, **dv)
        dH, dW = c.distill_bwd(case.cfg, **dv, lse=out["lse"])
    for turn in (1, 2):
        dv["H"].copy_(dv["H"].roll(7 * turn, 0))
        dv["logits"].mul_(0.9)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        want = ctx.distill_fwd(case.cfg, **dv)
        wH, wW = ctx.distill_bwd(case.cfg, **dv, lse=want["lse"])
        assert torch.equal(out["lse"], want["lse"]) and torch.equal(out["loss"], want["loss"])
        assert torch.equal(dH, wH) and torch.equal(dW, wW)
    assert c.last_status() == 0
    del g
    c.close()


def test_two_calls_at_once(ctx):
    """Two contexts on two streams, their calls under way at the same time: the same bits as one after the other."""
    cases = [Case(T=300, d=192, V=5000, K=9, R=4), Case(T=700, d=256, V=3000, K=20, R=6)]
    inputs = [c.device()[0] for c in cases]
    want = [ctx.distill_fwd_bwd(c.cfg, **dv) for c, dv in zip(cases, inputs)]
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    own = [B.Context(0, stream=s) for s in side]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(4):
        for i in (0, 1):
            with torch.cuda.stream(side[i]):
                got[i].append(own[i].distill_fwd_bwd(cases[i].cfg, **inputs[i]))
    torch.cuda.synchronize()
    for i in (0, 1):
        for o, dH, dW in got[i]:
            assert torch.equal(o["kl"], want[i][0]["kl"]) and torch.equal(o["loss"], want[i][0]["loss"])
            assert torch.equal(dH, want[i][1]) and torch.equal(dW, want[i][2])
        assert own[i].last_status() == 0
        own[i].close()


def test_with_stage_b_in_one_process(ctx):
    """Stage (b) and the distillation share kernels, whichever of them a process runs first: the log-prob pass and the
    three calls of the loss, the distillation's, and the first again, each with the same bits as before."""
    case = Case(T=300, d=192, V=1000, K=8)
    dv, _ = case.device()
    T, R = case.T, len(case.keep)
    g = torch.Generator().manual_seed(3)
    y = torch.randint(0, case.V, (T,), generator=g).int().cuda()
    old = (-torch.rand(T, generator=g) * 5).cuda()
    adv = torch.randn(R, generator=g).cuda()

    def stage_b():
        f = ctx.grpo_loss_fwd(case.cfg, dv["H"], dv["W"], y, old, dv["cs"], adv, dv["w"], dv["keep"])
        dH, dW = ctx.grpo_loss_bwd(case.cfg, dv["H"], dv["W"], y, dv["cs"], dv["keep"], f["lse"], f["g"], logp=f["logp"])
        f2, dH2, dW2 = ctx.grpo_loss_fwd_bwd(case.cfg, dv["H"], dv["W"], y, old, dv["cs"], adv, dv["w"], dv["keep"])
        kept = dv["keep"].bool()[torch.searchsorted(dv["cs"], torch.arange(T, device="cuda"), right=True) - 1]
        return [f["lse"][kept].clone(), dW.clone(), f2["lse"][kept].clone(), dW2.clone()]

    def distill():
        f = ctx.distill_fwd(case.cfg, **dv)
        dH, dW = ctx.distill_bwd(case.cfg, **dv, lse=f["lse"])
        f2, dH2, dW2 = ctx.distill_fwd_bwd(case.cfg, **dv)
        return [f["lse"].clone(), dH.clone(), dW.clone(), f2["lse"].clone(), dH2.clone(), dW2.clone()]

    b, e = stage_b(), distill()
    for was, now in zip(b + e, stage_b() + distill()):
        assert torch.equal(was, now)
    check_forward(case, ctx.distill_fwd(case.cfg, **dv), case.reference())
    assert ctx.last_status() == 0


def test_a_step_of_the_ends_together(ctx):
    """As a training step uses them: the frozen teacher's final norm with its 8-bit output and the 8-bit product give
    logits, whose largest are the teacher's list; the student's norm gives H; the group stage gives keep and weights; the
    distillation gives dH and the tied weight's dW; the norm's backward gives the gradient of the last hidden state, the
    embedding's backward adds its share to the tied dW."""
    T, d, V, K, P = 600, 256, 3000, 12, 6
    g = torch.Generator().manual_seed(11)
    bf = lambda *s, std=1.0: (torch.randn(*s, generator=g) * std).to(torch.bfloat16).cuda()
    x, res, gamma, W = bf(T, d), bf(T, d), bf(d, std=0.1) + 1, bf(V, d, std=0.1)
    tx, tgamma, tW = bf(T, d), bf(d, std=0.1) + 1, bf(V, d, std=0.1)
    cfg = B.cfg_default()
    # teacher
    t8 = ctx.rmsnorm_fwd(cfg, tx, tgamma, h=False, quant=True)
    w8, ws = ctx.quantize_rows(cfg, tW)
    z = ctx.lmhead_q8(t8["q"], t8["q_scale"], w8, ws, out_dtype=torch.float32)
    top = torch.topk(z, K, dim=1)
    ids, logits = top.indices.int().contiguous(), top.values.contiguous()
    tlse = torch.logsumexp(z, dim=1)
    exact = M.rmsnorm_fwd(tx.double().cpu().numpy(), tgamma.double().cpu().numpy())[2] @ tW.double().cpu().numpy().T
    # each operand is off by at most half a step of its row: 1/254 of the row's largest value
    h = np.abs(M.rmsnorm_fwd(tx.double().cpu().numpy(), tgamma.double().cpu().numpy())[2])
    wv = np.abs(tW.double().cpu().numpy())
    bound = (h.max(1)[:, None] * wv.sum(1)[None, :] + h.sum(1)[:, None] * wv.max(1)[None, :]) / 254 + d * h.max(1)[:, None] * wv.max(1)[None, :] / 254 ** 2
    assert (np.abs(z.double().cpu().numpy() - exact) <= 1.01 * bound).all()
    # student
    cs = torch.arange(0, T + 1, T // (P * 4), dtype=torch.int64, device="cuda")
    go = torch.arange(0, P * 4 + 1, 4, dtype=torch.int32, device="cuda")
    reward = torch.tensor(([1.0, 0, 0, 1] + [1.0] * 4 + [0.0, 1, 0, 0]) * 2, device="cuda")
    grp = ctx.group_stats(cfg, go, reward, cs)
    n = ctx.rmsnorm_fwd(cfg, x, gamma, residual=res)
    out, dH, dW = ctx.distill_fwd_bwd(cfg, n["h"], W, ids, logits, cs, grp["w"], grp["keep"], teacher_lse=tlse)
    dx, dgamma = ctx.rmsnorm_bwd(cfg, dH, n["sum"], gamma, n["rstd"])
    y = torch.randint(0, V, (T,), generator=g).int().cuda()
    emb = ctx.embed_fwd(cfg, W, y, scale=16.0)
    tied = ctx.embed_bwd(cfg, dx, y, V, scale=16.0, dW=dW.clone(), accumulate_dW=True)
    assert ctx.last_status() == 0
    # the same chain in fp64 from what each operator was given
    f = lambda t: t.double().cpu().numpy()
    s64, r64, h64 = M.rmsnorm_fwd(f(x), f(gamma), f(res))
    ref = M.distill(f(n["h"]), f(W), ids.cpu().numpy(), f(logits), cs.cpu().numpy(), f(grp["w"]), grp["keep"].cpu().numpy(), f(tlse))
    assert grp["keep"].sum().item() == 16 and float(out["metrics"][3]) == 400
    assert abs(float(out["loss"]) - ref["loss"]) <= 1e-4 * abs(ref["loss"])
    rdx, rdg = M.rmsnorm_bwd(ref["dH"], s64, f(gamma), r64)
    rtied = ref["dW"] + M.embed_bwd(rdx, y.cpu().numpy(), V, 16.0)[0]
    # bf16 roundings along the way (h, dz, scaled rows, dH, dx: 2^-8 each at most)
    assert TL.rel_l2(f(n["h"]), h64) <= 2.0 ** -8
    assert TL.rel_l2(f(dx), rdx) <= 5 * 2.0 ** -8 and TL.rel_l2(f(dgamma), rdg) <= 5 * 2.0 ** -8
    assert TL.rel_l2(f(tied), rtied) <= 5 * 2.0 ** -8
    assert TL.rel_l2(f(emb), M.embed_fwd(f(W), y.cpu().numpy(), 16.0)) <= 2.0 ** -8

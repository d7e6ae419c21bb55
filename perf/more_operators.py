"""Measured cases of the operators of a preference-training step: the loss on pairs of rollouts through the lm_head, the AdamW
step over many tensors, and the lm_head product in 4-bit floating point with its quantisation.

run() computes an operator in plain torch, or, with `own` set, through this library's calls.  Sizes are those of the
library's workloads (d = 1536, V = 151936 and d = 3584, V = 152064) and generic ones around them."""
import math

import torch

own = False

SMALL, LARGE = (1536, 151936), (3584, 152064)
BETAS, EPS, DECAY, RATE, MAX_NORM = (0.9, 0.95), 1e-8, 0.1, 1e-3, 1.0
BETA = 0.1
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
_CTX = {}


def _context():
    """The handle a program keeps for the current device, on the current stream."""
    device = torch.cuda.current_device()
    ctx = _CTX.get(device)
    if ctx is None:
        from paper_2602_14338_b200 import binding

        ctx = _CTX[device] = binding.Context(device)
    if ctx.stream.cuda_stream != torch._C._cuda_getCurrentRawStream(device):
        ctx.set_stream(torch.cuda.current_stream())
    return ctx


def _cfg(dtype):
    from paper_2602_14338_b200 import binding

    return binding.cfg_default(dtype=binding.AERO_FP32 if dtype == "fp32" else binding.AERO_BF16)


def listed():
    s, big = dict(d=SMALL[0], V=SMALL[1]), dict(d=LARGE[0], V=LARGE[1])
    return [
        # evaluation of the preference loss on a few held-out groups of the small policy
        dict(name="preference loss 1000", op="pref", grads=False, T=1000, R=10, kind="logistic", mean=False, dtype="bf16", **s),
        # a micro-batch of a few short pairs of the small policy, loss and gradients
        dict(name="preference step 333", op="pref", grads=True, T=333, R=5, kind="logistic", mean=False, dtype="bf16", **s),
        # an ordinary micro-batch of the large policy, loss and gradients, log-probs averaged over a rollout's tokens
        dict(name="preference step 4096", op="pref", grads=True, T=4096, R=16, kind="square", mean=True, dtype="bf16", **big),
        # the norms and biases of the small policy, updated in full precision
        dict(name="adamw 32 bits 60 tensors", op="adamw", bits=32, numel=1536, count=60, small=1536, param="fp32", grad="fp32"),
        # an adapter of the large policy: bf16 weights with their fp32 master
        dict(name="adamw 32 bits adapters", op="adamw", bits=32, numel=3584 * 64, count=40, small=64 * 1537, param="bf16",
             grad="bf16"),
        # the tied weight of the small policy and its final norm, states in 8 bits
        dict(name="adamw 8 bits tied weight", op="adamw", bits=8, numel=SMALL[0] * SMALL[1], count=2, small=1536, param="bf16",
             grad="bf16"),
        # final hidden states of a batch of sequences being decoded, to 4 bits and back
        dict(name="4 bits and back 61 rows", op="fp4_rows", T=61, d=SMALL[0], block=16, dtype="bf16"),
        # the lm_head weight of the large policy, once per weight, and read back
        dict(name="4 bits and back lm_head", op="fp4_rows", T=LARGE[1], d=LARGE[0], block=16, dtype="bf16"),
        # next-token logits of one sequence
        dict(name="product 4 bits 1", op="fp4", T=1, out="fp32", block=16, **big),
        # next-token logits of a batch of sequences being decoded, in the format with a power of two per 32
        dict(name="product 4 bits 61", op="fp4", T=61, out="bf16", block=32, **s),
        # logits of a frozen reference over a chunk of tokens
        dict(name="product 4 bits 2048", op="fp4", T=2048, out="bf16", block=16, **big),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["pref", "pref", "adamw", "adamw", "fp4_rows", "fp4", "fp4"])
    if op == "pref":
        kind, mean = rng.choice(["logistic", "logistic", "square", "hinge"]), rng.random() < 0.4
        if rng.random() < 0.2:          # the plain fp32 path, for small shapes
            T = _log_int(rng, 4, 200)
            return dict(op=op, grads=rng.random() < 0.7, T=T, R=rng.randint(2, min(T, 10)), kind=kind, mean=mean, dtype="fp32",
                        d=rng.randint(8, 96), V=rng.randint(100, 900))
        d, V = rng.choice([SMALL, LARGE, (64 * rng.randint(1, 64), _log_int(rng, 600, LARGE[1]))])
        T = _log_int(rng, 16, 3000 * LARGE[0] // max(d, LARGE[0]))
        return dict(op=op, grads=rng.random() < 0.7, T=T, R=rng.randint(2, min(T, 24)), kind=kind, mean=mean, dtype="bf16", d=d, V=V)
    if op == "adamw":
        if rng.random() < 0.5:          # many small tensors
            count = rng.randint(2, 200)
            numel = small = _log_int(rng, 1, 100000)
        else:                           # one large tensor and a few small ones
            count, numel, small = rng.randint(1, 4), _log_int(rng, 100000, 160 * 10 ** 6), rng.randint(1, 9000)
        return dict(op=op, bits=rng.choice([8, 32]), numel=numel, count=count, small=small, param=rng.choice(["bf16", "fp32"]),
                    grad=rng.choice(["bf16", "fp32"]))
    block = rng.choice([16, 32])
    d, V = rng.choice([SMALL, LARGE, (32 * rng.randint(2, 150), _log_int(rng, 200, LARGE[1]))])
    if op == "fp4_rows":
        return dict(op=op, T=_log_int(rng, 1, min(V, LARGE[0] * LARGE[1] // d)), d=d, block=block, dtype=rng.choice(["bf16", "bf16", "fp32"]))
    return dict(op=op, T=_log_int(rng, 1, 2048 * LARGE[0] // max(d, LARGE[0])), d=d, V=V, block=block, out=rng.choice(["bf16", "fp32"]))


# ---- shapes that follow from a case ----------------------------------------------------------------------------------

def _rollouts(case):
    """Token offsets of a case's rollouts (ragged), and its pairs (chosen, rejected): of every five rollouts two are
    preferred to two others, each to each, and the fifth is in no pair."""
    T, R = case["T"], case["R"]
    cs = [T * i // R + (i % 3 if 0 < i < R and T >= 8 * R else 0) for i in range(R + 1)]
    pairs = []
    for g in range(0, R, 5):
        if g + 4 <= R:
            pairs += [(g, g + 2), (g, g + 3), (g + 1, g + 2), (g + 1, g + 3)]
        elif g + 2 <= R:
            pairs.append((g + 1, g))
    return cs, pairs


def _rows_in_pairs(case):
    cs, pairs = _rollouts(case)
    return sum(cs[i + 1] - cs[i] for i in {i for p in pairs for i in p})


def _size(dtype):
    return 4 if dtype == "fp32" else 2


def _dt(dtype):
    return torch.float32 if dtype == "fp32" else torch.bfloat16


def _pad(n, m):
    return (n + m - 1) // m * m


# ---- the 8-bit states: m as e4m3 times a scale per 256 elements, the root of v as an unsigned 8-bit float times another --------

def _encode_m(m):
    """(codes, scales) of [blocks, 256] values."""
    top = m.abs().amax(1).clamp(min=2.0 ** -100)
    return (m * (448.0 / top)[:, None]).to(torch.float8_e4m3fn), top / 448.0


def _encode_v(v):
    """The root of v with four exponent and four mantissa bits (0 .. 496): the bits of a float whose exponent is moved so that
    the smallest normal numbers of the two fall together, rounded to even; what is not zero does not become zero."""
    r = torch.sqrt(v)
    top = r.amax(1).clamp(min=2.0 ** -100)
    bits = ((r * (496.0 / top)[:, None]) * 2.0 ** -120).view(torch.int32)
    code = ((bits + 0x3FFFF + ((bits >> 19) & 1)) >> 19).clamp(max=255)
    return torch.where(r > 0, code.clamp(min=1), code).to(torch.uint8), top / 496.0


def _decode_m(code, scale):
    return code.float() * scale[:, None]


def _decode_v(code, scale):
    r = (code.int() << 19).view(torch.float32) * 2.0 ** 120 * scale[:, None]
    return r * r


# ---- the 4-bit rows: two e2m1 codes to a byte, in tiles of 128 rows and 256 columns, scales in groups of 128 rows and 4 blocks --------

def _round_e2m1(y):
    """Codes 0 .. 7 (with the sign in bit 3) of the nearest e2m1 values, ties to the even code, 6 at most."""
    a = y.abs()
    code = ((a > 0.25).byte() + (a >= 0.75).byte() + (a > 1.25).byte() + (a >= 1.75).byte() + (a > 2.5).byte() + (a >= 3.5).byte()
            + (a > 5.0).byte())
    return code | (torch.signbit(y).byte() << 3)


def _quantise(x, block):
    """Codes [rows, d], scale bytes [rows, d / block], scale values [rows, d / block] and row scales [rows] of rows in fp32."""
    T, d = x.shape
    xb = x.view(T, d // block, block)
    top = xb.abs().amax(2)
    if block == 32:
        # the power of two that brings the largest of 32 into [4, 8)
        e = (torch.frexp(top).exponent - 3).clamp(-127, 127)
        e = torch.where(top > 0, e, torch.full_like(e, -127))
        scale = torch.ldexp(torch.ones_like(top), e)
        return _round_e2m1(xb / scale[:, :, None]).view(T, d), (e + 127).byte(), scale, None
    # a power of two per row that brings the largest scale of 16 under 448
    part = torch.frexp(top.amax(1) / 2688.0)
    e = (part.exponent - (part.mantissa == 0.5).int()).clamp(min=-126)
    row = torch.where(top.amax(1) > 0, torch.ldexp(torch.ones_like(top[:, 0]), e), torch.zeros_like(top[:, 0]))
    unit = torch.where(row > 0, row, torch.ones_like(row))
    scale8 = (top / unit[:, None] / 6.0).clamp(max=448.0).to(torch.float8_e4m3fn)
    scale = scale8.float()
    y = xb / unit[:, None, None] / torch.where(scale > 0, scale, torch.ones_like(scale))[:, :, None]
    code = torch.where((scale > 0)[:, :, None], _round_e2m1(y), torch.zeros_like(y, dtype=torch.uint8))
    return code.view(T, d), scale8.view(torch.uint8), scale * row[:, None], row


def _values(code, scale, block):
    """The values that codes and scale values stand for."""
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=code.device)
    T, d = code.shape
    return (table[code.int()].view(T, d // block, block) * scale[:, :, None]).view(T, d)


def _swizzle(rows):
    """Where the 16-byte chunk c of a row stands in its 128 bytes: at c xor (row mod 8)."""
    return torch.arange(8, device="cuda")[None, :] ^ (torch.arange(rows, device="cuda")[:, None] & 7)


def _lay_out(code, scale8, block):
    """Rows as the library keeps them: [row tiles][slabs of 256 columns][128 rows][128 bytes], 16-byte chunks swizzled, and
    [row tiles][groups of 4 blocks][32][4][4] scale bytes."""
    T, d = code.shape
    rt, slabs = _pad(T, 128) // 128, _pad(d, 256) // 256
    packed = torch.zeros(rt * 128, slabs * 128, dtype=torch.uint8, device="cuda")
    packed[:T, :d // 2] = code[:, 0::2] | (code[:, 1::2] << 4)
    at = _swizzle(128)[None, None, :, :, None]
    chunks = packed.view(rt, 128, slabs, 8, 16).transpose(1, 2)
    codes = torch.gather(chunks, 3, at.expand(rt, slabs, 128, 8, 16))
    groups = slabs * 256 // (4 * block)
    s = torch.zeros(rt * 128, groups * 4, dtype=torch.uint8, device="cuda")
    s[:T, :d // block] = scale8
    return codes.reshape(-1), s.view(rt, 4, 32, groups, 4).permute(0, 3, 2, 1, 4).reshape(-1)


def _unfold(codes, scales, row_scale, T, d, block):
    """The values of rows laid out like that, in fp32."""
    rt, slabs = _pad(T, 128) // 128, _pad(d, 256) // 256
    at = _swizzle(128)[None, None, :, :, None]
    chunks = torch.gather(codes.view(rt, slabs, 128, 8, 16), 3, at.expand(rt, slabs, 128, 8, 16))
    packed = chunks.transpose(1, 2).reshape(rt * 128, slabs * 128)[:T, :d // 2]
    code = torch.stack((packed & 15, packed >> 4), dim=2).view(T, d)
    groups = slabs * 256 // (4 * block)
    s = scales.view(rt, groups, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(rt * 128, groups * 4)[:T, :d // block]
    if block == 32:
        scale = torch.ldexp(torch.ones(s.shape, device="cuda"), s.int() - 127)
    else:
        scale = s.contiguous().view(torch.float8_e4m3fn).float() * row_scale[:, None]
    return _values(code, scale, block)


# ---- inputs -------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, std=1.0, dtype=torch.float32):
        return torch.randn(*shape, generator=g, device="cuda").mul_(std).to(dtype)

    op = case["op"]
    s = dict(case=case)
    if op == "pref":
        T, d, V, dt = case["T"], case["d"], case["V"], _dt(case["dtype"])
        cs, pairs = _rollouts(case)
        s["W"] = normal(V, d, std=0.02, dtype=dt)
        # text-like targets (id v about as often as 1 / v); half of the rows lean towards theirs, as a trained policy does
        u = torch.rand(T, generator=g, device="cuda", dtype=torch.float64)
        y = torch.randperm(V, generator=g, device="cuda")[(V ** u - 1).long().clamp_(0, V - 1)]
        H = normal(T, d)
        lean = s["W"][y[::2]].float()
        H[::2] = 0.25 * H[::2] + lean * (math.log(V) / lean.square().sum(1, keepdim=True))
        s["H"] = H.to(dt)
        # the reference's log-probs: the policy's own, moved a little for each token and a little more for each rollout
        ref = torch.empty(T, device="cuda")
        for t in range(0, T, 512):
            z = (s["H"][t:t + 512] @ s["W"].T).float()
            ref[t:t + 512] = torch.log_softmax(z, 1).gather(1, y[t:t + 512, None])[:, 0]
        owner = torch.searchsorted(torch.tensor(cs, device="cuda"), torch.arange(T, device="cuda"), right=True) - 1
        s["ref"] = ref + normal(T, std=0.3) - normal(case["R"], std=0.1)[owner.clamp(0, case["R"] - 1)]
        masked = torch.rand(T, generator=g, device="cuda") < 0.05           # tokens that are not scored
        s["y"] = y.int().masked_fill_(masked, -1)
        s["cs"] = torch.tensor(cs, dtype=torch.int64, device="cuda")
        s["pairs"] = torch.tensor(pairs, dtype=torch.int32, device="cuda")
    elif op == "adamw":
        # flat buffers; each tensor starts at a multiple of 256 elements, with zeros up to the next one
        first, rest, n_rest = case["numel"], case["small"], case["count"] - 1
        total = _pad(first, 256) + n_rest * _pad(rest, 256)
        live = torch.zeros(total, dtype=torch.bool, device="cuda")
        live[:first] = True
        live[_pad(first, 256):].view(n_rest, _pad(rest, 256))[:, :rest] = True
        size = torch.exp(normal(total // 256, 1, std=1.0)).expand(-1, 256).reshape(-1) * 1e-4      # gradients of rows differ in size
        s["grad"] = (normal(total) * size * live).to(_dt(case["grad"]))
        m = normal(total, std=0.3) * size * live
        v = (size * live * torch.exp(normal(total, std=0.5))).square()
        p = normal(total, std=0.02) * live
        del live, size
        if case["param"] == "bf16":
            s["master"], s["param"] = p, p.bfloat16()
        else:
            s["param"] = p
        if case["bits"] == 8:
            s["m"], s["m_scale"] = _encode_m(m.view(-1, 256))
            s["v"], s["v_scale"] = _encode_v(v.view(-1, 256))
        else:
            s["m"], s["v"] = m, v
        s["step"] = torch.full((1,), 100, dtype=torch.int64, device="cuda")
    elif op == "fp4_rows":
        T, d = case["T"], case["d"]
        # hidden states and weights: some columns are larger than the rest
        s["x"] = (normal(T, d) * torch.exp(normal(d, std=0.5)) * torch.exp(normal(T, 1, std=0.5)) * 0.05).to(_dt(case["dtype"]))
    else:
        T, d, V, block = case["T"], case["d"], case["V"], case["block"]
        for name, rows, std in (("h", T, 1.0), ("w", V, 0.02)):
            code, scale8, row = [], [], []
            for r in range(0, rows, 32768):
                c, s8, _, rs = _quantise(normal(min(32768, rows - r), d, std=std), block)
                code.append(c)
                scale8.append(s8)
                row.append(rs)
            s[name], s[name + "_scale"] = _lay_out(torch.cat(code), torch.cat(scale8), block)
            s[name + "_row"] = None if block == 32 else torch.cat(row)
    return s


# ---- plain forms ------------------------------------------------------------------------------------------------------

def _plain_pref(s):
    case = s["case"]
    H, W, cs, T, R = s["H"].float(), s["W"].float(), s["cs"], case["T"], case["R"]
    owner = torch.searchsorted(cs, torch.arange(T, device="cuda"), right=True) - 1
    used = torch.zeros(R, device="cuda").index_fill_(0, s["pairs"].flatten().long(), 1.0)
    scored = (s["y"] >= 0) & (used[owner] > 0)
    at = s["y"].long().clamp(min=0)
    z = H @ W.T
    top = z.amax(1)
    lse = top + torch.log(torch.exp(z - top[:, None]).sum(1))
    logp = torch.where(scored, z.gather(1, at[:, None])[:, 0] - lse, torch.zeros_like(lse))
    diff = torch.where(scored, logp - s["ref"], torch.zeros_like(lse)).double()
    ratio = torch.zeros(R, dtype=torch.float64, device="cuda").index_add_(0, owner, diff)
    count = torch.zeros(R, dtype=torch.float64, device="cuda").index_add_(0, owner, scored.double()).clamp(min=1.0)
    per = 1.0 / count if case["mean"] else torch.ones_like(count)
    ratio = ratio * per
    chosen, rejected = s["pairs"][:, 0].long(), s["pairs"][:, 1].long()
    margin = BETA * (ratio[chosen] - ratio[rejected])
    n = margin.numel()
    if case["kind"] == "logistic":
        each, slope = torch.log1p(torch.exp(-margin.abs())) + (-margin).clamp(min=0.0), -1.0 / (1.0 + torch.exp(margin))
    elif case["kind"] == "square":
        each, slope = (margin - 0.5).square(), 2.0 * (margin - 0.5)
    else:
        each, slope = (1.0 - margin).clamp(min=0.0), -(margin < 1.0).double()
    out = dict(logp=logp, ratio=(ratio * used).float(), margin=margin.float(), loss=each.mean().float())
    if case["grads"]:
        coef = torch.zeros(R, dtype=torch.float64, device="cuda").index_add_(0, chosen, BETA / n * slope)
        coef = coef.index_add_(0, rejected, -BETA / n * slope) * per
        g = (coef[owner] * scored).float()
        dz = -g[:, None] * torch.exp(z - lse[:, None])
        dz.scatter_add_(1, at[:, None], g[:, None])
        out["dH"] = (dz @ W).to(s["H"].dtype)
        out["dW"] = (dz.T @ H).to(s["W"].dtype)
    return out


def _plain_adamw(s):
    case = s["case"]
    first = _pad(case["numel"], 256)
    g = s["grad"].float()
    norm = torch.sqrt(s["grad"].double().square().sum())
    clip = (MAX_NORM / (norm + 1e-6)).clamp(max=1.0).float()
    g = g * clip
    if case["bits"] == 8:
        m, v = _decode_m(s["m"], s["m_scale"]).view(-1), _decode_v(s["v"], s["v_scale"]).view(-1)
    else:
        m, v = s["m"], s["v"]
    m = BETAS[0] * m + (1.0 - BETAS[0]) * g
    v = BETAS[1] * v + (1.0 - BETAS[1]) * g * g
    t = (s["step"] + 1).double()
    c1, c2 = (1.0 - BETAS[0] ** t).float(), (1.0 - BETAS[1] ** t).float()
    p = s["master"] if "master" in s else s["param"]
    p[:first] *= 1.0 - RATE * DECAY                                          # the rest is not decayed
    p -= RATE * (m / c1) / (torch.sqrt(v / c2) + EPS)
    if "master" in s:
        s["param"].copy_(p)
    s["step"] += 1
    out = dict(param=s["param"], norm=norm.float())
    if "master" in s:
        out["master"] = s["master"]
    if case["bits"] == 8:
        s["m"], s["m_scale"] = _encode_m(m.view(-1, 256))
        s["v"], s["v_scale"] = _encode_v(v.view(-1, 256))
        # what is held in 8 bits, as the values it stands for
        out["m"] = _decode_m(s["m"], s["m_scale"]).view(-1).bfloat16()
        out["v"] = _decode_v(s["v"], s["v_scale"]).view(-1).bfloat16()
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
        out.update(m=s["m"], v=s["v"])
    return out


def _plain_rows(s):
    code, _, scale, row = _quantise(s["x"].float(), s["case"]["block"])
    out = dict(value=_values(code, scale, s["case"]["block"]).bfloat16())
    return out if row is None else dict(out, row_scale=row)


def _plain_product(s):
    c = s["case"]
    h = _unfold(s["h"], s["h_scale"], s["h_row"], c["T"], c["d"], c["block"])
    w = _unfold(s["w"], s["w_scale"], s["w_row"], c["V"], c["d"], c["block"])
    return (h @ w.T).to(_dt(c["out"]))


# ---- the library's calls ----------------------------------------------------------------------------------------------

def _own_pref(ctx, s):
    from paper_2602_14338_b200 import binding

    case = s["case"]
    pc = binding.pref_cfg_default(beta=BETA, mean=int(case["mean"]), kind=dict(
        logistic=binding.AERO_PREF_LOGISTIC, square=binding.AERO_PREF_SQUARE, hinge=binding.AERO_PREF_HINGE)[case["kind"]])
    args = (_cfg(case["dtype"]), pc, s["H"], s["W"], s["y"], s["cs"], s["pairs"])
    if case["grads"]:
        out, dH, dW = ctx.pref_fwd_bwd(*args, ref_logp=s["ref"], dw_dtype=s["W"].dtype)
    else:
        out = ctx.pref_fwd(*args, ref_logp=s["ref"])
    got = dict(logp=out["logp"], ratio=out["ratio"], margin=out["margin"], loss=out["loss"].reshape(()))
    return dict(got, dH=dH, dW=dW) if case["grads"] else got


def _own_adamw(ctx, s):
    from paper_2602_14338_b200 import binding

    case = s["case"]
    if "plan" not in s:                 # the tensors' addresses, laid out once by a program that keeps its buffers
        first, rest, tensors = _pad(case["numel"], 256), _pad(case["small"], 256), []
        for i in range(case["count"]):
            at, n = (0, case["numel"]) if i == 0 else (first + (i - 1) * rest, case["small"])
            blocks = slice(at // 256, at // 256 + (n + 255) // 256)
            t = {name: s[name][at:at + n] for name in ("param", "grad", "master") if name in s}
            if case["bits"] == 8:
                t.update(m=s["m"].view(-1)[at:at + n], v=s["v"].view(-1)[at:at + n], m_scale=s["m_scale"][blocks],
                         v_scale=s["v_scale"][blocks])
            else:
                t.update(m=s["m"][at:at + n], v=s["v"][at:at + n])
            tensors.append(dict(t, weight_decay=DECAY if i == 0 else 0.0))
        s["plan"] = binding.AdamWPlan(tensors)
        if case["bits"] == 8:
            s["values"] = [torch.zeros(s["param"].numel(), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
            s["parts"] = [[x[t["param"].storage_offset():][:t["param"].numel()] for t in tensors] for x in s["values"]]
    ac = binding.adamw_cfg_default(lr=RATE, beta1=BETAS[0], beta2=BETAS[1], eps=EPS, max_norm=MAX_NORM)
    stats = ctx.adamw_step(ac, s["plan"], s["step"])
    out = dict(param=s["param"], norm=stats[0])
    if "master" in s:
        out["master"] = s["master"]
    if case["bits"] == 8:
        ctx.adamw_states(s["plan"], m=s["parts"][0], v=s["parts"][1])
        return dict(out, m=s["values"][0], v=s["values"][1])
    return dict(out, m=s["m"], v=s["v"])


def _fp4(s, name, rows):
    from paper_2602_14338_b200 import binding

    case = s["case"]
    return binding.Fp4Rows(rows, case["d"], case["block"], s[name], s[name + "_scale"], s[name + "_row"])


def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        return dict(pref=_plain_pref, adamw=_plain_adamw, fp4_rows=_plain_rows, fp4=_plain_product)[op](s)
    ctx = _context()
    if op == "pref":
        return _own_pref(ctx, s)
    if op == "adamw":
        return _own_adamw(ctx, s)
    if op == "fp4_rows":
        rows = ctx.quantize_fp4(_cfg(case["dtype"]), s["x"], block=case["block"])
        out = dict(value=ctx.dequantize_fp4(rows, out_dtype=torch.bfloat16))
        return out if case["block"] == 32 else dict(out, row_scale=rows.row_scale)
    return ctx.lmhead_fp4(_fp4(s, "h", case["T"]), _fp4(s, "w", case["V"]), out_dtype=_dt(case["out"]))


def work(case):
    op = case["op"]
    if op == "pref":
        T, d, V, n, e = case["T"], case["d"], case["V"], _rows_in_pairs(case), _size(case["dtype"])
        rows = e * n * d + 12 * n
        if not case["grads"]:
            return dict(bytes=e * V * d + rows, flops=2 * n * V * d)
        return dict(bytes=2 * e * V * d + rows + e * T * d, flops=6 * n * V * d)
    if op == "adamw":
        n = case["numel"] + (case["count"] - 1) * case["small"]
        each = 2 * (4 + (2 * 1 if case["bits"] == 8 else 8)) + _size(case["grad"]) + (2 if case["param"] == "bf16" else 0)
        # with 8-bit states what comes back is also the values they stand for, in two bytes each
        return dict(bytes=n * (each + (4 if case["bits"] == 8 else 0)), flops=16 * n)
    d, block = case["d"], case["block"]
    row = d / 2 + d / block + (4 if block == 16 else 0)
    if op == "fp4_rows":
        # the rows in 4 bits, and what comes back of them in two bytes each
        return dict(bytes=case["T"] * (_size(case["dtype"]) * d + row + 2 * d), flops=4 * case["T"] * d)
    T, V = case["T"], case["V"]
    return dict(bytes=(T + V) * row + T * V * _size(case["out"]), flops=2 * T * V * d)


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------------

def _exact_pref(s):
    case, f8 = s["case"], torch.float64
    T, d, V, R = case["T"], case["d"], case["V"], case["R"]
    W = s["W"].to(f8)
    cs, pairs = _rollouts(case)
    used = sorted({i for p in pairs for i in p})
    logp = torch.zeros(T, dtype=f8, device="cuda")
    ratio = torch.zeros(R, dtype=f8, device="cuda")
    scored = {i: torch.nonzero(s["y"][cs[i]:cs[i + 1]] >= 0)[:, 0] + cs[i] for i in used}
    for i in used:
        for rows in scored[i].split(512):
            lp = torch.log_softmax(s["H"][rows].to(f8) @ W.T, dim=1)
            logp[rows] = lp[torch.arange(len(rows), device="cuda"), s["y"][rows].long()]
        ratio[i] = (logp - s["ref"].to(f8))[scored[i]].sum()
        if case["mean"]:
            ratio[i] /= max(1, len(scored[i]))
    x = ratio.clone().requires_grad_()
    margin = torch.stack([BETA * (x[a] - x[b]) for a, b in pairs])
    if case["kind"] == "logistic":
        loss = -torch.log(torch.sigmoid(margin)).mean()
    elif case["kind"] == "square":
        loss = ((margin - 0.5) ** 2).mean()
    else:
        loss = torch.relu(1.0 - margin).mean()
    out = dict(logp=logp, ratio=ratio, margin=margin.detach(), loss=loss.detach())
    if case["grads"]:
        (coef,) = torch.autograd.grad(loss, x)
        dH = torch.zeros(T, d, dtype=f8, device="cuda")
        dW = torch.zeros(V, d, dtype=f8, device="cuda")
        for i in used:
            c = coef[i] / max(1, len(scored[i])) if case["mean"] else coef[i]
            for rows in scored[i].split(512):
                h = s["H"][rows].to(f8)
                dz = torch.nn.functional.one_hot(s["y"][rows].long(), V) - torch.softmax(h @ W.T, dim=1)
                dH[rows] = c * (dz @ W)
                dW += c * (dz.T @ h)
        out.update(dH=dH, dW=dW)
    return out


def _nearest(x, table):
    """x moved to the nearest value of a rising table, the one at an even place where two are as near."""
    hi = torch.searchsorted(table, x).clamp(1, len(table) - 1)
    lo = hi - 1
    below, above = x - table[lo], table[hi] - x
    return table[torch.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)]


def _exact_adamw(s):
    case, f8 = s["case"], torch.float64
    e4m3 = torch.arange(127, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).to(f8)
    e4m4 = torch.tensor([(c % 16 + 16 * (c > 15)) * 2.0 ** (max(c // 16, 1) - 11) for c in range(256)], dtype=f8, device="cuda")
    g = s["grad"].to(f8)
    norm = g.norm()
    g = g * min(1.0, float(MAX_NORM / (norm + 1e-6)))
    if case["bits"] == 8:
        m = (s["m"].to(f8) * s["m_scale"].to(f8)[:, None]).reshape(-1)
        v = ((e4m4[s["v"].long()] * s["v_scale"].to(f8)[:, None]) ** 2).reshape(-1)
    else:
        m, v = s["m"].to(f8), s["v"].to(f8)
    m = m + (1.0 - BETAS[0]) * (g - m)
    v = v + (1.0 - BETAS[1]) * (g * g - v)
    t = int(s["step"].item()) + 1
    p = (s["master"] if "master" in s else s["param"]).to(f8)
    decay = torch.ones_like(p)
    decay[:_pad(case["numel"], 256)] -= RATE * DECAY
    p = decay * p - RATE / (1.0 - BETAS[0] ** t) * m / ((v / (1.0 - BETAS[1] ** t)) ** 0.5 + EPS)
    out = dict(param=p, norm=norm)
    if "master" in s:
        out["master"] = p
    if case["bits"] == 8:
        m, r = m.view(-1, 256), v.view(-1, 256).sqrt()
        ms, rs = m.abs().amax(1, keepdim=True).clamp(min=2.0 ** -100) / 448, r.amax(1, keepdim=True).clamp(min=2.0 ** -100) / 496
        least = torch.where(r > 0, e4m4[1], e4m4[0])
        m = torch.sign(m) * _nearest((m.abs() / ms).contiguous(), e4m3) * ms
        v = (torch.maximum(_nearest((r / rs).contiguous(), e4m4), least) * rs) ** 2
    return dict(out, m=m.reshape(-1), v=v.reshape(-1))


def _exact_rows(s):
    case, f8 = s["case"], torch.float64
    block, T, d = case["block"], case["T"], case["d"]
    table = torch.tensor(E2M1, dtype=f8, device="cuda")
    value = torch.empty(T, d, dtype=f8, device="cuda")
    rows = torch.zeros(T, dtype=f8, device="cuda")
    for r in range(0, T, 16384):
        x = s["x"][r:r + 16384].to(f8).view(-1, d // block, block)
        top = x.abs().amax(2)
        if block == 32:
            unit = torch.exp2(torch.floor(torch.log2(top) + 1e-9) - 2).nan_to_num(0.0)      # (log2 of a power of two may fall short)
        else:
            e = torch.ceil(torch.log2(top.amax(1) / 2688) - 1e-9).clamp(min=-126)
            row = torch.where(top.amax(1) > 0, torch.exp2(e), torch.zeros_like(e))
            rows[r:r + 16384] = row
            e4m3 = torch.arange(127, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).to(f8)
            unit = _nearest((top / 6 / row[:, None]).nan_to_num(0.0), e4m3) * row[:, None]
        y = (x.abs() / unit[:, :, None]).nan_to_num(0.0, posinf=0.0)
        value[r:r + 16384] = (torch.sign(x) * _nearest(y.contiguous(), table) * unit[:, :, None]).view(-1, d)
    return dict(value=value) if block == 32 else dict(value=value, row_scale=rows)


def _exact_product(s):
    case, f8 = s["case"], torch.float64
    T, V, d, block = case["T"], case["V"], case["d"], case["block"]
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), dtype=f8, device="cuda")

    def rows(name, n, r0, r1):
        """Values of rows r0 .. r1 (a multiple of 128 but for the last), read from their places one column of bytes at a time."""
        rt, slabs = _pad(n, 128) // 128, _pad(d, 256) // 256
        r = torch.arange(r0, r1, device="cuda")[:, None]
        b = torch.arange(d // 2, device="cuda")[None, :]
        at = ((r // 128 * slabs + b // 128) * 128 + r % 128) * 128 + ((b % 128 // 16) ^ (r % 8)) * 16 + b % 16
        byte = s[name][at].long()
        code = torch.stack((byte % 16, byte // 16), 2).reshape(r1 - r0, d)
        k = torch.arange(d // block, device="cuda")[None, :]
        groups = slabs * 256 // (4 * block)
        where = (r // 128 * groups + k // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + k % 4
        raw = s[name + "_scale"][where]
        if block == 32:
            scale = torch.exp2(raw.to(f8) - 127)
        else:
            scale = raw.view(torch.float8_e4m3fn).to(f8) * s[name + "_row"][r0:r1, None].to(f8)
        return (table[code].view(r1 - r0, d // block, block) * scale[:, :, None]).view(r1 - r0, d)

    z = torch.empty(T, V, dtype=f8, device="cuda")
    h = rows("h", T, 0, T)
    for v0 in range(0, V, 8192):
        z[:, v0:v0 + 8192] = h @ rows("w", V, v0, min(V, v0 + 8192)).T
    return z


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "pref" and _rows_in_pairs(case) * case["V"] * case["d"] * 6 > 4e13:
        return None
    return dict(pref=_exact_pref, adamw=_exact_adamw, fp4_rows=_exact_rows, fp4=_exact_product)[case["op"]](s)

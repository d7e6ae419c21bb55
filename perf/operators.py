"""Measured cases of the operators around the lm_head: distillation from a teacher's top logits, the final RMS norm, the
tied embedding, and the lm_head product in 8-bit integers.

run() computes an operator in plain torch, or, with `own` set, through this library's calls.  Sizes are those of the
library's workloads (d = 1536, V = 151936 and d = 3584, V = 152064) and generic ones around them."""
import math

import torch

own = False

SMALL, LARGE = (1536, 151936), (3584, 152064)
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
        # evaluation of the distillation loss on a few held-out rollouts of the small policy
        dict(name="distill loss 1000", op="distill", grads=False, T=1000, R=7, K=16, lse=True, dtype="bf16", **s),
        # a micro-batch of one short rollout group, loss and gradients
        dict(name="distill step 300", op="distill", grads=True, T=300, R=4, K=64, lse=False, dtype="bf16", **s),
        # an ordinary micro-batch of the large policy, loss and gradients
        dict(name="distill step 4096", op="distill", grads=True, T=4096, R=8, K=32, lse=False, dtype="bf16", **big),
        # one token of a rollout worker: the final norm with its 8-bit output
        dict(name="norm 8 bits 1", op="norm", T=1, d=SMALL[0], residual=True, quant=True, dtype="bf16"),
        # the final norm over a training chunk of the large policy
        dict(name="norm 16384", op="norm", T=16384, d=LARGE[0], residual=True, quant=False, dtype="bf16"),
        # its gradient over an odd number of tokens of the small policy, with the gradient of the residual stream
        dict(name="norm gradient 20011", op="norm_grad", T=20011, d=SMALL[0], dsum=True, dtype="bf16"),
        # embedding of a training batch of the large policy
        dict(name="embedding 30000", op="embed", T=30000, d=LARGE[0], V=LARGE[1], dtype="bf16"),
        # its gradient for one micro-batch of the small policy
        dict(name="embedding gradient 777", op="embed_grad", T=777, d=SMALL[0], V=SMALL[1], dtype="bf16"),
        # and for a whole batch of the small policy (token ids as skewed as text is)
        dict(name="embedding gradient 204780", op="embed_grad", T=204780, d=SMALL[0], V=SMALL[1], dtype="bf16"),
        # next-token logits of one sequence
        dict(name="product 8 bits 1", op="q8", T=1, out="fp32", **big),
        # next-token logits of a batch of sequences being decoded
        dict(name="product 8 bits 61", op="q8", T=61, out="bf16", **s),
        # logits of a frozen teacher over a chunk of tokens
        dict(name="product 8 bits 2048", op="q8", T=2048, out="bf16", **big),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["distill", "distill", "norm", "norm_grad", "embed", "embed_grad", "q8", "q8"])
    if op == "distill":
        if rng.random() < 0.2:          # the plain fp32 path, for small shapes
            T = _log_int(rng, 1, 200)
            return dict(op=op, grads=rng.random() < 0.7, T=T, R=rng.randint(1, min(T, 6)), K=rng.randint(1, 24),
                        lse=rng.random() < 0.5, dtype="fp32", d=rng.randint(8, 96), V=rng.randint(100, 900))
        d, V = rng.choice([SMALL, LARGE, (64 * rng.randint(1, 64), _log_int(rng, 600, 160000))])
        T = _log_int(rng, 1, 4096)
        return dict(op=op, grads=rng.random() < 0.7, T=T, R=rng.randint(1, min(T, 12)), K=rng.choice([1, rng.randint(2, 64)]),
                    lse=rng.random() < 0.5, dtype="bf16", d=d, V=V)
    if op in ("norm", "norm_grad"):
        d = rng.choice([SMALL[0], LARGE[0], rng.randint(33, 8192)])
        T = _log_int(rng, 1, max(1, min(60000, 16384 * 3584 // d)))
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        if op == "norm":
            return dict(op=op, T=T, d=d, residual=rng.random() < 0.7, quant=rng.random() < 0.5, dtype=dtype)
        return dict(op=op, T=T, d=d, dsum=rng.random() < 0.6, dtype=dtype)
    if op in ("embed", "embed_grad"):
        d, V = rng.choice([SMALL, LARGE, (rng.randint(40, 4096), _log_int(rng, 300, 160000))])
        return dict(op=op, T=_log_int(rng, 1, 200000 * 1536 // max(d, 1536)), d=d, V=V, dtype=rng.choice(["bf16", "bf16", "fp32"]))
    d, V = rng.choice([SMALL, LARGE, (16 * rng.randint(4, 300), _log_int(rng, 200, 160000))])
    return dict(op=op, T=_log_int(rng, 1, 2048), d=d, V=V, out=rng.choice(["bf16", "fp32"]))


def _rollouts(case):
    """Token offsets and keep flags of a case's rollouts: ragged lengths, every fourth rollout dropped."""
    T, R = case["T"], case["R"]
    cs = [T * i // R + (i % 3 if 0 < i < R and T >= 8 * R else 0) for i in range(R + 1)]
    return cs, [0 if i % 4 == 3 else 1 for i in range(R)]


def _kept_rows(case):
    cs, keep = _rollouts(case)
    return sum(b - a for a, b, k in zip(cs, cs[1:], keep) if k)


def _size(dtype):
    return 4 if dtype == "fp32" else 2


def _dt(dtype):
    return torch.float32 if dtype == "fp32" else torch.bfloat16


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, std=1.0, dtype=torch.float32):
        return torch.randn(*shape, generator=g, device="cuda").mul_(std).to(dtype)

    def tokens(T, V):
        """Token ids as skewed as text: id ~ V^u, so that id v comes up about as often as 1 / v, under a fixed permutation."""
        u = torch.rand(T, generator=g, device="cuda", dtype=torch.float64)
        rank = (V ** u - 1).long().clamp_(0, V - 1)
        return torch.randperm(V, generator=g, device="cuda")[rank].int()

    op, T, d = case["op"], case["T"], case["d"]
    s = dict(case=case)
    if op == "distill":
        V, K, dt = case["V"], case["K"], _dt(case["dtype"])
        cs, keep = _rollouts(case)
        kept = max(1, _kept_rows(case))
        s["W"] = normal(V, d, std=0.02, dtype=dt)
        H = normal(T, d)
        ids = torch.randint(0, V, (T, K), generator=g, device="cuda")
        ids[:, 0] = tokens(T, V).long()
        # half of the rows lean towards the teacher's first token, as a policy close to its teacher does: its logit is
        # about log V, its probability about a half
        lean = s["W"][ids[::2, 0]].float()
        H[::2] = 0.25 * H[::2] + lean * (math.log(V) / lean.square().sum(1, keepdim=True))
        s["H"] = H.to(dt)
        a = torch.sort(normal(T, K, std=2.5), dim=1, descending=True).values + 18.0
        short = torch.randint(1, K + 1, (T, 1), generator=g, device="cuda")
        ragged = (torch.rand(T, 1, generator=g, device="cuda") < 0.1) & (torch.arange(K, device="cuda") >= short)
        s["ids"] = ids.int().masked_fill_(ragged, -1)       # a tenth of the rows have a shorter list
        s["a"] = a
        s["tlse"] = torch.logsumexp(a, dim=1) + 0.05 if case["lse"] else None
        s["cs"] = torch.tensor(cs, dtype=torch.int64, device="cuda")
        s["keep"] = torch.tensor(keep, dtype=torch.uint8, device="cuda")
        s["w"] = torch.full((case["R"],), 1.0 / kept, device="cuda") * s["keep"]
    elif op in ("norm", "norm_grad"):
        dt = _dt(case["dtype"])
        rows = torch.exp(normal(T, 1, std=0.5)) * 4.0       # residual streams grow to some multiples of one
        s["x"] = (normal(T, d) * rows).to(dt)
        s["gamma"] = (1.0 + normal(d, std=0.2)).to(dt)
        if op == "norm":
            s["residual"] = (normal(T, d) * rows).to(dt) if case["residual"] else None
        else:
            s["rstd"] = torch.rsqrt(s["x"].float().square().mean(1) + 1e-6)
            s["dh"] = normal(T, d, std=1e-3, dtype=dt)
            s["dsum"] = normal(T, d, std=1e-4, dtype=dt) if case["dsum"] else None
    elif op == "embed":
        s["W"] = normal(case["V"], d, std=0.02, dtype=_dt(case["dtype"]))
        s["y"] = tokens(T, case["V"])
    elif op == "embed_grad":
        s["dx"] = normal(T, d, std=1e-3, dtype=_dt(case["dtype"]))
        s["y"] = tokens(T, case["V"])
    else:
        V = case["V"]
        s["h8"] = normal(T, d, std=30.0).round_().clamp_(-127, 127).to(torch.int8)
        s["w8"] = normal(V, d, std=30.0).round_().clamp_(-127, 127).to(torch.int8)
        s["sh"] = torch.rand(T, generator=g, device="cuda") * 0.02 + 0.02
        s["sw"] = torch.rand(V, generator=g, device="cuda") * 5e-4 + 5e-4
    return s


def _plain_distill(s):
    H, W, ids, a = s["H"].float(), s["W"].float(), s["ids"].long(), s["a"]
    T = H.shape[0]
    owner = torch.searchsorted(s["cs"], torch.arange(T, device="cuda"), right=True) - 1
    wt = (s["w"] * s["keep"])[owner]
    kept = s["keep"][owner] != 0
    z = H @ W.T
    top = z.amax(1)
    lse = top + torch.log(torch.exp(z - top[:, None]).sum(1))
    there, at = ids >= 0, ids.clamp(min=0)
    a = torch.where(there, a, torch.full_like(a, -math.inf))
    if s["tlse"] is None:
        high = a.amax(1)
        norm = high + torch.log(torch.exp(a - high[:, None]).sum(1))
    else:
        norm = s["tlse"]
    logq = a - norm[:, None]
    q = torch.exp(logq)
    logp = z.gather(1, at) - lse[:, None]
    kl = torch.where(there, q * (logq - logp), torch.zeros_like(q)).sum(1) * kept
    out = dict(lse=lse * kept, kl=kl, loss=(wt * kl).sum())
    if s["case"]["grads"]:
        dz = torch.exp(z - lse[:, None]) * (wt * q.sum(1))[:, None]
        dz.scatter_add_(1, at, -wt[:, None] * q)
        out["dH"] = (dz @ W).to(s["H"].dtype)
        out["dW"] = (dz.T @ H).to(s["W"].dtype)
    return out


def _plain_norm(s):
    x = s["x"].float()
    if s["residual"] is not None:
        x = x + s["residual"].float()
    rstd = torch.rsqrt(x.square().mean(1) + 1e-6)
    h = x * rstd[:, None] * s["gamma"].float()
    out = dict(rstd=rstd)
    if s["residual"] is not None:
        out["sum"] = x.to(s["x"].dtype)
    if s["case"]["quant"]:
        scale = h.abs().amax(1) / 127.0
        out["scale"] = scale
        out["value"] = (torch.round(h / scale[:, None]).clamp(-127, 127) * scale[:, None]).to(torch.bfloat16)
    else:
        out["h"] = h.to(s["x"].dtype)
    return out


def _plain_norm_grad(s):
    x, dh, rstd = s["x"].float(), s["dh"].float(), s["rstd"][:, None]
    hat = x * rstd
    gdh = dh * s["gamma"].float()
    dx = rstd * (gdh - hat * (gdh * hat).mean(1, keepdim=True))
    if s["dsum"] is not None:
        dx = dx + s["dsum"].float()
    return dict(dx=dx.to(s["x"].dtype), dgamma=(dh * hat).sum(0))


def _scale(case):
    return float(case["d"]) ** 0.5


def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        if op == "distill":
            return _plain_distill(s)
        if op == "norm":
            return _plain_norm(s)
        if op == "norm_grad":
            return _plain_norm_grad(s)
        if op == "embed":
            return (s["W"][s["y"].long()].float() * _scale(case)).to(s["W"].dtype)
        if op == "embed_grad":
            dW = torch.zeros(case["V"], case["d"], device="cuda")
            return dW.index_add_(0, s["y"].long(), s["dx"].float() * _scale(case))
        z = (s["h8"].float() @ s["w8"].float().T) * s["sh"][:, None] * s["sw"]
        return z.to(_dt(case["out"]))
    ctx = _context()
    if op == "distill":
        if case["grads"]:
            out, dH, dW = ctx.distill_fwd_bwd(_cfg(case["dtype"]), s["H"], s["W"], s["ids"], s["a"], s["cs"], s["w"], s["keep"],
                                              teacher_lse=s["tlse"], dw_dtype=s["W"].dtype)
            return dict(lse=out["lse"], kl=out["kl"], loss=out["loss"].reshape(()), dH=dH, dW=dW)
        out = ctx.distill_fwd(_cfg(case["dtype"]), s["H"], s["W"], s["ids"], s["a"], s["cs"], s["w"], s["keep"],
                              teacher_lse=s["tlse"])
        return dict(lse=out["lse"], kl=out["kl"], loss=out["loss"].reshape(()))
    if op == "norm":
        out = ctx.rmsnorm_fwd(_cfg(case["dtype"]), s["x"], s["gamma"], residual=s["residual"], eps=1e-6,
                              h=not case["quant"], quant=case["quant"])
        got = dict(rstd=out["rstd"])
        if s["residual"] is not None:
            got["sum"] = out["sum"]
        if case["quant"]:
            value = torch.empty(s["x"].shape, dtype=torch.bfloat16, device="cuda")
            torch.mul(out["q"], out["q_scale"][:, None], out=value)      # the values the 8 bits stand for
            got.update(scale=out["q_scale"], value=value)
        else:
            got["h"] = out["h"]
        return got
    if op == "norm_grad":
        dx, dgamma = ctx.rmsnorm_bwd(_cfg(case["dtype"]), s["dh"], s["x"], s["gamma"], s["rstd"], dsum=s["dsum"])
        return dict(dx=dx, dgamma=dgamma)
    if op == "embed":
        return ctx.embed_fwd(_cfg(case["dtype"]), s["W"], s["y"], scale=_scale(case))
    if op == "embed_grad":
        return ctx.embed_bwd(_cfg(case["dtype"]), s["dx"], s["y"], case["V"], scale=_scale(case))
    return ctx.lmhead_q8(s["h8"], s["sh"], s["w8"], s["sw"], out_dtype=_dt(case["out"]))


def work(case):
    op, T, d = case["op"], case["T"], case["d"]
    if op == "distill":
        V, K, n, e = case["V"], case["K"], _kept_rows(case), _size(case["dtype"])
        rows = e * n * d + 8 * n * K + 8 * T + (4 * n if case["lse"] else 0)
        if not case["grads"]:
            return dict(bytes=e * V * d + rows, flops=2 * n * V * d)
        return dict(bytes=2 * e * V * d + rows + e * T * d, flops=6 * n * V * d)
    if op == "norm":
        e = _size(case["dtype"])
        rows = T * d * e * (3 if case["residual"] else 1) + T * 4 + d * e
        # with the 8-bit form what comes back is the values the 8 bits stand for, in two bytes each
        return dict(bytes=rows + (T * d * 2 + T * 4 if case["quant"] else T * d * e), flops=6 * T * d)
    if op == "norm_grad":
        e = _size(case["dtype"])
        return dict(bytes=T * d * e * (4 if case["dsum"] else 3) + T * 4 + d * (e + 4), flops=10 * T * d)
    if op == "embed":
        e = _size(case["dtype"])
        return dict(bytes=min(2 * T, T + case["V"]) * d * e + 4 * T, flops=T * d)
    if op == "embed_grad":
        return dict(bytes=T * d * _size(case["dtype"]) + 4 * case["V"] * d + 4 * T, flops=2 * T * d)
    V = case["V"]
    return dict(bytes=V * d + T * d + 4 * (T + V) + T * V * _size(case["out"]), flops=2 * T * V * d)


def exact(case, seed):
    s = prepare(case, seed)
    op, T, f8 = case["op"], case["T"], torch.float64
    if op == "distill":
        kept_rows, R = _kept_rows(case), case["R"]
        if kept_rows * case["V"] * case["d"] * 6 > 4e13:
            return None
        W = s["W"].to(f8)
        lse, kl = torch.zeros(T, dtype=f8, device="cuda"), torch.zeros(T, dtype=f8, device="cuda")
        loss = torch.zeros((), dtype=f8, device="cuda")
        dH = torch.zeros(T, case["d"], dtype=f8, device="cuda")
        dW = torch.zeros(case["V"], case["d"], dtype=f8, device="cuda")
        cs, keep = _rollouts(case)
        for i in range(R):
            for t0 in range(cs[i], cs[i + 1] if keep[i] else cs[i], 512):
                t1 = min(t0 + 512, cs[i + 1])
                h, ids, a = s["H"][t0:t1].to(f8), s["ids"][t0:t1].long(), s["a"][t0:t1].to(f8)
                logp = torch.log_softmax(h @ W.T, dim=1)
                lse[t0:t1] = torch.logsumexp(h @ W.T, dim=1)
                # the teacher's probabilities laid out over the vocabulary, one listed token at a time
                mass = torch.zeros_like(logp)
                n = s["tlse"][t0:t1].to(f8) if s["tlse"] is not None else torch.logsumexp(a.masked_fill(ids < 0, -math.inf), dim=1)
                row = torch.arange(t1 - t0, device="cuda")
                for k in range(case["K"]):
                    on = ids[:, k] >= 0
                    q = torch.exp(a[:, k] - n) * on
                    at = ids[:, k] * on
                    mass[row, at] += q
                    kl[t0:t1] += torch.where(on, q * (a[:, k] - n - logp[row, at]), torch.zeros_like(q))
                wi = s["w"][i].to(f8)
                loss = loss + wi * kl[t0:t1].sum()
                if case["grads"]:
                    dz = wi * (mass.sum(1, keepdim=True) * torch.exp(logp) - mass)
                    dH[t0:t1] = dz @ W
                    dW += dz.T @ h
        out = dict(lse=lse, kl=kl, loss=loss)
        return dict(out, dH=dH, dW=dW) if case["grads"] else out
    if op == "norm":
        x = s["x"].to(f8) + (s["residual"].to(f8) if s["residual"] is not None else 0.0)
        rms = torch.sqrt((x * x).sum(1) / case["d"] + 1e-6)
        h = x / rms[:, None] * s["gamma"].to(f8)
        out = dict(rstd=1.0 / rms)
        if s["residual"] is not None:
            out["sum"] = x
        if not case["quant"]:
            return dict(out, h=h)
        step = h.abs().max(dim=1).values / 127.0
        return dict(out, scale=step, value=torch.round(h / step[:, None]) * step[:, None])
    if op == "norm_grad":
        # the derivative of sum(dh * h) by definition of h, from the given 1 / rms
        x, r, dh = s["x"].to(f8), s["rstd"].to(f8), s["dh"].to(f8)
        inner = (dh * s["gamma"].to(f8) * x).sum(1)
        dx = dh * s["gamma"].to(f8) * r[:, None] - x * (r ** 3 * inner / case["d"])[:, None]
        if s["dsum"] is not None:
            dx = dx + s["dsum"].to(f8)
        return dict(dx=dx, dgamma=torch.einsum("td,td,t->d", dh, x, r))
    if op == "embed":
        return s["W"].to(f8).index_select(0, s["y"].long()) * _scale(case)
    if op == "embed_grad":
        order = torch.argsort(s["y"].long(), stable=True)
        ids, counts = torch.unique_consecutive(s["y"].long()[order], return_counts=True)
        dW = torch.zeros(case["V"], case["d"], dtype=f8, device="cuda")
        for c0 in range(0, case["d"], 256):
            part = torch.cumsum(s["dx"][order, c0:c0 + 256].to(f8), 0)
            ends = torch.cumsum(counts, 0) - 1
            sums = part[ends]
            sums[1:] -= part[ends[:-1]]
            dW[ids, c0:c0 + 256] = sums * _scale(case)
        return dW
    z = torch.empty(T, case["V"], dtype=f8, device="cuda")
    for v0 in range(0, case["V"], 16384):
        w = s["w8"][v0:v0 + 16384].to(f8) * s["sw"][v0:v0 + 16384, None].to(f8)
        z[:, v0:v0 + 16384] = (s["h8"].to(f8) * s["sh"][:, None].to(f8)) @ w.T
    return z

"""Cases that measure the training operators around a compressed step: the layer norm, the softmax cross
entropy of a large vocabulary, and the AdamW update.

``own`` chooses what ``run`` calls: the library's operators, or the same formulas in elementary torch operations
(32-bit arithmetic, rounded once to the output's type).  A case is a dict of plain values:

op "norm"   y = gain * (x - mean(x)) * rstd(x) + bias over rows of `dim` values; `train`: also dx, dgain, dbias
            from a given dy.  `dtype` is the type of x, y, dy, dx; `params` that of gain, bias and their gradients.
op "xent"   loss_i = log sum_v exp(h_i . w_v) - h_i . w_target(i); `train`: also dh and dw from a given dloss.
            `dtype` is the type of h and w, `grads` that of dh and dw.  A negative target takes no part.
op "adamw"  one AdamW step over `tensors` tensors, `d` values in all, that lie in one flat vector the way the
            layer blocks of the benchmark workloads do; `grads` is the type of the gradients, `bits` the width of
            the two states, `copy` asks for a 16-bit copy of the updated parameters.  With 8-bit states the pass
            also writes out the values that the states stand for, as a checkpoint does.

The 8-bit states.  Blocks of 256 consecutive values of a tensor share one fp32 scale s per state.  The first
moment is held as sign * c^2 * s, c = 0 .. 127, with s = max|m| / 127^2 over the block; of the second moment its
root is held, r = sqrt(v) = c^2 * s, c = 0 .. 255, s = max(r) / 255^2.  c is the code whose value is nearest
(ties to the smaller code), except that a positive r never gets code 0.  A block whose s would be below the
smallest normal number holds zeros.
"""
import math
import random

import torch

own = False

BLOCK = 256
LR, BETA1, BETA2, ADAM_EPS, STEP = 3e-4, 0.9, 0.999, 1e-8, 1000
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"fp32": 4, "bf16": 2}


def listed():
    return [
        # one row of a 768-wide model in 16 bits, as a single position is normalised: latency
        {"name": "norm 1x768 forward", "op": "norm", "rows": 1, "dim": 768, "dtype": "bf16", "params": "fp32", "train": False},
        # a ragged batch of odd width in fp32, the library's own type, both directions
        {"name": "norm 1001x1023 fp32", "op": "norm", "rows": 1001, "dim": 1023, "dtype": "fp32", "params": "fp32", "train": True},
        # an ordinary training batch of the 124M-parameter workload's width
        {"name": "norm 8192x768", "op": "norm", "rows": 8192, "dim": 768, "dtype": "bf16", "params": "fp32", "train": True},
        # a large batch of a wide model, everything in 16 bits
        {"name": "norm 16384x4096", "op": "norm", "rows": 16384, "dim": 4096, "dtype": "bf16", "params": "bf16", "train": True},
        # scoring a short text: the weights are read once, almost no arithmetic
        {"name": "loss 61 tokens", "op": "xent", "tokens": 61, "vocab": 50257, "dim": 768, "dtype": "bf16", "grads": "bf16", "train": False},
        # fp32 throughout at odd sizes: a small head whose gradient goes into the compressed step as it is
        {"name": "xent 513 tokens fp32", "op": "xent", "tokens": 513, "vocab": 10007, "dim": 255, "dtype": "fp32", "grads": "fp32", "train": True},
        # one worker's short batch, gradients in fp32 for the compressed step
        {"name": "xent 1000 tokens", "op": "xent", "tokens": 1000, "vocab": 50257, "dim": 768, "dtype": "bf16", "grads": "fp32", "train": True},
        # an ordinary training batch, all in 16 bits
        {"name": "xent 8192 tokens", "op": "xent", "tokens": 8192, "vocab": 50257, "dim": 768, "dtype": "bf16", "grads": "bf16", "train": True},
        # the largest head: a wide model with a large vocabulary
        {"name": "xent 4096 tokens wide", "op": "xent", "tokens": 4096, "vocab": 131072, "dim": 2048, "dtype": "bf16", "grads": "bf16", "train": True},
        # the smallest of the paper's models: one launch's latency
        {"name": "adamw 29034 in 6", "op": "adamw", "d": 29034, "tensors": 6, "grads": "fp32", "bits": 32, "copy": False},
        # the 124M-parameter workload in its 150 layer blocks, states in 32 bits, the dense message as the gradient
        {"name": "adamw 124M in 150", "op": "adamw", "d": 124_000_000, "tensors": 150, "grads": "fp32", "bits": 32, "copy": False},
        # the same with 16-bit gradients, states in 8 bits and a 16-bit copy of the weights for the next forward pass
        {"name": "adamw 124M in 150 8 bit", "op": "adamw", "d": 124_000_000, "tensors": 150, "grads": "bf16", "bits": 8, "copy": True},
    ]


def _spread(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "xent", "adamw"])
    if op == "norm":
        dim = _spread(rng, 64, 8192)
        rows = _spread(rng, 1, min(65536, 16384 * 4096 // dim))
        if rng.random() < 0.5:
            dim = -(-dim // 64) * 64
            rows = min(rows, 16384 * 4096 // dim)
        dtype = rng.choice(["fp32", "bf16"])
        if dtype == "fp32":
            rows = max(1, rows // 2)
        return {"op": "norm", "rows": rows, "dim": dim, "dtype": dtype,
                "params": rng.choice(["fp32", dtype]), "train": rng.random() < 0.7}
    if op == "xent":
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        grads = rng.choice(["fp32", dtype])
        dim, vocab = _spread(rng, 64, 2048), _spread(rng, 1000, 131072)
        if rng.random() < 0.5:
            dim = -(-dim // 64) * 64
        most = 4096 * 131072 * 2048 // (8 if dtype == "fp32" else 2)
        tokens = _spread(rng, 1, max(1, min(8192, most // (vocab * dim))))
        return {"op": "xent", "tokens": tokens, "vocab": vocab, "dim": dim, "dtype": dtype, "grads": grads,
                "train": rng.random() < 0.7}
    d = _spread(rng, 1000, 124_000_000)
    return {"op": "adamw", "d": d, "tensors": min(_spread(rng, 1, 150), max(1, d // 8)), "grads": rng.choice(["fp32", "bf16"]),
            "bits": rng.choice([8, 32]), "copy": rng.random() < 0.5}


def _sizes(d, tensors):
    """Sizes of the layer blocks: log-uniform over four decades, one value at least, `d` in all."""
    r = random.Random(1000003 * tensors + d)
    share = [math.exp(r.uniform(0, math.log(1e4))) for _ in range(tensors)]
    total, sizes = sum(share), []
    for s in share:
        sizes.append(1 + int(s / total * (d - tensors)))
    sizes[max(range(tensors), key=lambda i: sizes[i])] += d - sum(sizes)
    return sizes


def _views(flat, sizes):
    return list(torch.split(flat, sizes))


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev)

    if case["op"] == "norm":
        rows, dim, dt, pt = case["rows"], case["dim"], DTYPES[case["dtype"]], DTYPES[case["params"]]
        # activations: rows of different scale, channels with an offset, a few of them large
        x = normal(rows, dim) * (0.5 + 2 * torch.rand((rows, 1), generator=g, device=dev)) + normal(dim) * 0.5
        x[:, :: max(1, dim // 5)] *= 8.0
        state = {"x": x.to(dt), "gain": (1 + 0.1 * normal(dim)).to(pt), "bias": (0.1 * normal(dim)).to(pt), "eps": 1e-5}
        if case["train"]:
            state["dy"] = (normal(rows, dim) * 1e-2).to(dt)
        return {**case, **state}
    if case["op"] == "xent":
        tokens, vocab, dim, dt = case["tokens"], case["vocab"], case["dim"], DTYPES[case["dtype"]]
        w = normal(vocab, dim) * (1.0 / math.sqrt(dim))
        target = torch.randint(0, vocab, (tokens,), generator=g, device=dev)
        # hidden states that point towards their target by different amounts: losses from near zero to above log(vocab)
        h = normal(tokens, dim) + w[target] * (14.0 * torch.rand((tokens, 1), generator=g, device=dev))
        ignored = torch.rand((tokens,), generator=g, device=dev) < 0.06
        target = torch.where(ignored, torch.full_like(target, -100), target).to(torch.int32)
        state = {"h": h.to(dt), "w": w.to(dt), "target": target}
        if case["train"]:
            state["dloss"] = torch.where(ignored, 0.0, 1.0 / max(1, tokens)).to(torch.float32)
        return {**case, **state}
    d, sizes = case["d"], _sizes(case["d"], case["tensors"])
    r = random.Random(seed)
    scale = [math.exp(r.uniform(math.log(1e-6), math.log(1e-3))) for _ in sizes]
    p, grad, m, v = normal(d) * 0.02, normal(d), normal(d), torch.rand((d,), generator=g, device=dev)
    for gv, mv, vv, s in zip(_views(grad, sizes), _views(m, sizes), _views(v, sizes), scale):
        gv *= s
        mv *= 0.3 * s
        vv.add_(0.05).mul_(s).square_()
    grad = grad.to(DTYPES[case["grads"]])
    decay = [0.1 if n >= 1000 else 0.0 for n in sizes]
    copy = torch.zeros(d, device=dev, dtype=torch.bfloat16) if case["copy"] else None
    state = {"p": p, "grad": grad, "sizes": sizes, "decay": decay, "copy16": copy, "step": STEP}
    if own:
        from paper_2209_15203_b200 import binding
        opt = binding.AdamW(_views(p, sizes), state_bits=case["bits"], lr=LR, betas=(BETA1, BETA2), eps=ADAM_EPS,
                            weight_decay=decay, copies=_views(copy, sizes) if case["copy"] else None)
        opt.tk_adamw_set_state(_views(m, sizes), _views(v, sizes), step=STEP)
        state.update(opt=opt, views=_views(grad, sizes), m=m, v=v, mv=_views(m, sizes), vv=_views(v, sizes))
    elif case["bits"] == 8:
        held = _hold(m, v, sizes)
        state.update(held=held)
    else:
        state.update(m=m, v=v)
    return {**case, **state}


# ---- the plain form of the 8-bit states: padded to blocks, all tensors of the flat vector at once ----

def _layout(sizes, dev):
    """Where each value of the flat vector lies among the blocks, and the number of blocks."""
    n = torch.tensor(sizes, device=dev)
    blocks = (n + BLOCK - 1) // BLOCK
    first = (torch.cumsum(blocks, 0) - blocks) * BLOCK
    start = torch.cumsum(n, 0) - n
    place = torch.arange(int(sum(sizes)), device=dev) + torch.repeat_interleave(first - start, n, output_size=int(sum(sizes)))
    return place, sum(-(-k // BLOCK) for k in sizes)


def _to_codes(a, levels):
    """(codes, scales) of non-negative values a, [blocks][256]."""
    s = a.amax(1, keepdim=True) * torch.tensor(1.0 / (levels * levels), device=a.device, dtype=torch.float32)
    s = torch.where(s < 2.0 ** -126, torch.zeros_like(s), s)
    y = a * torch.where(s > 0, 1.0 / s, torch.zeros_like(s))
    k = torch.arange(levels, device=a.device, dtype=torch.float32)
    return torch.bucketize(y, k * k + k + 0.5), s


def _pack(m, v, place, blocks):
    """The held form of fp32 states: signed codes and scales of m, codes and scales of r = sqrt(v)."""
    pm, pr = (torch.zeros(blocks * BLOCK, device=m.device) for _ in range(2))
    pm[place], pr[place] = m, v.sqrt()
    pm, pr = pm.view(-1, BLOCK), pr.view(-1, BLOCK)
    cm, sm = _to_codes(pm.abs(), 127)
    cr, sr = _to_codes(pr, 255)
    cr = torch.maximum(cr, (pr > 0).to(cr.dtype) * (sr > 0))
    cm = torch.where(pm < 0, -cm, cm).to(torch.int8)
    return [cm, sm, cr.to(torch.uint8), sr]


def _unpack(held, place):
    cm, sm, cr, sr = held
    c = cm.float()
    m = (c * c.abs()) * sm
    c = cr.float()
    r = (c * c) * sr
    return m.view(-1)[place], r.view(-1)[place]


def _hold(m, v, sizes):
    place, blocks = _layout(sizes, m.device)
    return {"codes": _pack(m, v, place, blocks), "place": place, "blocks": blocks}


def _plain_adamw(s):
    p, g, sizes, dev = s["p"], s["grad"].float(), s["sizes"], s["p"].device
    s["step"] += 1
    if s["bits"] == 8:
        held = s["held"]
        m, r = _unpack(held["codes"], held["place"])
        v = r * r
    else:
        m, v = s["m"], s["v"]
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + (g * (1.0 - BETA2)) * g
    decay = torch.repeat_interleave(torch.tensor(s["decay"], device=dev), torch.tensor(sizes, device=dev), output_size=p.numel())
    step = m / (v.sqrt() * (1.0 / math.sqrt(1.0 - BETA2 ** s["step"])) + ADAM_EPS)
    new = p - LR * decay * p - (LR / (1.0 - BETA1 ** s["step"])) * step
    p.copy_(new)
    out = {"p": p}
    if s["copy16"] is not None:
        s["copy16"].copy_(p)
        out["copy16"] = s["copy16"]
    if s["bits"] == 8:
        held["codes"] = _pack(m, v, held["place"], held["blocks"])
        m, r = _unpack(held["codes"], held["place"])
        v = r * r
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    return {**out, "m": m, "v": v}


def _plain_norm(s):
    x, gain, bias = s["x"].float(), s["gain"].float(), s["bias"].float()
    mean = x.mean(1, keepdim=True)
    c = x - mean
    rstd = 1.0 / ((c * c).mean(1, keepdim=True) + s["eps"]).sqrt()
    xhat = c * rstd
    out = {"y": (xhat * gain + bias).to(s["x"].dtype)}
    if s["train"]:
        dy = s["dy"].float()
        t = dy * gain
        dx = (t - t.mean(1, keepdim=True) - xhat * (t * xhat).mean(1, keepdim=True)) * rstd
        out.update(dx=dx.to(s["x"].dtype), dgain=(dy * xhat).sum(0).to(s["gain"].dtype), dbias=dy.sum(0).to(s["gain"].dtype))
    return out


def _plain_xent(s):
    h, w, target = s["h"].float(), s["w"].float(), s["target"].long()
    logits = h @ w.t()
    top = logits.amax(1, keepdim=True)
    lse = (top + (logits - top).exp().sum(1, keepdim=True).log())
    held = target >= 0
    at = target.clamp(min=0)[:, None]
    loss = torch.where(held, (lse - logits.gather(1, at))[:, 0], 0.0)
    if not s["train"]:
        return {"loss": loss, "lse": lse[:, 0]}
    dl = (logits - lse).exp()
    dl.scatter_add_(1, at, torch.full_like(lse, -1.0))
    dl *= torch.where(held, s["dloss"], 0.0)[:, None]
    dt = DTYPES[s["grads"]]
    return {"loss": loss, "dh": (dl @ w).to(dt), "dw": (dl.t() @ h).to(dt)}


def run(state):
    s = state
    if not own:
        return {"norm": _plain_norm, "xent": _plain_xent, "adamw": _plain_adamw}[s["op"]](s)
    from paper_2209_15203_b200 import binding
    if s["op"] == "norm":
        y, mean, rstd = binding.tk_layernorm_forward(s["x"], s["gain"], s["bias"], s["eps"])
        if not s["train"]:
            return {"y": y}
        dx, dgain, dbias = binding.tk_layernorm_backward(s["dy"], s["x"], s["gain"], mean, rstd)
        return {"y": y, "dx": dx, "dgain": dgain, "dbias": dbias}
    if s["op"] == "xent":
        loss, lse = binding.tk_xent_loss(s["h"], s["w"], s["target"])
        if not s["train"]:
            return {"loss": loss, "lse": lse}
        dh, dw = binding.tk_xent_grad(s["h"], s["w"], s["target"], lse, s["dloss"], grad_dtype=DTYPES[s["grads"]])
        return {"loss": loss, "dh": dh, "dw": dw}
    s["opt"].tk_adamw_step(s["views"])
    out = {"p": s["p"]}
    if s["copy16"] is not None:
        out["copy16"] = s["copy16"]
    if s["bits"] == 8:
        s["opt"].tk_adamw_get_state(s["mv"], s["vv"])   # the values that the codes stand for
        return {**out, "m": s["m"], "v": s["v"]}
    return {**out, "m": s["opt"].m, "v": s["opt"].v}


def work(case):
    if case["op"] == "norm":
        n, e, pe = case["rows"] * case["dim"], SIZE[case["dtype"]], SIZE[case["params"]]
        if not case["train"]:
            return {"bytes": 2 * n * e + 2 * case["dim"] * pe, "flops": 8 * n}
        return {"bytes": 4 * n * e + 4 * case["dim"] * pe, "flops": 22 * n}
    if case["op"] == "xent":
        t, v, dim, e, ge = case["tokens"], case["vocab"], case["dim"], SIZE[case["dtype"]], SIZE[case["grads"]]
        if not case["train"]:
            return {"bytes": (t + v) * dim * e + 12 * t, "flops": 2 * t * v * dim}
        return {"bytes": (t + v) * dim * (e + ge) + 12 * t, "flops": 6 * t * v * dim}
    per = 8 + SIZE[case["grads"]] + (16 if case["bits"] == 32 else 4 + 16 / BLOCK + 8) + (2 if case["copy"] else 0)
    return {"bytes": case["d"] * per, "flops": 16 * case["d"]}


# ---- the definitions in 64 bits ----

def _nearest(a, levels, top):
    """The nearest of top * (c / levels)^2 to each of the values a (one block's, top its largest), by search."""
    table = top * (torch.arange(levels + 1, dtype=torch.float64, device=a.device) / levels) ** 2
    at = torch.searchsorted(table, a).clamp(1, levels)
    below, above = table[at - 1], table[at]
    return torch.where(a - below <= above - a, below, above), table[1]


def _exact_held(m, v, sizes):
    """What m and v become by being held in 8 bits, tensor by tensor in rows of 256."""
    out_m, out_v = [], []
    for a, b in zip(torch.split(m, sizes), torch.split(v, sizes)):
        n, rows = a.numel(), -(-a.numel() // BLOCK)
        pa, pr = (torch.nn.functional.pad(t, (0, rows * BLOCK - n)).view(rows, BLOCK) for t in (a, b.sqrt()))
        held = []
        for t, levels in ((pa.abs(), 127), (pr, 255)):
            top = t.amax(1, keepdim=True)
            unit = torch.where(top > 0, top, torch.ones_like(top))
            near, least = _nearest((t / unit).reshape(-1), levels, 1.0)
            if levels == 255:
                near = torch.where((t.reshape(-1) > 0) & (near == 0), least, near)
            held.append(near.view(rows, BLOCK) * top)
        out_m.append((held[0] * pa.sign()).view(-1)[:n])
        out_v.append((held[1] ** 2).view(-1)[:n])
    return torch.cat(out_m), torch.cat(out_v)


def exact(case, seed):
    s = prepare(case, seed)
    f64 = torch.float64
    if case["op"] == "norm":
        x, gain, bias = s["x"].to(f64), s["gain"].to(f64), s["bias"].to(f64)
        var, mean = torch.var_mean(x, dim=1, unbiased=False, keepdim=True)
        z = (x - mean) / torch.sqrt(var + s["eps"])
        out = {"y": torch.addcmul(bias, z, gain)}
        if case["train"]:
            dy, n = s["dy"].to(f64), x.shape[1]
            a = dy * gain
            sums = a.sum(1, keepdim=True) + z * torch.einsum("ij,ij->i", a, z)[:, None]
            out.update(dx=(n * a - sums) / (n * torch.sqrt(var + s["eps"])), dgain=torch.einsum("ij,ij->j", dy, z), dbias=dy.sum(0))
        return out
    if case["op"] == "xent":
        chunk = 1024
        h, w, target = s["h"].to(f64), s["w"].to(f64), s["target"].long()
        losses, lses, dhs, dw = [], [], [], torch.zeros_like(w)
        for i in range(0, h.shape[0], chunk):
            hc, tc = h[i:i + chunk], target[i:i + chunk]
            z = torch.einsum("td,vd->tv", hc, w)
            lse = torch.logsumexp(z, 1)
            keep = (tc >= 0).to(f64)
            rows = torch.arange(hc.shape[0], device=h.device)
            losses.append((lse - z[rows, tc.clamp(min=0)]) * keep)
            lses.append(lse)
            if case["train"]:
                soft = torch.softmax(z, 1)
                soft[rows, tc.clamp(min=0)] -= 1.0
                soft *= (keep * s["dloss"][i:i + chunk].to(f64))[:, None]
                dhs.append(torch.einsum("tv,vd->td", soft, w))
                dw += torch.einsum("tv,td->vd", soft, hc)
        if not case["train"]:
            return {"loss": torch.cat(losses), "lse": torch.cat(lses)}
        return {"loss": torch.cat(losses), "dh": torch.cat(dhs), "dw": dw}
    sizes = s["sizes"]
    p, g = s["p"].to(f64), s["grad"].to(f64)
    if "held" in s:  # what the states are before the step: the definition's, from the values before they were held
        raw = prepare({**case, "bits": 32}, seed)
        m, v = _exact_held(raw["m"].to(f64), raw["v"].to(f64), sizes)
    else:
        m, v = s["m"].to(f64), s["v"].to(f64)
    t = s["step"] + 1
    m = torch.lerp(g, m, BETA1)
    v = torch.lerp(g.square(), v, BETA2)
    decay = torch.cat([torch.full((n,), w, dtype=f64, device=p.device) for n, w in zip(sizes, s["decay"])])
    p = p * (1 - LR * decay) - LR * (m / (1 - BETA1 ** t)) / (torch.sqrt(v / (1 - BETA2 ** t)) + ADAM_EPS)
    out = {"p": p}
    if case["copy"]:
        out["copy16"] = p
    if case["bits"] == 8:
        m, v = _exact_held(m, v, sizes)
    return {**out, "m": m, "v": v}

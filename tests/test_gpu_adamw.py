"""tk_adamw_step and the 8-bit states against the formulas.

The moments are formed with one rounding per operation, in the order the header states, so elementary torch
operations in 32 bits give the same bits; codes and scales of the 8-bit states then agree exactly.  Parameters are
compared with the formula in 64 bits on the states the step started from: three roundings of p (3 u |p|) and about
12 roundings of the update (16 u of it), u = 2^-24; bf16 parameters add their own rounding, u16 = 2^-8.
"""
import math

import pytest
import torch

from paper_2209_15203_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U, U16 = 2.0 ** -24, 2.0 ** -8
F32, BF16 = torch.float32, torch.bfloat16
B1, B2 = 0.9, 0.999


def quantise(a, levels):
    """Values that non-negative a ([n] fp32) become, per 256: nearest c^2 s by direct comparison with every code."""
    out = torch.zeros_like(a)
    for i in range(0, a.numel(), 256):
        b = a[i:i + 256]
        s = b.max() * torch.tensor(1.0 / levels ** 2, dtype=F32, device=a.device)
        if float(s) < 2.0 ** -126:
            continue
        y = b * (1.0 / s)
        k = torch.arange(levels, dtype=F32, device=a.device)
        c = (y[:, None] > (k * k + k + 0.5)[None, :]).sum(1).float()
        if levels == 255:
            c = torch.where(b > 0, c.clamp(min=1), c)
        out[i:i + 256] = c * c * s
    return out


def hold(m, v):
    return quantise(m.abs(), 127) * m.sign(), quantise(v.sqrt(), 255) ** 2


def make(sizes, seed, pdt, gdt):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda n: torch.randn(n, generator=g, device=DEV)
    scale = [10.0 ** -(i % 5) for i in range(len(sizes))]
    params = [(r(n) * 0.02).to(pdt) for n in sizes]
    grads = [(r(n) * s * 1e-3).to(gdt) for n, s in zip(sizes, scale)]
    ms = [r(n) * s * 3e-4 for n, s in zip(sizes, scale)]
    vs = [(r(n) * s * 1e-3) ** 2 for n, s in zip(sizes, scale)]
    return params, grads, ms, vs


def check_step(opt, params, grads, before, decay, bits, copies, gs=1.0):
    """One step from the states `before` (fp32 values); the states after it."""
    old = [p.clone() for p in params]
    opt.tk_adamw_step(grads, grad_scale=gs)
    t = opt.steps
    m2, v2 = [torch.empty_like(m) for m in before[0]], [torch.empty_like(m) for m in before[0]]
    assert opt.tk_adamw_get_state(m2, v2) == t
    for i, p in enumerate(params):
        m, v, g = before[0][i], before[1][i], grads[i].float()
        if gs != 1.0:
            g = g * gs
        m, v = m * B1 + g * (1 - B1), v * B2 + (g * (1 - B2)) * g
        step = m.double() / (v.double().sqrt() / math.sqrt(1 - B2 ** t) + opt.eps) * (opt.lr / (1 - B1 ** t))
        want = old[i].double() * (1 - opt.lr * decay[i]) - step
        tol = 3 * U * old[i].double().abs() + 16 * U * step.abs() + 4 * U * want.abs()
        if p.dtype == BF16:
            tol = tol * (1 + U16) + U16 * want.abs()
        assert torch.all((p.double() - want).abs() <= tol), "tensor %d" % i
        if bits == 8:
            m, v = hold(m, v)
        assert torch.equal(m2[i], m) and torch.equal(v2[i], v), "states of tensor %d" % i
        if copies[i] is not None:
            assert torch.equal(copies[i], p.to(BF16))
    return m2, v2


SIZES = [1, 2, 31, 32, 33, 255, 256, 257, 511, 4095, 4096, 4097, 5000, 1]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("pdt", [F32, BF16])
@pytest.mark.parametrize("gdt", [F32, BF16])
def test_steps_from_states(bits, pdt, gdt):
    params, grads, ms, vs = make(SIZES, 1, pdt, gdt)
    decay = [0.1 * (i % 3) for i in range(len(SIZES))]
    copies = [torch.zeros_like(p, dtype=BF16) if i % 2 else None for i, p in enumerate(params)]
    opt = binding.AdamW(params, state_bits=bits, lr=3e-4, betas=(B1, B2), weight_decay=decay, copies=copies)
    opt.tk_adamw_set_state(ms, vs, step=41)
    before = ([m.clone() for m in ms], [v.clone() for v in vs]) if bits == 32 else tuple(zip(*[hold(m, v) for m, v in zip(ms, vs)]))
    for k in range(3):
        before = check_step(opt, params, grads, before, decay, bits, copies, gs=1.0 if k < 2 else 0.25)
    assert opt.steps == 44


@pytest.mark.parametrize("bits", [32, 8])
def test_first_steps_from_zero_states(bits):
    params, grads, ms, vs = make([300, 1000], 2, F32, F32)
    grads[0][:] = 0.0           # a tensor without gradient: only the decay moves it
    grads[1][::2] = 0.0
    opt = binding.AdamW(params, state_bits=bits, lr=1e-2, betas=(B1, B2), weight_decay=0.1)
    zero = ([torch.zeros_like(m) for m in ms], [torch.zeros_like(m) for m in ms])
    for _ in range(2):
        zero = check_step(opt, params, grads, zero, [0.1, 0.1], bits, [None, None])
    assert not zero[0][0].any() and not zero[1][0].any()


@pytest.mark.parametrize("bits", [32, 8])
def test_views_of_a_flat_vector(bits):
    # layer blocks of a flat vector: no tensor starts on a 16-byte boundary, more of them than one launch takes
    sizes = [1 + (37 * i) % 700 for i in range(1100)]
    flat, gflat = torch.randn(sum(sizes) + 1, device=DEV)[1:], torch.randn(sum(sizes) + 3, device=DEV)[3:] * 1e-3
    params, grads = list(torch.split(flat, sizes)), list(torch.split(gflat, sizes))
    one = [flat.clone()]
    opt = binding.AdamW(params, state_bits=bits, lr=1e-3, weight_decay=0.0)
    opt.tk_adamw_step(grads)
    ref = binding.AdamW(one, state_bits=32, lr=1e-3, weight_decay=0.0)
    ref.tk_adamw_step([gflat.contiguous()])
    assert torch.equal(flat, one[0])        # the first step does not see how the states are held


def test_held_values_special_cases():
    n = 256 * 6 + 40
    m, v = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    m[256:512], v[256:512] = 1e-3, 1e-6                                    # constant blocks: exact up to the scale's rounding
    m[512:768] = torch.linspace(-1, 1, 256, device=DEV)
    v[512:768] = torch.linspace(0, 1, 256, device=DEV) ** 8               # 19 decades: small ones get code 1, zero stays zero
    m[768:1024], v[768:1024] = 1e-41, 1e-44                               # m below the smallest normal number; the root of v is not
    m[1024], v[1024 + 17] = -3e38, 3e38
    m[1536:], v[1536:] = -1e-30, 1e-37
    p = torch.zeros(n, device=DEV)
    opt = binding.AdamW([p], state_bits=8)
    opt.tk_adamw_set_state([m], [v], step=5)
    gm, gv = torch.empty_like(m), torch.empty_like(v)
    assert opt.tk_adamw_get_state([gm], [gv]) == 5
    wm, wv = hold(m, v)
    assert torch.equal(gm, wm) and torch.equal(gv, wv)
    assert torch.equal(gv > 0, v > 0) and not gm[768:1024].any()
    # holding what is already held changes at most the last bits of the scale
    opt.tk_adamw_set_state([gm], [gv], step=5)
    hm, hv = torch.empty_like(m), torch.empty_like(v)
    opt.tk_adamw_get_state([hm], [hv])
    assert torch.all((hm - gm).abs() <= 4 * U * gm.abs()) and torch.all((hv - gv).abs() <= 8 * U * gv.abs())


def test_descent_on_a_quadratic():
    # the gradient of sum (p - c)^2 / 2, by the difference of the loss along a step too: 8-bit states must descend like 32-bit ones
    g = torch.Generator(device=DEV).manual_seed(4)
    c = torch.randn(5000, generator=g, device=DEV)
    left = {}
    for bits in (32, 8):
        p = torch.zeros(5000, device=DEV)
        opt = binding.AdamW([p], state_bits=bits, lr=0.05, weight_decay=0.0)
        for _ in range(200):
            opt.tk_adamw_step([p - c])
        left[bits] = float((p - c).square().mean())
    assert left[32] < 1e-2 and left[8] < 2e-2


def test_another_stream():
    params, grads, ms, vs = make([5000, 300], 6, F32, BF16)
    twin = [p.clone() for p in params]
    a, b = binding.AdamW(params, state_bits=8), binding.AdamW(twin, state_bits=8)
    a.tk_adamw_set_state(ms, vs, 3)
    s = torch.cuda.Stream()
    b.tk_adamw_set_state(ms, vs, 3, stream=s)
    a.tk_adamw_step(grads)
    b.tk_adamw_step(grads, stream=s)
    assert all(torch.equal(x, y) for x, y in zip(params, twin))

"""tk_layernorm_forward / tk_layernorm_backward against the formulas in 64 bits.

Tolerances.  u = 2^-24 (fp32), u16 = 2^-8 (bf16), both unit roundoffs.  A sum of n values held in registers is
formed by at most n / threads sequential additions and a tree of ten levels; K = 24 + n / 32 roundings bound any of
the row sums here, relative to the sum of absolute values.  An output in bf16 adds u16 of itself.
"""
import pytest
import torch

from paper_2209_15203_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U, U16 = 2.0 ** -24, 2.0 ** -8
F32, BF16 = torch.float32, torch.bfloat16


def reference(x, gain, bias, eps, dy=None):
    x, gain = x.double(), gain.double()
    n = x.shape[1]
    mean = x.mean(1, keepdim=True)
    rstd = ((x - mean).square().mean(1, keepdim=True) + eps).rsqrt()
    z = (x - mean) * rstd
    k = 24 + n / 32
    spread = (x.abs() + x.abs().mean(1, keepdim=True)) * rstd          # what z is the difference of, at z's scale
    dz = k * U * (spread + z.abs() * (1 + (spread * spread).mean(1, keepdim=True).sqrt()))
    y = z * gain + (bias.double() if bias is not None else 0)
    out = {"y": (y, dz * gain.abs() + 4 * U * (z * gain).abs() + 4 * U * y.abs()), "mean": mean[:, 0], "rstd": rstd[:, 0]}
    if dy is not None:
        dy = dy.double()
        t = dy * gain
        m1, m2 = t.mean(1, keepdim=True), (t * z).mean(1, keepdim=True)
        dx = rstd * (t - m1 - z * m2)
        ta, tz = t.abs().mean(1, keepdim=True), (t * z).abs().mean(1, keepdim=True)
        e2 = (t.abs() * dz).mean(1, keepdim=True) + k * U * tz         # error of m2
        edx = rstd * (8 * U * t.abs() + k * U * ta + dz * m2.abs() + z.abs() * e2) + (k * U * (1 + spread.amax(1, keepdim=True))) * \
            rstd * (t.abs() + ta + z.abs() * tz)
        rows = x.shape[0]
        kr = 24 + rows                                                  # sequential additions over the rows at most
        out.update(dx=(dx, edx), dgain=((dy * z).sum(0), kr * U * (dy * z).abs().sum(0) + (dy.abs() * dz).sum(0)),
                   dbias=(dy.sum(0), kr * U * dy.abs().sum(0)))
    return out


def close(got, want, what):
    ref, tol = want
    assert got.shape == ref.shape, what
    if got.dtype == BF16:
        tol = tol * (1 + U16) + U16 * ref.abs()
    err = (got.double() - ref).abs()
    bad = err > tol + 1e-38
    assert not bad.any(), "%s: %d of %d values beyond tolerance, worst %.3g times" % (
        what, int(bad.sum()), bad.numel(), float((err / (tol + 1e-38)).max()))


def run(x, gain, bias, dy, eps=1e-5, grad_dtype=None):
    y, mean, rstd = binding.tk_layernorm_forward(x, gain, bias, eps)
    ref = reference(x, gain, bias, eps, dy)
    close(y, ref["y"], "y")
    assert y.dtype == x.dtype and mean.dtype == rstd.dtype == F32
    torch.testing.assert_close(rstd.double(), ref["rstd"], rtol=1e-4, atol=0)
    got = binding.tk_layernorm_backward(dy, x, gain, mean, rstd, grad_dtype=grad_dtype)
    for name, g in zip(("dx", "dgain", "dbias"), got):
        close(g, ref[name], name)
    return y, got


def make(rows, dim, dtype, params, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed + rows * 31 + dim)
    x = (torch.randn((rows, dim), generator=g, device=DEV) * 2 + 0.5).to(dtype)
    gain = (1 + 0.2 * torch.randn(dim, generator=g, device=DEV)).to(params)
    bias = (0.1 * torch.randn(dim, generator=g, device=DEV)).to(params)
    dy = torch.randn((rows, dim), generator=g, device=DEV).to(dtype)
    return x, gain, bias, dy


# every group size of both load widths, the widths around their limits, and rows too long for registers
@pytest.mark.parametrize("dtype,params", [(F32, F32), (BF16, F32), (BF16, BF16), (F32, BF16)])
@pytest.mark.parametrize("rows,dim", [(1, 1), (3, 2), (5, 7), (1, 768), (7, 31), (9, 64), (33, 255), (40, 256), (17, 257), (64, 768),
                                      (1001, 1023), (600, 1024), (11, 1025), (5, 4096), (3, 4104), (3, 8191), (2, 16384), (2, 20000),
                                      (2, 33000), (2, 40001)])
def test_against_formula(rows, dim, dtype, params):
    run(*make(rows, dim, dtype, params))


@pytest.mark.parametrize("dim", [96, 100, 4100])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides_and_alignment(dim, dtype):
    rows = 13
    for pad, offset in ((0, 0), (8, 0), (3, 1), (8, 5)):
        x, gain, bias, dy = make(rows, dim, dtype, F32, seed=pad + offset)
        store = torch.full((rows, dim + pad + offset + 8), float("nan"), dtype=dtype, device=DEV)
        xs = store[:, offset:offset + dim]
        xs.copy_(x)
        ds = torch.full((rows * 2, dim + 1), float("nan"), dtype=dtype, device=DEV)[::2, :dim]
        ds.copy_(dy)
        run(xs, gain, bias, ds)      # by single values
        run(x, gain, bias, dy)       # by 16 bytes where the width allows


def test_many_rows_and_gradients_into_a_row():
    x, gain, bias, dy = make(20_000, 384, BF16, F32)
    ref = reference(x, gain, bias, 1e-5, dy)
    y, mean, rstd = binding.tk_layernorm_forward(x, gain, bias)
    row = torch.full((1 + 3 * 384,), 7.0, device=DEV)      # a gradient row: slices start off the 16-byte grid
    _, a, b = binding.tk_layernorm_backward(dy, x, gain, mean, rstd, dgain=row[1:385], dbias=row[385:769])
    close(row[1:385], ref["dgain"], "dgain")
    close(row[385:769], ref["dbias"], "dbias")
    assert row[0] == 7.0 and torch.all(row[769:] == 7.0)
    again = binding.tk_layernorm_backward(dy, x, gain, mean, rstd)
    assert torch.equal(again[1], row[1:385]) and torch.equal(again[2], row[385:769])   # the same bits every time


def test_no_bias_partial_needs_and_empty():
    x, gain, bias, dy = make(6, 40, F32, F32)
    y, mean, rstd = binding.tk_layernorm_forward(x, gain, None)
    close(y, reference(x, gain, None, 1e-5)["y"], "y")
    dx, a, b = binding.tk_layernorm_backward(dy, x, gain, mean, rstd, need_params=False)
    assert a is None and b is None
    dx2, a, b = binding.tk_layernorm_backward(dy, x, gain, mean, rstd, need_dx=False)
    assert dx2 is None
    full = binding.tk_layernorm_backward(dy, x, gain, mean, rstd)
    assert torch.equal(full[0], dx) and torch.equal(full[1], a) and torch.equal(full[2], b)
    e = x[:0]
    y, mean, rstd = binding.tk_layernorm_forward(e, gain, bias)
    assert y.shape == (0, 40)
    dx, a, b = binding.tk_layernorm_backward(e, e, gain, mean, rstd)
    assert dx.shape == (0, 40) and not a.any() and not b.any()


def test_constant_rows_and_large_offsets():
    # variance zero: z = 0, y = bias; a mean of 1000 times the spread must not cancel the spread away
    dim = 512
    x = torch.full((4, dim), 3.25, device=DEV)
    gain, bias = torch.ones(dim, device=DEV), torch.arange(dim, device=DEV, dtype=F32)
    y, mean, rstd = binding.tk_layernorm_forward(x, gain, bias)
    assert torch.equal(y, bias.expand(4, dim)) and torch.all(mean == 3.25)
    x = torch.randn((64, dim), device=DEV, generator=torch.Generator(device=DEV).manual_seed(3)) + 1000.0
    run(x, gain, bias, torch.randn_like(x))
    # infinities and NaN stay in their own row
    x = torch.randn((3, dim), device=DEV)
    clean = binding.tk_layernorm_forward(x, gain, bias)[0]
    x[1, 7] = float("inf")
    y = binding.tk_layernorm_forward(x, gain, bias)[0]
    assert torch.equal(y[0], clean[0]) and torch.equal(y[2], clean[2]) and torch.isnan(y[1]).any()


def test_gradient_against_differences():
    # L = sum c * y for a fixed c.  Central differences of step e along d have error e^2 L''' / 6 and rounding L_err / e;
    # with 64-bit evaluation of the formula replaced by the kernel's fp32 y, L_err <= sum |c| tol(y).
    x, gain, bias, c = make(8, 120, F32, F32, seed=9)
    _, mean, rstd = binding.tk_layernorm_forward(x, gain, bias)
    grads = binding.tk_layernorm_backward(c, x, gain, mean, rstd)

    def value(x, gain, bias):
        return float((binding.tk_layernorm_forward(x, gain, bias)[0].double() * c.double()).sum())

    err = float((reference(x, gain, bias, 1e-5)["y"][1] * c.double().abs()).sum())
    e = 2.0 ** -6
    for at, g in zip((0, 1, 2), grads):
        for seed in range(3):
            args = [x, gain, bias]
            d = torch.randn(args[at].shape, device=DEV, generator=torch.Generator(device=DEV).manual_seed(seed)).sign() / 8
            plus, minus = list(args), list(args)
            plus[at], minus[at] = args[at] + e * d, args[at] - e * d
            numeric = (value(*plus) - value(*minus)) / (2 * e)
            exact = float((g.double() * d.double()).sum())
            # third derivative along d: bounded by 6 * rstd^3 |d|^3 times the size of y and c
            third = 6 * float(rstd.max()) ** 3 * (1 / 8) ** 3 * float(c.double().abs().sum()) * 4
            # x +- e d is rounded to fp32: a move of u |x| per value, felt through the gradient
            moved = float((g.double().abs() * args[at].double().abs()).sum()) * U / e
            assert abs(numeric - exact) <= err / e + e * e / 6 * third + moved, (at, seed, numeric, exact)


def test_another_stream():
    x, gain, bias, dy = make(500, 768, BF16, F32)
    want = run(x, gain, bias, dy)
    s = torch.cuda.Stream()
    y, mean, rstd = binding.tk_layernorm_forward(x, gain, bias, stream=s)
    got = binding.tk_layernorm_backward(dy, x, gain, mean, rstd, stream=s)
    assert torch.equal(y, want[0]) and all(torch.equal(a, b) for a, b in zip(got, want[1]))

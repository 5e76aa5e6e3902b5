"""tk_xent_loss / tk_xent_grad against the definition in 64 bits.

Tolerances.  u = 2^-24, u16 = 2^-8.  The matrix instructions add 16 products at a time to an fp32 accumulator; allowing one
truncation (2 u) per 16 products and part pair, a logit is off by at most eps_l = 2 u (pairs * dim / 16 + 8) * sum_d |h w| (for
fp32 inputs the three part products left out are below 2^-24 of it).  Then
  lse:   max_v eps_l + (16 + vocab / 256) u on the sum, as an absolute error, + 2 u |lse|
  P:     relative eps_l(v) + err(lse) + 8 u, the exponent being formed in fp32: + 4 u (|l| + |lse|)
  D:     |dloss| (P err_P), and u16 of |D| when the gradients are bf16 (2^-24 when three parts hold it)
  dh, dw: sum err_D |w| (|h|) + 2 u (pairs n / 16 + 8 + pieces) sum |D w| over the n terms, + u16 of the result when it is bf16.
"""
import pytest
import torch

from paper_2209_15203_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U, U16 = 2.0 ** -24, 2.0 ** -8
F32, BF16 = torch.float32, torch.bfloat16


def make(tokens, vocab, dim, dtype, seed=0, ignored=0.2, boost=8.0):
    g = torch.Generator(device=DEV).manual_seed(seed + 7 * tokens + 3 * vocab + dim)
    w = torch.randn((vocab, dim), generator=g, device=DEV) / dim ** 0.5
    target = torch.randint(0, vocab, (tokens,), generator=g, device=DEV)
    h = torch.randn((tokens, dim), generator=g, device=DEV) + w[target] * boost * torch.rand((tokens, 1), generator=g, device=DEV)
    dloss = torch.randn(tokens, generator=g, device=DEV)
    target[torch.rand(tokens, generator=g, device=DEV) < ignored] = -100
    return h.to(dtype), w.to(dtype), target.to(torch.int32), dloss


def reference(h, w, target, dloss, gdt, pieces=1):
    wide = h.dtype == F32
    pairs, gpairs = (6, 6) if wide else (1, 3 if gdt == F32 else 1)
    h, w, g = h.double(), w.double(), dloss.double()
    tokens, dim = h.shape
    vocab = w.shape[0]
    l = h @ w.t()
    el = 2 * U * (pairs * dim / 16 + 8) * (h.abs() @ w.abs().t())
    lse = torch.logsumexp(l, 1)
    elx = el.amax(1) + (16 + vocab / 256) * U + 2 * U * lse.abs()
    held = target >= 0
    at = target.long().clamp(min=0)
    rows = torch.arange(tokens, device=h.device)
    loss = torch.where(held, lse - l[rows, at], 0.0)
    eloss = torch.where(held, elx + el[rows, at] + 2 * U * loss.abs(), 0.0)
    p = (l - lse[:, None]).exp()
    ep = p * (el + elx[:, None] + 8 * U + 4 * U * (l.abs() + lse.abs()[:, None]))
    d = p.clone()
    d[rows, at] -= 1
    g = torch.where(held, g, 0.0)[:, None]
    ed = ep * g.abs()
    d = d * g
    ed = ed + (U16 if gdt == BF16 else U) * d.abs()
    out = {"loss": (loss, eloss), "lse": (lse, elx)}
    for name, a, ea, b in (("dh", d, ed, w), ("dw", d.t(), ed.t(), h)):
        n = a.shape[1]
        ref = a @ b
        tol = ea @ b.abs() + 2 * U * (gpairs * n / 16 + 8 + pieces) * (a.abs() @ b.abs())
        if gdt == BF16:
            tol = tol * (1 + U16) + U16 * ref.abs()
        out[name] = (ref, tol)
    return out


def close(got, want, what):
    ref, tol = want
    assert got.shape == ref.shape, what
    err = (got.double() - ref).abs()
    bad = ~(err <= tol + 1e-37)
    assert not bad.any(), "%s: %d of %d values beyond tolerance, worst %.3g times, first at %s" % (
        what, int(bad.sum()), bad.numel(), float((err / (tol + 1e-37)).nan_to_num(1e9).max()), bad.nonzero()[0].tolist())


def run(h, w, target, dloss, gdt, pieces=1):
    ref = reference(h, w, target, dloss, gdt, pieces)
    loss, lse = binding.tk_xent_loss(h, w, target)
    close(lse, ref["lse"], "lse")
    close(loss, ref["loss"], "loss")
    dh, dw = binding.tk_xent_grad(h, w, target, lse, dloss, grad_dtype=gdt)
    assert dh.dtype == dw.dtype == gdt
    close(dh, ref["dh"], "dh")
    close(dw, ref["dw"], "dw")
    assert binding.tk_xent_status() == 0
    return loss, lse, dh, dw


TYPES = [(BF16, BF16), (BF16, F32), (F32, F32)]


@pytest.mark.parametrize("dt,gdt", TYPES)
@pytest.mark.parametrize("tokens,vocab,dim", [(1, 1, 1), (1, 2, 8), (1, 5001, 768), (2, 255, 63), (5, 256, 64), (31, 257, 65), (127, 1000, 7),
                                              (128, 1000, 256), (129, 513, 255), (300, 777, 520), (257, 2049, 264), (64, 50257, 96)])
def test_against_definition(tokens, vocab, dim, dt, gdt):
    run(*make(tokens, vocab, dim, dt), gdt)


@pytest.mark.parametrize("dt,gdt", TYPES)
def test_more_tiles_than_multiprocessors(dt, gdt):
    run(*make(1500, 9000, 128, dt), gdt)


# results 1, 3, 5, 9 and 17 tiles wide: teams of different sizes, tiles cut by the ends of their stretches
@pytest.mark.parametrize("dt,gdt", TYPES)
@pytest.mark.parametrize("tokens,vocab,dim", [(2000, 700, 100), (90, 30_000, 600), (700, 3000, 1290), (300, 5000, 2310), (200, 600, 4200)])
def test_cut_tiles(tokens, vocab, dim, dt, gdt):
    run(*make(tokens, vocab, dim, dt), gdt)


@pytest.mark.parametrize("gdt", [BF16, F32])
def test_several_pieces(gdt):
    # more columns than one piece of the workspace holds; the last piece ends inside a tile
    tokens, vocab, dim = 4100, 70_001, 40
    run(*make(tokens, vocab, dim, BF16), gdt, pieces=8)


@pytest.mark.parametrize("dt,gdt", TYPES)
def test_strides_and_alignment(dt, gdt):
    tokens, vocab, dim = 70, 600, 72
    h, w, target, dloss = make(tokens, vocab, dim, dt)
    ref = reference(h, w, target, dloss, gdt)
    for pad, offset in ((8, 0), (1, 0), (8, 3)):
        hs = torch.full((tokens, dim + pad + offset), float("nan"), dtype=dt, device=DEV)[:, offset:offset + dim]
        ws = torch.full((vocab, dim + pad + offset), float("nan"), dtype=dt, device=DEV)[:, offset:offset + dim]
        hs.copy_(h)
        ws.copy_(w)
        loss, lse = binding.tk_xent_loss(hs, ws, target)
        close(loss, ref["loss"], "loss")
        dh = torch.full((tokens, dim + 5), 9.0, dtype=gdt, device=DEV)
        row = torch.full((vocab * dim + 3,), 9.0, dtype=gdt, device=DEV)         # a gradient row, off the 16-byte grid
        binding.tk_xent_grad(hs, ws, target, lse, dloss, dh=dh[:, 1:1 + dim], dw=row[1:-2].view(vocab, dim))
        close(dh[:, 1:1 + dim], ref["dh"], "dh")
        close(row[1:-2].view(vocab, dim), ref["dw"], "dw")
        assert torch.all(dh[:, 0] == 9) and torch.all(dh[:, 1 + dim:] == 9) and row[0] == 9 and torch.all(row[-2:] == 9)


@pytest.mark.parametrize("dt,gdt", TYPES)
def test_one_gradient_at_a_time(dt, gdt):
    h, w, target, dloss = make(150, 700, 100, dt)
    loss, lse, dh, dw = run(h, w, target, dloss, gdt)
    a, none = binding.tk_xent_grad(h, w, target, lse, dloss, grad_dtype=gdt, need_dw=False)
    assert none is None and torch.equal(a, dh)
    none, b = binding.tk_xent_grad(h, w, target, lse, dloss, grad_dtype=gdt, need_dh=False)
    assert none is None and torch.equal(b, dw)
    again = binding.tk_xent_grad(h, w, target, lse, dloss, grad_dtype=gdt)
    assert torch.equal(again[0], dh) and torch.equal(again[1], dw)                   # the same bits every time


@pytest.mark.parametrize("dt,gdt", TYPES)
def test_targets(dt, gdt):
    h, w, target, dloss = make(140, 300, 64, dt, ignored=0.0)
    target[:] = -1                                                                     # nothing takes part
    loss, lse, dh, dw = run(h, w, target, dloss, gdt)
    assert not loss.any() and not dh.any() and not dw.any()
    target[0], target[1], target[2] = 0, 299, 255                                     # first, last, last of a tile
    loss, lse, dh, dw = run(h, w, target, dloss, gdt)
    bad = target.clone()
    bad[5], bad[6] = 300, 2 ** 31 - 1                                                 # out of range: NaN loss, no gradient
    loss2, lse2 = binding.tk_xent_loss(h, w, bad)
    assert torch.isnan(loss2[5:7]).all() and torch.equal(loss2[7:], loss[7:]) and torch.equal(lse2, lse)
    dh2, dw2 = binding.tk_xent_grad(h, w, bad, lse2, dloss, grad_dtype=gdt)
    assert torch.equal(dh2, dh) and torch.equal(dw2, dw)


def test_large_logits_and_saturated_rows():
    # logits of +-300: exp underflows for all but one entry; a target far below the maximum has a loss of hundreds
    for dt in (BF16, F32):
        h, w, target, dloss = make(200, 500, 64, dt, boost=0.0)
        h, w = h * 60, w * 8
        run(h, w, target, dloss, dt)
        h[:, 1:] = 0
        w[:, 1:] = 0
        w[:, 0] = 3.0          # all logits of a row equal
        run(h, w, target, dloss, dt)


def test_empty():
    h, w, target, dloss = make(4, 50, 16, BF16)
    loss, lse = binding.tk_xent_loss(h[:0], w, target[:0])
    assert loss.shape == (0,)
    dh, dw = binding.tk_xent_grad(h[:0], w, target[:0], lse, dloss[:0])
    assert dh.shape == (0, 16) and not dw.any()


def test_gradient_against_differences():
    # L = sum dloss_i loss_i along a direction d of h and of w, central differences of step e: error e^2 L''' / 6 (the third
    # derivative of log sum exp along d is at most 6 max|d l|^3 per row) plus the rounding of the losses / e
    h, w, target, dloss = make(40, 300, 48, F32)
    ref = reference(h, w, target, dloss, F32)
    loss, lse = binding.tk_xent_loss(h, w, target)
    dh, dw = binding.tk_xent_grad(h, w, target, lse, dloss)
    err = float((ref["loss"][1] * dloss.double().abs()).sum())
    e = 2.0 ** -5

    def value(h, w):
        return float((binding.tk_xent_loss(h, w, target)[0].double() * dloss.double()).sum())

    for seed in range(3):
        g = torch.Generator(device=DEV).manual_seed(seed)
        for which, grad in (("h", dh), ("w", dw)):
            d = torch.randn(grad.shape, device=DEV, generator=g).sign() / 8
            if which == "h":
                numeric = (value(h + e * d, w) - value(h - e * d, w)) / (2 * e)
                move = (d.double() @ w.double().t()).abs().amax(1)
            else:
                numeric = (value(h, w + e * d) - value(h, w - e * d)) / (2 * e)
                move = (h.double() @ d.double().t()).abs().amax(1)
            third = float((6 * move ** 3 * dloss.double().abs()).sum())
            x = h if which == "h" else w
            moved = float((grad.double().abs() * x.double().abs()).sum()) * U / e
            exact = float((grad.double() * d.double()).sum())
            assert abs(numeric - exact) <= 2 * err / e + e * e / 6 * third + moved


def test_another_stream_and_graph():
    h, w, target, dloss = make(300, 2000, 128, BF16)
    want = run(h, w, target, dloss, BF16)
    s = torch.cuda.Stream()
    loss, lse = binding.tk_xent_loss(h, w, target, stream=s)
    dh, dw = binding.tk_xent_grad(h, w, target, lse, dloss, stream=s)
    assert torch.equal(loss, want[0]) and torch.equal(dh, want[2]) and torch.equal(dw, want[3])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, lse = binding.tk_xent_loss(h, w, target)
        dh, dw = binding.tk_xent_grad(h, w, target, lse, dloss)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(loss, want[0]) and torch.equal(dh, want[2]) and torch.equal(dw, want[3])

"""The training operators on matrices and tensors of more than 2^31 values: their far end against the same rows by themselves."""
import pytest
import torch

from paper_2209_15203_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


def test_norm_rows_beyond_two_to_the_31():
    rows, dim = 2_200_000, 1000
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.zeros((rows, dim), dtype=BF16, device=DEV)
    x[-5:] = torch.randn((5, dim), generator=g, device=DEV).to(BF16)
    gain, bias = torch.rand(dim, generator=g, device=DEV), torch.rand(dim, generator=g, device=DEV)
    y, mean, rstd = binding.tk_layernorm_forward(x, gain, bias)
    ty, tm, tr = binding.tk_layernorm_forward(x[-5:].contiguous(), gain, bias)
    assert torch.equal(y[-5:], ty) and torch.equal(mean[-5:], tm) and torch.equal(rstd[-5:], tr)
    assert torch.equal(y[0], bias.to(BF16))                       # a constant row
    y.zero_()                                                     # dy: zero but for the last rows
    y[-5:] = ty
    dx, dgain, dbias = binding.tk_layernorm_backward(y, x, gain, mean, rstd)
    tx, tg, tb = binding.tk_layernorm_backward(ty, x[-5:].contiguous(), gain, tm, tr)
    assert torch.equal(dx[-5:], tx) and not dx[0].any()
    # five terms per column, in another order: 8 roundings of the largest
    for a, b in ((dgain, tg), (dbias, tb)):
        assert float((a - b).abs().max()) <= 8 * 2.0 ** -24 * 5 * float(ty.float().abs().max()) * 6


def test_adamw_tensor_beyond_two_to_the_31():
    n, start = 2 ** 31 + 777, 2 ** 31 - 512
    g = torch.Generator(device=DEV).manual_seed(2)
    p, grad = torch.zeros(n, dtype=BF16, device=DEV), torch.zeros(n, dtype=BF16, device=DEV)
    p[start:] = torch.randn(n - start, generator=g, device=DEV).to(BF16)
    grad[start:] = torch.randn(n - start, generator=g, device=DEV).to(BF16)
    tp, tg = p[start:].clone(), grad[start:].clone()
    for bits in (8, 32):
        a, b = binding.AdamW([p], state_bits=bits, lr=1e-2), binding.AdamW([tp], state_bits=bits, lr=1e-2)
        for _ in range(2):
            a.tk_adamw_step([grad])
            b.tk_adamw_step([tg])
        assert torch.equal(p[start:], tp) and not p[:1000].any()
        if bits == 32:
            assert torch.equal(a.m[start:], b.m) and torch.equal(a.v[start:], b.v)
        del a, b


def test_head_rows_beyond_two_to_the_31():
    tokens, vocab, dim = 8, 2_200_000, 1000
    g = torch.Generator(device=DEV).manual_seed(3)
    w = torch.empty((vocab, dim), dtype=BF16, device=DEV)
    for i in range(0, vocab, 100_000):
        w[i:i + 100_000] = torch.randn((100_000, dim), generator=g, device=DEV).to(BF16) * 0.03
    h = torch.randn((tokens, dim), generator=g, device=DEV).to(BF16)
    target = torch.tensor([vocab - 1, 0, vocab - 300, 5, -1, vocab - 2, 7, 2_100_000], dtype=torch.int32, device=DEV)
    logits = torch.cat([h.double() @ w[i:i + 200_000].double().t() for i in range(0, vocab, 200_000)], 1)
    lse_ref = torch.logsumexp(logits, 1)
    loss, lse = binding.tk_xent_loss(h, w, target)
    held = target >= 0
    ref = torch.where(held, lse_ref - logits.gather(1, target.long().clamp(min=0)[:, None])[:, 0], 0.0)
    # logits of size 1, sums of 2.2 million terms in tiles: 1e-5 is 80 roundings of the result
    assert float((lse.double() - lse_ref).abs().max()) <= 1e-5 * float(lse_ref.abs().max())
    assert float((loss.double() - ref).abs().max()) <= 1e-5 * float(ref.abs().max())
    dloss = torch.randn(tokens, generator=g, device=DEV)
    dh, dw = binding.tk_xent_grad(h, w, target, lse, dloss)
    d = (logits - lse_ref[:, None]).exp()
    d[held, target[held].long()] -= 1
    d *= torch.where(held, dloss, 0.0).double()[:, None]
    for sl in (slice(0, 400), slice(vocab - 400, vocab)):
        want = d[:, sl].t() @ h.double()
        # D and the result are rounded to bf16 (2^-8 each)
        assert torch.all((dw[sl].double() - want).abs() <= 2.0 ** -7 * (d[:, sl].abs().t() @ h.double().abs()) + 1e-30)
    want = torch.stack([sum((d[t, i:i + 200_000] @ w[i:i + 200_000].double() for i in range(0, vocab, 200_000))) for t in range(tokens)])
    size = torch.stack([sum((d[t, i:i + 200_000].abs() @ w[i:i + 200_000].double().abs() for i in range(0, vocab, 200_000))) for t in range(tokens)])
    assert torch.all((dh.double() - want).abs() <= 2.0 ** -7 * size + 2.0 ** -8 * want.abs())

"""The operators as they are used together: a head trained through the compressed step (train_head)."""
import pytest
import torch

from paper_2209_15203_b200 import binding, train_head as T

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_gradient_row_is_the_gradient_of_the_whole():
    # norm -> head -> mean loss, differentiated by torch in 64 bits.  Every value of the chain carries a few roundings of 2^-24 of
    # sums of some hundred terms of its own size: 1e-5 of the largest entry of each slice covers them.
    head, data = T.Head(96, 700, DEV), T.Data(96, 700, DEV)
    head.gain.mul_(1.5)
    head.bias.add_(0.1)
    x, target = data.batch(130)
    row = torch.full_like(head.w, float("nan"))
    loss = head.gradient(x, target, row)
    w = [p.double().clone().requires_grad_() for p in head.split(head.w)]
    y = torch.nn.functional.layer_norm(x.double(), (96,), w[0], w[1])
    ref = torch.nn.functional.cross_entropy(y @ w[2].t(), target.long(), ignore_index=-100, reduction="none")
    held = target >= 0
    ref[held].mean().backward()
    assert torch.allclose(loss.double(), ref.detach(), rtol=1e-5, atol=1e-5)
    for got, want in zip(head.split(row), w):
        assert float((got.double() - want.grad).abs().max()) <= 1e-5 * float(want.grad.abs().max())


def test_adamw_on_the_message_is_adamw_on_what_the_server_sent():
    head, data = T.Head(64, 300, DEV), T.Data(64, 300, DEV)
    d, k = head.w.numel(), 500
    ctx = binding.Context(d, 3, k, k, torch.full((3,), 1 / 3))
    ctx.tk_ef_attach()
    G = torch.empty((3, d), device=DEV)
    for q in range(3):
        head.gradient(*data.batch(100), G[q])
    message = torch.zeros(d, device=DEV)
    ctx.tk_step(message, G, -1.0, binding.TK_MODE_BIDIR | binding.TK_MODE_EF)
    idx, val = ctx.tk_last_downlink()
    dense = torch.zeros(d, device=DEV)
    dense[idx.long()] = -val
    assert torch.equal(message, dense) and int((message != 0).sum()) <= k
    twin = head.w.clone()
    a = binding.AdamW(head.split(head.w), lr=1e-2, weight_decay=0.0)
    b = binding.AdamW([twin], lr=1e-2, weight_decay=0.0)
    a.tk_adamw_step(head.split(message))
    b.tk_adamw_step([dense])
    assert torch.equal(head.w, twin)
    moved = (head.w != T.Head(64, 300, DEV).w)
    assert int(moved.sum()) <= k and int(moved.sum()) > 0
    ctx.close()


@pytest.mark.parametrize("kw", [dict(), dict(states=8), dict(update="sgd")])
def test_the_loss_falls(kw):
    losses = T.train(workers=3, tokens=200, vocab=1000, dim=64, keep=0.05, steps=40, **kw)
    assert losses[0] == pytest.approx(6.9, abs=0.3)          # log 1000
    assert losses[-1] < 0.6 * losses[0]

"""Refusals of the training operators: argument checks run on the host before any CUDA call (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2209_15203_b200 import binding

F32, BF16 = binding.TK_F32, binding.TK_BF16
P = 4096          # stands for a device address: never dereferenced by a refused call
INVALID, ALLOC = -1, -2


def norm_forward(**kw):
    a = dict(x=P, x_type=F32, rows=2, dim=8, xs=8, gain=P, bias=P, pt=F32, eps=1e-5, y=P, ys=8, mean=P, rstd=P)
    a.update(kw)
    return binding.load().tk_layernorm_forward(a["x"], a["x_type"], a["rows"], a["dim"], a["xs"], a["gain"], a["bias"], a["pt"], a["eps"],
                                               a["y"], a["ys"], a["mean"], a["rstd"], None)


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(dim=0), dict(dim=2 ** 24 + 1), dict(x_type=2), dict(pt=-1), dict(xs=7), dict(ys=7),
                                 dict(x=None), dict(x=P + 2), dict(y=P + 1), dict(gain=None), dict(bias=P + 2), dict(mean=None),
                                 dict(rstd=None), dict(mean=P + 2), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
                                 dict(x_type=BF16, x=P + 1)])
def test_norm_forward_refuses(bad):
    assert norm_forward(**bad) == INVALID


def test_norm_forward_of_no_rows_is_nothing():
    assert norm_forward(rows=0, x=None, y=None) == 0


def norm_backward(**kw):
    a = dict(dy=P, ds=8, x=P, xs=8, x_type=F32, rows=2, dim=8, gain=P, pt=F32, mean=P, rstd=P, dx=P, dxs=8, dgain=P, dbias=P, gt=F32,
             ws=P, nbytes=1 << 20)
    a.update(kw)
    return binding.load().tk_layernorm_backward(a["dy"], a["ds"], a["x"], a["xs"], a["x_type"], a["rows"], a["dim"], a["gain"], a["pt"],
                                                a["mean"], a["rstd"], a["dx"], a["dxs"], a["dgain"], a["dbias"], a["gt"], a["ws"],
                                                a["nbytes"], None)


@pytest.mark.parametrize("bad,code", [(dict(rows=-1), INVALID), (dict(dim=0), INVALID), (dict(x_type=7), INVALID), (dict(gt=3), INVALID),
                                      (dict(ds=7), INVALID), (dict(dxs=1), INVALID), (dict(dy=None), INVALID), (dict(mean=None), INVALID),
                                      (dict(gain=None), INVALID), (dict(dgain=P + 2), INVALID), (dict(dx=None, dgain=None, dbias=None), INVALID),
                                      (dict(ws=None), ALLOC), (dict(ws=P + 8), ALLOC), (dict(nbytes=100), ALLOC)])
def test_norm_backward_refuses(bad, code):
    assert norm_backward(**bad) == code


def test_workspace_sizes():
    lib = binding.load()
    assert lib.tk_layernorm_workspace_bytes(-1, 8) == 0 and lib.tk_layernorm_workspace_bytes(8, 0) == 0
    assert lib.tk_layernorm_workspace_bytes(0, 8) >= 2 * 8 * 4
    for bad in ((-1, 10, 10, BF16, BF16), (10, 0, 10, BF16, BF16), (10, 10, 0, BF16, BF16), (10, 10, 10, 2, BF16), (10, 10, 10, F32, BF16),
                (10, 10, 10, BF16, 2), (2 ** 24 + 1, 10, 10, BF16, BF16), (10, 2 ** 26 + 1, 10, BF16, BF16), (10, 10, 2 ** 20 + 1, BF16, BF16)):
        assert lib.tk_xent_workspace_bytes(*bad, 1) == 0
    size = lib.tk_xent_workspace_bytes
    t, v, d = 8192, 50257, 768
    assert size(t, v, d, BF16, -1, 1) < t * v * 2 / 10                     # the loss keeps no logits
    assert size(t, v, d, BF16, BF16, 1) < t * v * 2                        # nor does the gradient
    assert size(t, v, d, BF16, BF16, 0) >= size(t, v, d, BF16, BF16, 1) + (t + v) * d * 2
    assert size(t, v, d, F32, F32, 1) >= 3 * (t + v) * d * 2
    assert size(0, v, d, BF16, BF16, 1) > 0


def xent_loss(**kw):
    a = dict(h=P, hs=64, w=P, wst=64, it=BF16, t=4, v=100, d=64, target=P, loss=P, lse=P, ws=P, nbytes=1 << 30)
    a.update(kw)
    return binding.load().tk_xent_loss(a["h"], a["hs"], a["w"], a["wst"], a["it"], a["t"], a["v"], a["d"], a["target"], a["loss"], a["lse"],
                                       a["ws"], a["nbytes"], None)


@pytest.mark.parametrize("bad,code", [(dict(t=-1), INVALID), (dict(v=0), INVALID), (dict(d=0), INVALID), (dict(it=5), INVALID),
                                      (dict(hs=63), INVALID), (dict(wst=10), INVALID), (dict(h=None), INVALID), (dict(w=P + 1), INVALID),
                                      (dict(target=P + 2), INVALID), (dict(loss=None), INVALID), (dict(lse=P + 1), INVALID),
                                      (dict(ws=None), ALLOC), (dict(ws=P + 128), ALLOC), (dict(nbytes=16), ALLOC)])
def test_loss_refuses(bad, code):
    assert xent_loss(**bad) == code


def xent_grad(**kw):
    a = dict(h=P, hs=64, w=P, wst=64, it=BF16, t=4, v=100, d=64, target=P, lse=P, dloss=P, dh=P, dhs=64, dw=P, dws=64, gt=BF16, ws=P,
             nbytes=1 << 30)
    a.update(kw)
    return binding.load().tk_xent_grad(a["h"], a["hs"], a["w"], a["wst"], a["it"], a["t"], a["v"], a["d"], a["target"], a["lse"], a["dloss"],
                                       a["dh"], a["dhs"], a["dw"], a["dws"], a["gt"], a["ws"], a["nbytes"], None)


@pytest.mark.parametrize("bad,code", [(dict(t=-1), INVALID), (dict(gt=-1), INVALID), (dict(it=F32, gt=BF16), INVALID), (dict(dhs=63), INVALID),
                                      (dict(dws=0), INVALID), (dict(dh=None, dw=None), INVALID), (dict(dw=P + 1), INVALID),
                                      (dict(gt=F32, dh=P + 2), INVALID), (dict(dloss=None), INVALID), (dict(lse=None), INVALID),
                                      (dict(nbytes=1000), ALLOC), (dict(ws=P + 4), ALLOC)])
def test_grad_refuses(bad, code):
    assert xent_grad(**bad) == code


def adamw(tensor={}, options={}, grad=P, count=1, null=()):
    t = dict(n=10, param=P, copy16=None, m=P, v=P, scales=P, weight_decay=0.1)
    t.update(tensor)
    o = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=1.0, step=1, param_type=F32, grad_type=F32, state_bits=8)
    o.update(options)
    table = (binding.tk_adamw_tensor * 1)(binding.tk_adamw_tensor(**t))
    opts = binding.tk_adamw_options(**o)
    grads = (ctypes.c_void_p * 1)(grad)
    return binding.load().tk_adamw_step(None if "tensors" in null else table, None if "grads" in null else grads, count,
                                        None if "options" in null else ctypes.byref(opts), None)


@pytest.mark.parametrize("kw", [dict(tensor=dict(n=-1)), dict(tensor=dict(param=None)), dict(tensor=dict(param=P + 2)),
                                dict(tensor=dict(copy16=P + 1)), dict(tensor=dict(m=None)), dict(tensor=dict(v=P + 4)),
                                dict(tensor=dict(scales=None)), dict(tensor=dict(scales=P + 4)), dict(tensor=dict(weight_decay=float("nan"))),
                                dict(options=dict(lr=float("inf"))), dict(options=dict(beta1=1.0)), dict(options=dict(beta2=-0.1)),
                                dict(options=dict(eps=-1e-8)), dict(options=dict(grad_scale=float("nan"))), dict(options=dict(step=0)),
                                dict(options=dict(param_type=2)), dict(options=dict(grad_type=-1)), dict(options=dict(state_bits=16)),
                                dict(grad=None), dict(grad=P + 2), dict(count=-1), dict(null=("tensors",)), dict(null=("grads",)),
                                dict(null=("options",))])
def test_adamw_refuses(kw):
    assert adamw(**kw) == INVALID


def test_adamw_of_nothing_is_nothing():
    assert adamw(count=0, null=("tensors", "grads")) == 0
    assert adamw(tensor=dict(n=0, param=None, m=None, v=None, scales=None), grad=None) == 0


def test_binding_refuses_what_it_cannot_pass_on():
    x, gain = torch.zeros(2, 8), torch.ones(8)
    with pytest.raises(ValueError):
        binding.tk_layernorm_forward(x, gain)                                          # not on a GPU
    with pytest.raises(ValueError):
        binding.tk_layernorm_forward(x.double(), gain)
    with pytest.raises(ValueError):
        binding.tk_layernorm_forward(x, torch.ones(7))
    with pytest.raises(ValueError):
        binding.tk_layernorm_forward(x.t(), torch.ones(2))                             # rows not contiguous
    with pytest.raises(ValueError):
        binding.tk_xent_loss(x, torch.zeros(5, 8), torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError):
        binding.tk_xent_loss(x, torch.zeros(5, 9), torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        binding.AdamW([])
    with pytest.raises(ValueError):
        binding.AdamW([x], state_bits=4)
    with pytest.raises(ValueError):
        binding.AdamW([x, gain.bfloat16()])
    opt = binding.AdamW([x, gain])
    with pytest.raises(ValueError):
        opt.tk_adamw_step([torch.zeros(2, 8)])                                         # one gradient missing
    with pytest.raises(ValueError):
        opt.tk_adamw_step([torch.zeros(2, 8), torch.zeros(8)])                         # not on a GPU
    assert opt.steps == 0

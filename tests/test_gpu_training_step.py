"""examples/train.py: its step as a whole, from item ids to updated parameters."""
import os
import sys

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def trainer(**kw):
    import train
    cfg = train.small_config(16)
    t = train.Trainer(cfg, 200, **kw)
    return train, cfg, t, train.batch(cfg, 200, 0, t.model.device)


def test_loss_falls():
    """Sixteen users whose labels the model can tell: 30 steps of the same batch halve the loss (from near log 2, chance)."""
    train, cfg, t, data = trainer()
    losses = []
    for _ in range(30):
        t.step(*data)
        losses.append(float(t.loss[0]))
    assert all(np.isfinite(losses)) and losses[-1] < 0.5 * losses[0], losses


def test_step_against_autograd_and_the_formulas():
    """Layer norms' gradients against autograd on the dH and dG that the model handed back, the norm over every parameter, and the
    update of every parameter in 64 bits.  fp32 sums over up to 16 x 96 rows: 1e-5 of the gradient's size; the update as in the
    update's own tests."""
    import paper_2505_04421_amd as lg
    train, cfg, t, (ids, lens, labels) = trainer(max_norm=0.05, lr=1e-2)
    w0 = {k: v.double() for k, v in t.wv.items()}
    p0 = t.p.double()
    kept = {}
    forward_backward = lg.longer_forward_backward

    def spy(*a):                               # the gradients as they were before the norm's backward pass overwrote dH
        forward_backward(*a)
        kept["dH"], kept["dG"] = t.dH.double(), t.dG.double()

    lg.longer_forward_backward = spy
    try:
        t.step(ids, lens, labels)
    finally:
        lg.longer_forward_backward = forward_backward
    torch.cuda.synchronize()
    valid = (torch.arange(cfg.L, device=ids.device) < lens[:, None]).double()[..., None]
    items, norm_h = w0["items"].requires_grad_(), w0["norm_h"].requires_grad_()
    tokens, norm_g = w0["globals"].requires_grad_(), w0["norm_g"].requires_grad_()
    H = torch.nn.functional.layer_norm(items[ids], (cfg.d_in,), norm_h[0], norm_h[1], cfg.ln_eps) * valid
    G = torch.nn.functional.layer_norm(tokens, (cfg.d,), norm_g[0], norm_g[1], cfg.ln_eps)
    loss = (H * kept["dH"]).sum() + (G[None] * kept["dG"]).sum()
    want = dict(zip(("items", "norm_h", "globals", "norm_g"), torch.autograd.grad(loss, (items, norm_h, tokens, norm_g))))
    for k, g in want.items():
        off = (t.gv[k].double() - g).norm() / g.norm()
        assert off < 1e-5, (k, float(off))
    g = torch.cat([x.reshape(-1) for x in t.grads.tensors]).double()
    norm = float(g.norm())
    assert abs(float(t.norm[0]) - norm) < 1e-6 * norm and norm > 0.05
    c = 0.05 / norm
    assert abs(float(t.norm[1]) - c) < 1e-6 * c
    lr, b1, b2, eps = t.how
    for p, gr, w, a in zip(t.params.tensors[0], t.params.tensors[3], t.params.tensors[4], t.params.array):
        at = (p.data_ptr() - t.p.data_ptr()) // 4
        old = p0[at:at + p.numel()]
        gi = c * gr.double().reshape(-1)
        new = old - lr * (gi / (gi.abs() + eps) + a.decay * old)          # first step: m and v hold the gradient alone
        # fp32 state: 24 u of the magnitudes; where |g| is near eps or its square below fp32's range the quotient keeps its sign alone
        small = gi.abs() < 1e-15
        off = (p.double().reshape(-1) - new).abs()
        assert bool((off <= 24 * 2.0 ** -24 * (old.abs() + lr) + 1e-30)[~small].all())
        assert bool((off <= 1.01 * lr)[small].all())
        assert torch.equal(w.reshape(-1), p.reshape(-1).to(w.dtype))


def test_a_batch_that_is_not_finite_is_dropped():
    train, cfg, t, (ids, lens, labels) = trainer()
    t.step(ids, lens, labels)
    before = [x.clone() for x in (t.p, t.m, t.v, t.w)]
    bad = labels.clone()
    bad[3] = float("nan")
    t.step(ids, lens, bad)
    assert float(t.norm[1]) == 0.0
    assert all(torch.equal(a, b) for a, b in zip(before, (t.p, t.m, t.v, t.w)))

"""examples/train.py: batches whose norm is not finite are dropped and do not count as updates, so that the next update's bias correction
belongs to the moments that are there."""
import numpy as np
import pytest
import torch

from test_gpu_training_step import trainer

pytestmark = pytest.mark.gpu


def bad(labels):
    labels = labels.clone()
    labels[3] = float("nan")
    return labels


def test_the_update_after_a_dropped_batch():
    """The first batch is dropped: the second is the first update, whose moments hold its gradient alone, p = p0 - lr (g / (|g| + eps) + decay p0).
    fp32 state: 24 u of the magnitudes; gradients whose squares leave fp32 are left out."""
    _, cfg, t, (ids, lens, labels) = trainer(max_norm=0.05, lr=1e-2)
    p0 = t.p.double()
    t.step(ids, lens, bad(labels))
    assert float(t.norm[1]) == 0.0
    t.step(ids, lens, labels)
    torch.cuda.synchronize()
    c = 0.05 / float(torch.cat([x.reshape(-1) for x in t.grads.tensors]).double().norm())
    lr, _, _, eps = t.how
    moved = 0
    for p, gr, a in zip(t.params.tensors[0], t.params.tensors[3], t.params.array):
        at = (p.data_ptr() - t.p.data_ptr()) // 4
        old = p0[at:at + p.numel()]
        gi = c * gr.double().reshape(-1)
        new = old - lr * (gi / (gi.abs() + eps) + a.decay * old)
        large = gi.abs() >= 1e-15
        off = (p.double().reshape(-1) - new).abs()
        assert bool((off <= 24 * 2.0 ** -24 * (old.abs() + lr) + 1e-30)[large].all())
        moved += int(large.sum())
    assert moved > 1000


def test_the_count_of_updates():
    _, cfg, t, (ids, lens, labels) = trainer()
    for drop in (False, True, True, False, False, True):
        t.step(ids, lens, bad(labels) if drop else labels)
    assert t.updates() == 3
    assert all(np.isfinite(x.float().cpu().numpy()).all() for x in (t.p, t.m, t.v, t.w))

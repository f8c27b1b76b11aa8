"""examples/train.py with dropout and with the table's gradient and update by rows."""
import numpy as np
import pytest
import torch

import paper_2505_04421_amd as lg
from embedding_oracle import factors
from test_gpu_training_step import trainer

pytestmark = pytest.mark.gpu


def test_rows_of_the_batch_alone_against_the_whole_table():
    """Without clipping and decay the first update of the tables and norms is the same by either way, bit for bit: rows that the batch does
    not name have no gradient.  (The model's own gradients are not compared: the head's sums are taken in an order that varies.)  The global
    norms differ by the roundings of a row's norm (8 u) and of theirs."""
    got = []
    for rows in (False, True):
        _, cfg, t, (ids, lens, labels) = trainer(max_norm=float("inf"), decay=0.0, rows=rows, dropout=0.1)
        t.step(ids, lens, labels)
        torch.cuda.synchronize()
        own = t.n - sum(a * b for _, (a, b) in t.extra)
        got.append([x[own:].clone() for x in (t.p, t.m, t.v)] + [t.wv[k].clone() for k, _ in t.extra] + [float(t.norm[0])])
        if rows:
            n = int(t.order.counts[0])
            assert 0 < n < 200 and t.table_g.shape == (200, cfg.d_in)
            assert torch.equal(t.order.rows[:n].long(), torch.unique(ids[torch.arange(cfg.L, device=ids.device) < lens[:, None]]))
    for a, b in zip(got[0][:-1], got[1][:-1]):
        assert torch.equal(a, b)
    assert abs(got[0][-1] - got[1][-1]) <= 10 * 2.0 ** -24 * got[0][-1] and got[0][-1] > 0


@pytest.mark.parametrize("rows", [False, True])
def test_the_tables_gradient_with_dropout_against_autograd(rows):
    """From the dH that the model handed back through the norm and the mask of the step's number: fp32 sums over up to 16 x 96 rows of values that
    bf16 rows of E (2^-8 of them) have gone into: the norm of E's rounding error is at most 2^-8 of E's, and as a relative change of the normalised rows and
    of 1 / sigma it moves dE by a few times that: 4 * 2^-8 of the gradient's norm."""
    _, cfg, t, (ids, lens, labels) = trainer(rows=rows, dropout=0.25, max_norm=1e-3)
    w0 = {k: v.double() for k, v in t.wv.items()}
    kept, forward_backward = {}, lg.longer_forward_backward

    def spy(*a):
        forward_backward(*a)
        kept["dH"] = t.dH.double()

    lg.longer_forward_backward = spy
    try:
        t.step(ids, lens, labels)
    finally:
        lg.longer_forward_backward = forward_backward
    torch.cuda.synchronize()
    assert t.key.tolist() == [0, 1]
    f = torch.from_numpy(factors(np.arange(cfg.B * cfg.L), cfg.d_in, 0.25, 0, 1, 0)).to(ids.device).view(cfg.B, cfg.L, cfg.d_in)
    valid = (torch.arange(cfg.L, device=ids.device) < lens[:, None]).double()[..., None]
    E = (w0["items"][ids] * f * valid).requires_grad_()
    H = torch.nn.functional.layer_norm(E, (cfg.d_in,), w0["norm_h"][0], w0["norm_h"][1], cfg.ln_eps) * valid
    dE, = torch.autograd.grad((H * kept["dH"]).sum(), E)
    want = torch.zeros_like(w0["items"]).index_add_(0, ids.reshape(-1), (dE * f).reshape(-1, cfg.d_in))
    if rows:
        n = int(t.order.counts[0])
        got = torch.zeros_like(want).index_copy_(0, t.order.rows[:n].long(), t.table_g[:n].double())
    else:
        got = t.gv["items"].double()
    assert float((got - want).norm() / want.norm()) <= 4 * 2.0 ** -8
    assert float((t.row_norms.double().norm() - got.norm()).abs() / got.norm()) <= 10 * 2.0 ** -24


def test_a_batch_that_is_not_finite_is_dropped():
    _, cfg, t, (ids, lens, labels) = trainer(rows=True, dropout=0.1)
    t.step(ids, lens, labels)
    before = [x.clone() for x in (t.p, t.m, t.v, t.w)]
    bad = labels.clone()
    bad[3] = float("nan")
    t.step(ids, lens, bad)
    assert float(t.norm[1]) == 0.0 and t.updates() == 1
    assert all(torch.equal(a, b) for a, b in zip(before, (t.p, t.m, t.v, t.w)))
    t.step(ids, lens, labels)
    assert t.updates() == 2 and not torch.equal(before[0], t.p)

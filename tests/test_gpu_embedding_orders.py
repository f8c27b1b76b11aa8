"""Orders that are kept for the largest batch and table and used for smaller ones."""
import numpy as np
import pytest
import torch

import paper_2505_04421_amd as lg
from embedding_oracle import gradient, order
from test_gpu_embedding import DEV, draw_ids, on_gpu

pytestmark = pytest.mark.gpu
scratch = lambda n: torch.empty(n, dtype=torch.uint8, device=DEV)


def fill(o, ids, R):
    B, L = ids.shape
    lg.longer_sort_ids(on_gpu(ids), None, R, o, scratch(lg.longer_sort_ids_workspace_bytes(B, L, R)))


@pytest.mark.parametrize("B,L,R", [(3, 40, 1000), (7, 90, 50), (1, 1, 1)])
def test_gradients_and_update_of_a_batch_smaller_than_its_order(B, L, R):
    """grads_out and g have min(B L, the table's rows) rows, whatever the order could hold; one row less is refused."""
    d, r = 24, np.random.default_rng(B)
    o = lg.TokenOrder.empty(10, 100, 5000, DEV)
    fill(o, draw_ids(r, 10, 100, 5000), 5000)                             # the largest batch came first
    ids, n = draw_ids(r, B, L, R, missing=False), min(B * L, R)
    fill(o, ids, R)
    de = torch.randint(-3, 4, (B, L, d), device=DEV).float()
    distinct, g, _, _ = gradient(ids, None, R, de.double().cpu().numpy(), 1.0)
    assert np.array_equal(o.rows[:len(distinct)].cpu().numpy(), order(ids, None, R)[2])
    grads, ws = torch.full((n, d), -77.0, device=DEV), scratch(lg.longer_embedding_backward_workspace_bytes(B, L, d))
    lg.longer_embedding_backward(o, de, 1.0, None, False, grads, None, ws)
    assert np.array_equal(grads[:len(distinct)].double().cpu().numpy(), g) and bool((grads[len(distinct):] == -77.0).all())
    dense = torch.empty(R, d, device=DEV)
    lg.longer_embedding_backward(o, de, 1.0, None, True, dense, None, ws)
    a = [torch.rand(R, d, device=DEV) for _ in range(3)]
    b, start = [t.clone() for t in a], [t.clone() for t in a]
    how = (1e-2, 0.9, 0.99, 1e-8, 2)
    lg.longer_adamw_rows(lg.AdamWRows(*a, None, 0.1), o, grads, None, *how)
    lg.longer_adamw_step(lg.AdamWList(*[[t] for t in b], [dense], None, [0.1]), None, *how)
    hit = torch.zeros(R, dtype=torch.bool, device=DEV)
    hit[torch.from_numpy(distinct).to(DEV)] = True
    for x, y, s in zip(a, b, start):
        assert torch.equal(x[hit], y[hit]) and torch.equal(x[~hit], s[~hit])
    with pytest.raises(lg.LongerError):
        lg.longer_embedding_backward(o, de, 1.0, None, False, grads[:n - 1], None, ws)
    with pytest.raises(lg.LongerError):
        lg.longer_adamw_rows(lg.AdamWRows(*a, None, 0.1), o, grads[:n - 1], None, *how)


def test_two_graphs_that_share_an_order():
    """The order of a graph's batch, whichever batch was captured last: the update behind a replay of the larger batch takes all of its rows."""
    d, R, r = 16, 300, np.random.default_rng(3)
    o, grads = lg.TokenOrder.empty(8, 50, R, DEV), torch.zeros(R, d, device=DEV)
    p = torch.rand(R, d, device=DEV)
    start = p.clone()
    graphs = []
    for B, L in ((8, 50), (1, 5)):
        ids = on_gpu(draw_ids(r, B, L, R, missing=False))
        ws, we = scratch(lg.longer_sort_ids_workspace_bytes(B, L, R)), scratch(lg.longer_embedding_backward_workspace_bytes(B, L, d))
        de = torch.ones(B, L, d, device=DEV)

        def step():
            lg.longer_sort_ids(ids, None, R, o, ws)
            lg.longer_embedding_backward(o, de, 1.0, None, False, grads, None, we)

        step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        graphs.append((graph, torch.unique(ids), ids, ws, we, de))
    for graph, distinct, *_ in graphs + graphs:
        p.copy_(start)
        m, v = torch.zeros_like(p), torch.zeros_like(p)
        graph.replay()
        lg.longer_adamw_rows(lg.AdamWRows(p, m, v, None, 0.0), o, grads, None, 1e-2, 0.9, 0.99, 1e-8, 1)
        torch.cuda.synchronize()
        assert torch.equal((p != start).any(1).nonzero()[:, 0], distinct)


def test_an_order_never_asks_for_more_rows_than_it_holds():
    """Whatever batch it is used with: no more than its rows, and of an order that was never filled, all that it has room for."""
    i32 = lambda n: torch.zeros(n, dtype=torch.int32, device=DEV)
    o = lg.TokenOrder(i32(300), i32(300), i32(40), i32(2))
    assert o._most_rows() == 40 and o._most_rows(30) == 30 and o._most_rows(300) == 40
    fill(o, np.arange(40)[None] % 7, 1000)
    assert o.counts.tolist() == [7, 40] and o._most_rows() == 40 and o._most_rows(300) == 40
    fill(o, np.arange(300)[None] % 7, 9)
    assert o._most_rows() == 9 and o._most_rows(300) == 9 and o._most_rows(4) == 4
    with pytest.raises(lg.LongerError):
        fill(o, np.arange(300)[None] % 7, 41)
    assert o._most_rows() == 9                                            # (a refused call leaves the last batch's)

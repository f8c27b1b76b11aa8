"""Calls of the embedding's operators at the borders of their launches and layouts: more rows than the largest grid takes in one turn, rows of users side by
side, tables that are not aligned to memory lines."""
import numpy as np
import pytest
import torch

import paper_2505_04421_amd as lg
from embedding_oracle import factors, gradient, named
from test_gpu_embedding import DEV, TYPES, U, backward, draw_ids, lengths, mask, on_gpu, order, sort

pytestmark = pytest.mark.gpu


def test_lookup_and_dropout_of_more_rows_than_one_turn_of_the_grid():
    """A lookup's grid takes 2^24 rows of 1025 values in a turn, a dropout's 2^23: every value of 2^24 and some more, and the last turn's rows by the oracle."""
    d, R, L = 1025, 300, (1 << 22) + 701
    B = 4
    assert B * L > 1 << 24
    table = torch.randn(R, d, device=DEV).to(torch.bfloat16)
    torch.manual_seed(7)
    ids = torch.randint(0, R, (B, L), device=DEV, dtype=torch.int32)
    E = torch.empty(B, L, d, dtype=torch.bfloat16, device=DEV)
    lg.longer_embedding(table, ids, None, 1.0, None, E)
    rows, item = E.view(-1, d), ids.view(-1).long()
    for a in range(0, B * L, 1 << 20):
        assert torch.equal(rows[a:a + (1 << 20)], table[item[a:a + (1 << 20)]]), a
    drop, f = mask(0.5)
    lg.longer_dropout(E, None, None, drop, E)
    at = np.r_[0:3, (1 << 23) - 2:(1 << 23) + 3, (1 << 24) - 2:(1 << 24) + 3, B * L - 300:B * L]
    i = torch.from_numpy(at).to(DEV)
    want = table[item[i]].double().cpu().numpy() * f(at, d)                # (twice a bf16 number)
    assert np.array_equal(rows[i].double().cpu().numpy(), want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [5, 64, 130])
def test_users_side_by_side(d, dtype):
    """[L, B, d] tensors as [B, L, d] views: users' rows lie between one another's."""
    B, L, R, t = 6, 41, 90, TYPES[dtype]
    r = np.random.default_rng(d)
    ids = draw_ids(r, B, L, R)
    lens, glens = lengths(r, B, L, "ragged")
    gids = torch.from_numpy(ids.T.copy()).to(DEV).T
    there = torch.from_numpy(named(ids, lens, R)).to(DEV)[..., None]
    empty = lambda dt: torch.empty(L, B, d, dtype=dt, device=DEV).transpose(0, 1)
    table = torch.randint(-3, 4, (R, d), device=DEV).to(t)
    drop, f = mask(0.5)
    k = torch.from_numpy(f(np.arange(B * L), d)).to(DEV).view(B, L, d)
    E, Y = empty(t), empty(t)
    lg.longer_embedding(table, gids, glens, 1.0, drop, E)
    want = torch.where(there, table[torch.from_numpy(np.where((ids >= 0) & (ids < R), ids, 0)).to(DEV)].double() * k, 0.0)
    assert torch.equal(E.double(), want)
    lg.longer_dropout(E, E, glens, drop, Y)
    assert torch.equal(Y.double(), want + want * k)
    o = lg.TokenOrder.empty(B, L, R, DEV)
    lg.longer_sort_ids(gids, glens, R, o, torch.empty(lg.longer_sort_ids_workspace_bytes(B, L, R), dtype=torch.uint8, device=DEV))
    distinct, g, _, _ = gradient(ids, lens, R, Y.double().cpu().numpy(), 0.5, f(np.arange(B * L), d))
    grads, _, _ = backward(o, Y, 0.5, drop, False, R)
    assert np.array_equal(grads[:len(distinct)].double().cpu().numpy(), g)


@pytest.mark.parametrize("off", [1, 4, 16])
@pytest.mark.parametrize("which", ["p", "m", "v", "w", "pmvw"])
@pytest.mark.parametrize("d", [32, 128])
def test_rows_update_of_tables_off_the_memory_lines(d, which, off):
    """Rows of whole lines whose table begins inside one: the bits of longer_adamw_step on the dense gradient, nothing written beside the table."""
    B, L, R = 5, 300, 400
    r = np.random.default_rng(d + off)
    ids = draw_ids(r, B, L, R, "popular")
    o, _ = sort(ids, torch.int64, 1, None, R)
    de = torch.randn(B, L, d, device=DEV)
    compact, _, _ = backward(o, de, 1.0, None, False, R)
    dense, _, _ = backward(o, de, 1.0, None, True, R)
    distinct = torch.from_numpy(order(ids, None, R)[2]).to(DEV)
    hit = torch.zeros(R, dtype=torch.bool, device=DEV)
    hit[distinct] = True
    bufs, views = [], []
    for name, s in zip("pmvw", (0.05, 0.003, 0.01, 1.0)):
        dt = torch.bfloat16 if name == "w" else torch.float32
        a = off if name in which else 0
        buf = torch.randn(R * d + 64, device=DEV).mul_(s).abs_().to(dt)
        bufs.append((buf, buf.clone(), a))
        views.append(buf[a:a + R * d].view(R, d))
        assert (views[-1].data_ptr() % 128 == 0) == (a == 0)
    start = [t.clone() for t in views]
    other = [t.clone() for t in views]
    how = (1e-2, 0.9, 0.999, 1e-8, 3)
    lg.longer_adamw_rows(lg.AdamWRows(*views, 0.1), o, compact, None, *how)
    lg.longer_adamw_step(lg.AdamWList(*[[t] for t in other[:3]], [dense], [other[3]], [0.1]), None, *how)
    for x, y, s, (buf, before, a) in zip(views, other, start, bufs):
        assert torch.equal(x[hit], y[hit]) and torch.equal(x[~hit], s[~hit])
        assert torch.equal(buf[:a], before[:a]) and torch.equal(buf[a + R * d:], before[a + R * d:])

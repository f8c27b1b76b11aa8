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


def test_as_many_tokens_as_a_call_takes():
    """2^31 - 2^21 - 1 places: 2^28 tokens of one user name row 0, 700 row 7, three the last row, the others are padding or name no row.  All places of a user
    share one row of dE, of whole numbers: every sum is exact, in any order that adds 128 tokens of row 0 at a time.  The dense gradient has
    more shares of zeros than the workgroups that its grid has left."""
    B, d = 5, 257
    n = (1 << 31) - (1 << 21) - 1
    L, R = n // B, 16 * (1 << 15) + 1003
    assert B * L == n and (1 << 24) - 1 - -(-n // 128) == (1 << 14) - 1
    ids = torch.tensor([7, R - 1, -1, 3, 0], device=DEV)[:, None].expand(B, L)
    count = torch.tensor([700, 3, L, 0, 1 << 28], dtype=torch.int32, device=DEV)
    torch.manual_seed(1)
    base = torch.randint(-3, 4, (B, 1, d), device=DEV).float()
    de = base.to(torch.bfloat16).expand(B, L, d)
    need = [lg.longer_sort_ids_workspace_bytes(B, L, R), lg.longer_embedding_backward_workspace_bytes(B, L, d)]
    ws, o = torch.empty(max(need), dtype=torch.uint8, device=DEV), lg.TokenOrder.empty(B, L, R, DEV)
    lg.longer_sort_ids(ids, count, R, o, ws)
    valid = (1 << 28) + 703
    assert o.counts.tolist() == [3, valid] and o.rows[:3].tolist() == [0, 7, R - 1]
    assert bool((o.runs[:1 << 28] == 0).all()) and bool((o.runs[1 << 28:valid - 3] == 1).all()) and o.runs[valid - 3:valid].tolist() == [2] * 3
    assert torch.equal(o.tokens[:1 << 28], torch.arange(4 * L, 4 * L + (1 << 28), dtype=torch.int32, device=DEV))
    assert o.tokens[1 << 28:valid].tolist() == list(range(700)) + [L, L + 1, L + 2]
    want = base[[4, 0, 1], 0].double() * torch.tensor([[1 << 28], [700], [3]], device=DEV) * 0.5
    norm = want.square().sum(1).sqrt()
    for dense in (False, True):
        grads, norms = torch.full((R, d), -77.0, device=DEV), torch.full((R,), -77.0, device=DEV)
        lg.longer_embedding_backward(o, de, 0.5, None, dense, grads, norms, ws)
        at = torch.tensor([0, 7, R - 1] if dense else [0, 1, 2], device=DEV)
        assert torch.equal(grads[at].double(), want)
        assert bool(((norms[at].double() - norm).abs() <= 1.01 * U * norm).all())
        grads[at], norms[at] = (0.0 if dense else -77.0), 0.0
        assert bool((grads == (0.0 if dense else -77.0)).all()) and bool((norms == 0).all())
    del ws, o
    E, table = torch.empty(B, L, 1, dtype=torch.bfloat16, device=DEV), torch.randn(R, 1, device=DEV).to(torch.bfloat16)
    lg.longer_embedding(table, ids, count, 2.0, None, E)
    place = torch.arange(L, device=DEV)
    for b, item in enumerate((7, R - 1, None, 3, 0)):
        assert torch.equal(E[b, :, 0], torch.where(place < count[b], 0.0 if item is None else table[item, 0] * 2, 0.0).to(torch.bfloat16))
    drop, f = mask(0.5)
    E.fill_(1.0)
    lg.longer_dropout(E, None, None, drop, E)
    at = np.r_[0:4, (1 << 30) - 3:(1 << 30) + 3, n - 2000:n]
    assert np.array_equal(E.view(-1, 1)[torch.from_numpy(at).to(DEV)].double().cpu().numpy(), f(at, 1))
    del E, place
    torch.cuda.empty_cache()

"""The table's gradient on data whose sums are exact: whole numbers of at most 3 in magnitude, fewer than 2^24 / 3 of them to a sum, with the factors 1 and 2
and a scale that is a power of two.  Every order of adding them up in fp32 gives the same number, so that one lost or doubled token shows, however long its run is;
gradients are compared for equality.  A norm comes from squares that 64 bits hold and is rounded once: 1.01 u.

The shapes take every range of tokens that a group adds up, 4, 8, 16 and 32: of one turn of the kernel's two batches, and of several.  That a shape still takes
its range is checked by the workspace that the call asks for, whose size follows from it."""
import numpy as np
import pytest
import torch

import paper_2505_04421_amd as lg
from embedding_oracle import factors, named
from test_gpu_embedding import DEV, TYPES, U, backward, draw_ids, lengths, mask, sort, strided

# (users, tokens of each, width, rows of the table), tokens of a range
SHAPES = [((150, 400, 16, 30), 4), ((60, 400, 65, 9), 4), ((1, 300_000, 24, 5), 4), ((40, 800, 128, 1000), 4), ((1, 60_000, 128, 3), 4), ((2, 30_000, 600, 50), 8),
          ((1, 4503, 4099, 513), 8), ((2, 2300, 4096, 600), 8), ((1, 140_001, 128, 3000), 8), ((300, 1000, 70, 2000), 8), ((1, 2_200_003, 7, 100), 8),
          ((70, 2000, 264, 900), 16), ((90, 3000, 264, 5000), 32), ((90, 3001, 259, 40), 32), ((600, 2000, 128, 100_000), 32), ((60, 70_001, 32, 20_000), 32)]


def workspace(n, d, tokens):
    """Bytes of the gradient's workspace where a range has so many tokens."""
    up = lambda k: (k + 255) & ~255
    pieces = (d + 7) // 8
    chunks, lanes = (pieces + 63) // 64, 1
    while lanes < min(pieces, 64):
        lanes *= 2
    blocks = -(-n // (tokens * (256 // lanes)))
    shared = d > 64 and blocks > 256
    return (up(blocks * 2 * d * 4) + up(blocks * 16) + (up(n * chunks * 8) if chunks > 1 else 0)
            + (up(blocks * chunks * 4) + up(blocks * chunks * 32) if shared else 0))


@pytest.mark.parametrize("shape,tokens", SHAPES)
def test_the_shapes_take_their_ranges(shape, tokens):
    B, L, d, _ = shape
    assert [k for k in (4, 8, 16, 32) if workspace(B * L, d, k) == lg.longer_embedding_backward_workspace_bytes(B, L, d)] == [tokens]


def kept(drop, f, B, L, d):
    """The mask's factors on the GPU, by dropout of ones, and of some rows by the oracle."""
    if drop is None:
        return None
    y = torch.ones(B, L, d, dtype=torch.bfloat16, device=DEV)
    lg.longer_dropout(y, None, None, drop, y)
    some = np.unique(np.r_[0, B * L - 1, np.random.default_rng(d).integers(0, B * L, 50)])
    assert np.array_equal(y.view(-1, d)[torch.from_numpy(some).to(DEV)].double().cpu().numpy(), f(some, d))
    return y


def sums(item, terms, rows):
    """The rows' sums of whole numbers, and the items that are there: differences of sums over the sorted terms, exact in 64 bits."""
    item, by = torch.sort(item)
    distinct, count = torch.unique_consecutive(item, return_counts=True)
    total = torch.zeros(terms.shape[1], len(item) + 1, dtype=torch.float64, device=DEV)
    torch.cumsum(terms[by].t().contiguous(), 1, out=total[:, 1:])
    ends = count.cumsum(0)
    out = torch.zeros(rows, terms.shape[1], dtype=torch.float64, device=DEV)
    out[distinct] = (total[:, ends] - total[:, ends - count]).t()
    return out, distinct


@pytest.mark.gpu
@pytest.mark.parametrize("skew", ["even", "popular", "one"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape,tokens", SHAPES)
def test_exact_sums(shape, tokens, dtype, skew):
    B, L, d, R = shape
    print("  longer_embedding_backward", shape, dtype, skew, flush=True)
    t = TYPES[dtype]
    r = np.random.default_rng(B + L + d)
    torch.manual_seed(B + L + d)
    for how, pad, p, scale in (("all", 0, 0.0, 1.0), ("ragged", 3, 0.5, -0.25)):
        ids = draw_ids(r, B, L, R, skew)
        lens, glens = lengths(r, B, L, how)
        there = torch.from_numpy(named(ids, lens, R)).to(DEV)
        whole = torch.randint(-3, 4, (B, L, d), device=DEV, dtype=torch.int8)
        de, _ = strided(B, L, d, t, pad)
        de.copy_(whole)
        de.masked_fill_(~there[..., None], float("nan"))
        drop, f = mask(p) if p else (None, None)
        k = kept(drop, f, B, L, d)
        item = torch.from_numpy(ids).to(DEV)[there]
        want, distinct = sums(item, whole[there].double() if k is None else whole[there].double() * k[there].double(), R)
        want *= scale
        norm = want.square().sum(1).sqrt()
        o, _ = sort(ids, torch.int64, 1, glens, R)
        assert o.counts.tolist() == [len(distinct), len(item)]
        for dense in (False, True):
            grads, norms, _ = backward(o, de, scale, drop, dense, R)
            if not dense:
                assert bool((grads[len(distinct):] == -77.0).all()) and bool((norms[len(distinct):] == 0).all())
            g, n, w, wn = (grads, norms, want, norm) if dense else (grads[:len(distinct)], norms[:len(distinct)], want[distinct], norm[distinct])
            assert torch.equal(g.double(), w)
            assert bool(((n.double() - wn).abs() <= 1.01 * U * wn).all())

"""Plain numpy forms of the embedding's operators and of the dropout mask, in 64 bits: what the GPU tests compare against."""
import numpy as np


def philox4x32(counter, key, rounds=10):
    """Philox4x32 on arrays of four counter words and two key words (uint64 arrays that hold 32 bits)."""
    low = np.uint64(0xffffffff)
    c = [np.asarray(x, dtype=np.uint64) for x in counter]
    k = [int(x) for x in key]
    for _ in range(rounds):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xffffffff, (k[1] + 0xBB67AE85) & 0xffffffff]
    return c


def factors(rows, d, p, seed, step, site):
    """[len(rows), d]: what value c of each of these rows counts, 0 where it is dropped."""
    t = int(np.floor(65536 * p + 0.5))
    seed, step = seed % (1 << 64), step % (1 << 64)
    rows = np.asarray(rows, dtype=np.uint64)[:, None]
    block = np.arange((d + 7) // 8, dtype=np.uint64)[None, :] + np.uint64(site << 16)
    block, rows = np.broadcast_arrays(block, rows)
    words = philox4x32([block, rows, np.full_like(rows, step & 0xffffffff), np.full_like(rows, step >> 32)], (seed & 0xffffffff, seed >> 32))
    h = np.stack([x for w in words for x in (w & np.uint64(0xffff), w >> np.uint64(16))], -1).reshape(rows.shape[0], -1)[:, :d]
    return np.where(h >= t, 65536 / (65536 - t), 0.0)


def named(ids, lens, rows):
    """[B, L]: whether a token is there and names a row."""
    there = (ids >= 0) & (ids < rows)
    return there if lens is None else there & (np.arange(ids.shape[1]) < np.asarray(lens)[:, None])


def order(ids, lens, rows):
    """tokens, runs, distinct rows."""
    there = np.flatnonzero(named(ids, lens, rows))
    item = ids.reshape(-1)[there]
    by = np.argsort(item, kind="stable")
    distinct, runs = np.unique(item[by], return_inverse=True)
    return there[by], runs.reshape(-1), distinct


def gradient(ids, lens, rows, de, scale, f=None):
    """distinct rows, their gradients, and the sums of the terms' magnitudes and the numbers of terms."""
    tokens, runs, distinct = order(ids, lens, rows)
    d = de.shape[-1]
    terms = de.reshape(-1, d)[tokens].astype(np.float64) * scale
    if f is not None:
        terms = np.where(f[tokens] == 0, 0.0, terms * f[tokens])
    g, mag, count = np.zeros((len(distinct), d)), np.zeros((len(distinct), d)), np.zeros(len(distinct))
    np.add.at(g, runs, terms)
    np.add.at(mag, runs, np.abs(terms))
    np.add.at(count, runs, 1)
    return distinct, g, mag, count

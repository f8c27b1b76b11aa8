"""Refusals of the embedding's entry points, dropout and the rows' update, from the host before anything is launched (no GPU needed; the
pointers are never dereferenced), and the tests' own generator against published values."""
import ctypes

import numpy as np
import pytest

import paper_2505_04421_amd as lg
from embedding_oracle import factors, gradient, order, philox4x32
from paper_2505_04421_amd.binding import CAdamW, CAdamWTable, CDropoutMask, CIds, COrder, CRows, CTable

F32, BF16, I32, I64 = 0, 1, 0, 1
FAKE, OUT, WS = 1 << 20, 1 << 24, 1 << 28
ref = ctypes.byref


def refused(rc, word, code=-1):
    assert rc == code and word in lg.longer_last_error(), (rc, lg.longer_last_error())


def rows(at=FAKE, user=640, row=64, dtype=F32):
    return CRows(at, user, row, dtype)


def mask(p=0.1, site=0, key=FAKE):
    return CDropoutMask(p, site, key)


def table(at=FAKE * 2, n=100, stride=64, dtype=F32):
    return CTable(at, n, stride, dtype)


def ids(at=FAKE * 3, user=10, row=1, kind=I64):
    return CIds(at, user, row, kind)


def some_order(**kw):
    at = dict(tokens=FAKE, runs=FAKE * 2, rows=FAKE * 3, counts=FAKE * 4)
    at.update(kw)
    return COrder(**at)


def dropout(x=None, residual=None, lens=None, B=4, L=10, d=64, drop=True, y=None):
    drop = mask() if drop is True else drop
    return lg.load_library().longer_dropout(ref(x or rows()), None if residual is None else ref(residual), lens, B, L, d,
                                            None if drop is None else ref(drop), ref(y or rows(OUT)), None)


def lookup(t=None, i=None, lens=None, B=4, L=10, d=64, scale=1.0, drop=None, e=None):
    return lg.load_library().longer_embedding(ref(t or table()), ref(i or ids()), lens, B, L, d, scale, None if drop is None else ref(drop),
                                              ref(e or rows(OUT)), None)


def sort(i=None, lens=None, B=4, L=10, n=100, o=None, ws=WS, ws_bytes=1 << 40):
    return lg.load_library().longer_sort_ids(ref(i or ids()), lens, B, L, n, ref(o or some_order()), ws, ws_bytes, None)


def back(o=None, de=None, B=4, L=10, d=64, scale=1.0, drop=None, dense=0, n=100, grads=OUT, norms=OUT * 2, ws=WS, ws_bytes=1 << 40):
    return lg.load_library().longer_embedding_backward(ref(o or some_order()), ref(de or rows()), B, L, d, scale, None if drop is None else ref(drop),
                                                       dense, n, grads, norms, ws, ws_bytes, None)


def adamw(o=None, B=4, L=10, g=FAKE * 8, norm=None, lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, step=1, **kw):
    t = dict(p=OUT, m=OUT * 2, v=OUT * 3, w=OUT * 4, rows=100, d=64, w_dtype=BF16, decay=0.0)
    t.update(kw)
    return lg.load_library().longer_adamw_rows(ref(CAdamWTable(**t)), ref(o or some_order()), B, L, g, ref(CAdamW(lr, beta1, beta2, eps, step)), norm, None)


@pytest.mark.parametrize("call", [dropout, lookup, back])
def test_sizes(call):
    refused(call(B=0), "B=0")
    refused(call(L=-1), "L=-1")
    refused(call(B=1 << 16, L=1 << 15), "2^31")
    refused(call(d=0), "d=0")
    refused(call(d=16385), "d=16385")
    for bad in (-0.1, 1.0, float("nan"), 1 - 2.0 ** -18):
        refused(call(drop=mask(p=bad)), "p=")
    refused(call(drop=mask(site=-1)), "site=-1")
    refused(call(drop=mask(site=65536)), "site=65536")
    refused(call(drop=mask(key=None)), "key")
    refused(call(drop=mask(key=FAKE + 4)), "key")


def test_dropout():
    refused(dropout(drop=None), "drop is NULL")
    refused(dropout(x=rows(None)), "x is NULL")
    refused(dropout(x=rows(dtype=7)), "dtype 7")
    refused(dropout(x=rows(FAKE + 2)), "x is not aligned")
    refused(dropout(x=rows(row=-64)), "strides")
    refused(dropout(residual=rows(None)), "residual is NULL")
    refused(dropout(residual=rows(FAKE * 3, dtype=BF16)), "one dtype")
    refused(dropout(y=rows(OUT, dtype=BF16)), "one dtype")
    refused(dropout(y=rows(OUT, row=63)), "overlap")
    refused(dropout(y=rows(FAKE, user=1280)), "the same memory")
    refused(dropout(residual=rows(OUT, user=1280)), "the same memory")
    refused(dropout(lens=FAKE + 2), "lens")


def test_lookup():
    refused(lookup(t=table(None)), "table is NULL")
    refused(lookup(t=table(dtype=5)), "dtype 5")
    refused(lookup(t=table(FAKE + 1)), "table is not aligned")
    refused(lookup(t=table(n=0)), "0 rows")
    refused(lookup(t=table(n=1 << 31)), "2^31")
    refused(lookup(t=table(stride=-1)), "stride")
    refused(lookup(i=ids(None)), "ids is NULL")
    refused(lookup(i=ids(kind=2)), "type 2")
    refused(lookup(i=ids(FAKE + 4)), "ids is not aligned")
    refused(lookup(i=ids(user=-1)), "strides")
    refused(lookup(lens=FAKE + 1), "lens")
    refused(lookup(e=rows(None)), "e is NULL")
    refused(lookup(e=rows(OUT, row=63)), "overlap")
    refused(lookup(e=rows(FAKE * 2)), "the table")
    for bad in (float("nan"), float("inf"), 3e38):
        refused(lookup(scale=bad, drop=mask(0.5)), "scale")


def test_sort():
    refused(sort(B=0), "B=0")
    refused(sort(n=0), "0 rows")
    refused(sort(n=1 << 31), "2^31")
    refused(sort(i=ids(kind=7)), "type 7")
    for f in ("tokens", "runs", "rows", "counts"):
        refused(sort(o=some_order(**{f: None})), "NULL")
        refused(sort(o=some_order(**{f: FAKE + 2})), "not aligned")
    refused(sort(o=some_order(runs=FAKE)), "the same memory")
    refused(back(o=some_order(counts=FAKE * 3)), "the same memory")
    refused(sort(ws=None), "ws")
    refused(sort(ws=WS + 64), "ws")
    for B, L, n in ((4, 10, 100), (100, 1000, 7), (100, 1000, 1 << 20), (1000, 1000, (1 << 31) - 1)):
        need = lg.longer_sort_ids_workspace_bytes(B, L, n)
        assert need > 0 and need % 256 == 0
        refused(sort(B=B, L=L, n=n, ws_bytes=need - 1), "workspace too small", -2)
    for B, L, n in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (1 << 20, 1 << 20, 8), (1, 1, 1 << 31)):
        assert lg.longer_sort_ids_workspace_bytes(B, L, n) == 0


def test_backward():
    refused(back(o=some_order(rows=None)), "NULL")
    refused(back(de=rows(dtype=3)), "dtype 3")
    refused(back(de=rows(None)), "de is NULL")
    refused(back(dense=2), "dense=2")
    refused(back(n=0), "0 rows")
    refused(back(grads=None), "grads_out is NULL")
    refused(back(grads=OUT + 2), "grads_out is not aligned")
    refused(back(norms=OUT + 1), "norms_out")
    refused(back(grads=FAKE), "the same memory")
    refused(back(norms=OUT), "the same memory")
    refused(back(scale=float("inf")), "scale")
    refused(back(ws=None), "ws")
    for B, L, d in ((4, 10, 64), (100, 1000, 4099)):
        need = lg.longer_embedding_backward_workspace_bytes(B, L, d)
        assert need > 0 and need % 256 == 0
        refused(back(B=B, L=L, d=d, de=rows(user=L * d, row=d), ws_bytes=need - 1), "workspace too small", -2)
    for B, L, d in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (1, 1, 16385), (1 << 20, 1 << 20, 8)):
        assert lg.longer_embedding_backward_workspace_bytes(B, L, d) == 0


@pytest.mark.parametrize("kw,word", [
    (dict(B=0), "B=0"), (dict(o=some_order(counts=None)), "NULL"), (dict(d=0), "d=0"), (dict(rows=0), "0 rows"), (dict(p=None), "p is NULL"), (dict(m=None), "m is NULL"),
    (dict(v=None), "v is NULL"), (dict(g=None), "g is NULL"), (dict(g=FAKE + 2), "g is not aligned"), (dict(w_dtype=4), "dtype 4 of w"), (dict(w=OUT * 4 + 1), "w is not aligned"),
    (dict(m=OUT), "same memory"), (dict(w=OUT * 3), "same memory"), (dict(lr=-1.0), "lr"), (dict(beta1=1.0), "beta1"), (dict(eps=0.0), "eps"), (dict(step=0), "step=0"),
    (dict(decay=-0.1), "decay"), (dict(decay=float("nan")), "decay"), (dict(norm=FAKE + 1), "norm")])
def test_adamw_rows(kw, word):
    refused(adamw(**kw), word)


def test_python_calls_check_their_tensors():
    import torch
    t, i = torch.zeros(2, 3, 8), torch.zeros(2, 3, dtype=torch.int64)
    if torch.cuda.is_available():
        pytest.skip("GPU present")
    with pytest.raises(lg.LongerError):
        lg.DropoutMask(0.1, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(lg.LongerError):
        lg.TokenOrder(i, i, i, i)
    with pytest.raises(lg.LongerError):
        lg.AdamWRows(t[0], t[0], t[0], None, 0.0)
    with pytest.raises(lg.LongerError):
        lg.longer_embedding(t[0], i, None, 1.0, None, t)


def test_the_generator_against_the_known_answers_of_its_authors():
    """The test vectors of philox4x32 with ten rounds that were published with the generator."""
    for counter, key, want in (
            ((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
            ((0xffffffff,) * 4, (0xffffffff,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
            ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0), (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1))):
        assert tuple(int(x) for x in philox4x32(counter, key)) == want


def test_the_oracle_on_a_batch_by_hand():
    i = np.array([[5, 2, 5, -1], [2, 9, 7, 5]])
    tokens, runs, distinct = order(i, [4, 3], 8)                 # 9 is no row; the last token is padding
    assert tokens.tolist() == [1, 4, 0, 2, 6] and runs.tolist() == [0, 0, 1, 1, 2] and distinct.tolist() == [2, 5, 7]
    de = np.arange(8.0).reshape(2, 4, 1) + 1
    _, g, mag, count = gradient(i, [4, 3], 8, de, 2.0)
    assert g[:, 0].tolist() == [14.0, 8.0, 14.0] and count.tolist() == [2, 2, 1] and (mag == g).all()
    f = factors(np.arange(2000), 33, 0.25, 77, 5, 2)
    assert set(np.unique(f)) == {0.0, 4 / 3}
    # 66000 draws of a share of a quarter: five standard deviations
    assert abs((f == 0).mean() - 0.25) < 5 * np.sqrt(0.25 * 0.75 / f.size)

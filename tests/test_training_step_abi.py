"""Refusals of the layer norm, gradient norm, clipping and AdamW entry points: status codes and messages from the host, before
anything is launched (no GPU needed; the pointers are never dereferenced)."""
import ctypes

import pytest

import paper_2505_04421_amd as lg
from paper_2505_04421_amd.binding import CAdamW, CAdamWTensor, CRows, CTensor

F32, BF16 = 0, 1
FAKE, OUT, WS = 1 << 20, 1 << 24, 1 << 28


def rows(at=FAKE, user=640, row=64, dtype=BF16):
    return CRows(at, user, row, dtype)


def norm(x=None, g=FAKE, b=FAKE, lens=None, B=4, L=10, d=64, eps=1e-5, y=None):
    x, y = x if x is not None else rows(), y if y is not None else rows(OUT)
    return lg.load_library().longer_layer_norm(ctypes.byref(x), g, b, lens, B, L, d, eps, ctypes.byref(y), None)


def back(x=None, g=FAKE, dy=None, lens=None, B=4, L=10, d=64, eps=1e-5, dx=None, grads=OUT, ws=WS, ws_bytes=1 << 40):
    x, dy, dx = x or rows(), dy or rows(FAKE * 3, dtype=F32), dx or rows(OUT, dtype=F32)
    return lg.load_library().longer_layer_norm_backward(ctypes.byref(x), g, ctypes.byref(dy), lens, B, L, d, eps, ctypes.byref(dx),
                                                        grads, ws, ws_bytes, None)


def refused(rc, word, code=-1):
    assert rc == code and word in lg.longer_last_error(), (rc, lg.longer_last_error())


@pytest.mark.parametrize("call", [norm, back])
def test_layer_norm_sizes_and_rows(call):
    refused(call(B=0), "B=0")
    refused(call(L=0), "L=0")
    refused(call(L=-1), "L=-1")
    refused(call(B=1 << 16, L=1 << 15), "2^31")
    refused(call(d=0), "d=0")
    refused(call(d=16385), "d=16385")
    refused(call(eps=0.0), "eps")
    refused(call(eps=float("nan")), "eps")
    refused(call(g=None), "ln_g is NULL")
    refused(call(g=FAKE + 1), "ln_g is not aligned")
    refused(call(lens=FAKE + 2), "lens")
    refused(call(x=rows(None)), "x is NULL")
    refused(call(x=rows(FAKE + 1)), "x is not aligned")
    refused(call(x=rows(dtype=7)), "dtype 7")
    refused(call(x=rows(row=-64)), "strides")
    refused(call(x=rows(user=(1 << 40) + 1)), "strides")


def test_layer_norm_outputs():
    refused(norm(y=rows(OUT, dtype=F32)), "one dtype")
    refused(norm(y=rows(None)), "y is NULL")
    refused(norm(y=rows(OUT, row=63)), "overlap")
    refused(norm(y=rows(OUT, user=639)), "overlap")
    refused(norm(y=rows(OUT, user=0)), "overlap")
    refused(norm(y=rows(OUT, user=64, row=255)), "overlap")          # users inside rows, one value short
    refused(norm(y=rows(FAKE, user=1280)), "the same memory")
    refused(norm(b=None), "ln_b is NULL")
    refused(back(dx=rows(OUT, row=63, dtype=F32)), "overlap")
    refused(back(dx=rows(OUT, dtype=BF16)), "dy and dx")
    refused(back(x=rows(dtype=F32), dy=rows(FAKE * 3), dx=rows(OUT)), "dy and dx")
    refused(back(dx=rows(FAKE * 3, user=1280, dtype=F32)), "the same memory")
    refused(back(dy=rows(FAKE * 3), dx=rows(FAKE)), "dx may not be x")
    refused(back(grads=None), "grads_out is NULL")
    refused(back(grads=OUT + 2), "grads_out is not aligned")
    refused(back(ws=None), "ws")
    refused(back(ws=WS + 16), "ws")
    need = lg.longer_layer_norm_backward_workspace_bytes(4, 10, 64)
    assert need > 0 and need % 256 == 0
    refused(back(ws_bytes=need - 1), "workspace too small", -2)


def test_layer_norm_workspace_query():
    for B, L, d in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (1, 1, 16385), (1 << 20, 1 << 20, 8)):
        assert lg.longer_layer_norm_backward_workspace_bytes(B, L, d) == 0
    assert lg.longer_layer_norm_backward_workspace_bytes(256, 2000, 128) < 64 << 20


def tensors(*ts):
    return (CTensor * max(1, len(ts)))(*[CTensor(*t) for t in ts])


def grad_norm(ts, count=None, max_norm=1.0, out=OUT, ws=WS, ws_bytes=1 << 40):
    return lg.load_library().longer_grad_norm(ts, len(ts) if count is None else count, max_norm, out, ws, ws_bytes, None)


BAD_LISTS = [(((FAKE, -1, F32),), "n=-1"), (((FAKE, 1 << 45, F32),), "out of range"), (((FAKE, 1 << 40, F32), (FAKE, 1, F32)), "2^40"),
             (((None, 4, F32),), "data is NULL"), (((FAKE, 4, F32), (FAKE + 2, 4, F32)), "tensor 1: data is not aligned"),
             (((FAKE, 4, BF16), (FAKE + 1, 4, BF16)), "not aligned"), (((FAKE, 4, 2),), "dtype 2")]


@pytest.mark.parametrize("ts,word", BAD_LISTS)
def test_bad_lists(ts, word):
    lib, ts = lg.load_library(), tensors(*ts)
    refused(grad_norm(ts), word)
    refused(lib.longer_clip_gradients(ts, None, len(ts), FAKE, None), word)
    refused(lib.longer_clip_gradients(tensors(*[(FAKE, 4, F32)] * len(ts)), ts, len(ts), FAKE, None), word)
    assert lib.longer_grad_norm_workspace_bytes(ts, len(ts)) == 0


def test_gradient_norm_and_clip_refusals():
    lib, ts = lg.load_library(), tensors((FAKE, 4000, F32), (None, 0, BF16), (FAKE, 9, BF16))
    refused(grad_norm(ts, count=0), "empty list")
    refused(grad_norm(ts, count=-1), "empty list")
    refused(lib.longer_grad_norm(None, 1, 1.0, OUT, WS, 1 << 20, None), "empty list")
    for bad in (0.0, -1.0, float("nan")):
        refused(grad_norm(ts, max_norm=bad), "max_norm")
    refused(grad_norm(ts, out=None), "null")
    refused(grad_norm(ts, out=OUT + 2), "norm_out")
    refused(grad_norm(ts, ws=None), "null")
    refused(grad_norm(ts, ws=WS + 8), "256-byte")
    need = lib.longer_grad_norm_workspace_bytes(ts, 3)
    assert need > 0 and need % 256 == 0
    refused(grad_norm(ts, ws_bytes=need - 1), "workspace too small", -2)
    refused(lib.longer_clip_gradients(ts, None, 3, None, None), "norm is NULL")
    refused(lib.longer_clip_gradients(ts, None, 3, FAKE + 1, None), "norm is NULL or not aligned")
    refused(lib.longer_clip_gradients(ts, tensors((OUT, 4000, F32), (None, 0, BF16), (OUT, 8, BF16)), 3, FAKE, None), "another size")
    refused(lib.longer_clip_gradients(ts, tensors((OUT, 4000, BF16), (None, 0, BF16), (OUT, 9, BF16)), 3, FAKE, None), "another size")


def adamw(count=1, norm=None, lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, step=1, **kw):
    t = dict(p=FAKE, m=FAKE * 2, v=FAKE * 3, g=FAKE * 4, w=FAKE * 5, n=64, g_dtype=F32, w_dtype=BF16, decay=0.0)
    t.update(kw)
    return lg.load_library().longer_adamw_step((CAdamWTensor * 1)(CAdamWTensor(**t)), count, ctypes.byref(CAdamW(lr, beta1, beta2, eps, step)), norm, None)


@pytest.mark.parametrize("kw,word", [
    (dict(count=0), "empty list"), (dict(lr=-1.0), "lr"), (dict(lr=float("inf")), "lr"), (dict(lr=float("nan")), "lr"), (dict(beta1=1.0), "beta1"),
    (dict(beta1=-0.1), "beta1"), (dict(beta2=1.0), "beta2"), (dict(beta2=float("nan")), "beta2"), (dict(eps=0.0), "eps"), (dict(eps=float("inf")), "eps"),
    (dict(step=0), "step=0"), (dict(step=-4), "step"), (dict(norm=FAKE + 1), "norm"), (dict(n=-1), "n=-1"), (dict(n=1 << 45), "out of range"),
    (dict(p=None), "p is NULL"), (dict(m=None), "m is NULL"), (dict(v=None), "v is NULL"), (dict(g=None), "g is NULL"),
    (dict(g_dtype=5), "dtype 5 of g"), (dict(w_dtype=5), "dtype 5 of w"), (dict(p=FAKE + 2), "p is not aligned"), (dict(w=FAKE * 5 + 1), "w is not aligned"),
    (dict(m=FAKE), "same memory"), (dict(w=FAKE * 4), "same memory"), (dict(decay=-0.1), "decay"), (dict(decay=float("nan")), "decay")])
def test_adamw_refusals(kw, word):
    refused(adamw(**kw), word)


def test_python_calls_check_their_tensors():
    import torch
    t = torch.zeros(2, 3, 8)
    if torch.cuda.is_available():
        pytest.skip("GPU present")
    with pytest.raises(lg.LongerError):
        lg.longer_layer_norm(t, t[0, 0], t[0, 0], None, 1e-5, t)
    with pytest.raises(lg.LongerError):
        lg.TensorList([t])
    with pytest.raises(lg.LongerError):
        lg.AdamWList([t], [t], [t], [t], None, [0.0, 0.0])

"""longer_layer_norm and longer_layer_norm_backward against the formulas in 64 bits: every width class, ragged and empty users,
strides, alignment, memory around the rows, reuse of buffers, and the gradient against differences.

Tolerances.  u = 2^-24 is half an ulp of fp32.  A sum of d values taken in parts that are joined has a relative error of at most
(longest chain of additions) u of the sum of magnitudes; no kernel adds more than d / 64 + 16 values of a row in a chain, so
k = d / 64 + 48 covers a row's sums and the few operations around them.  A normalised value xh = (x - mean) r inherits the mean's
error, u max|x| r at most per step: the factor 1 + max|x| r.  Results in bf16 add half an ulp, 2^-8 of the value (8 significant bits)."""
import numpy as np
import pytest
import torch

import paper_2505_04421_amd as lg
from gpu_util import guarded_empty

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
EPS = 1e-5
SHAPES = [(1, 1, 1), (3, 5, 2), (2, 3, 7), (4, 9, 8), (2, 7, 31), (4, 64, 32), (5, 33, 64), (3, 17, 65), (2, 9, 127), (3, 40, 128), (2, 5, 129),
          (1, 3, 255), (3, 11, 256), (2, 4, 257), (1, 6, 500), (2, 3, 512), (2, 3, 1023), (1, 5, 1025), (1, 3, 2049), (2, 2, 4099),
          (1, 3, 8191), (1, 2, 8193), (1, 2, 16383), (1, 2, 16384), (700, 3, 64), (1, 2500, 96), (9, 700, 24)]
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def draw(B, L, d, dtype, seed, ragged=False):
    r = np.random.default_rng(seed)
    x = r.standard_normal((B, L, d)) * np.exp(r.standard_normal((B, L, 1))) + 0.25
    g, b = r.uniform(0.9, 1.1, d), r.uniform(-0.05, 0.05, d)
    dy = r.standard_normal((B, L, d)) * np.exp(r.standard_normal((B, L, 1)))
    lens = None
    if ragged:
        lens = r.integers(0, L + 1, B).astype(np.int32)
        lens[0] = 0
        if B > 1:
            lens[1] = L + 3                      # beyond the rows: all of them count
        if B > 2:
            lens[2] = 1
    t = DTYPES[dtype]
    up = lambda a, t: torch.from_numpy(a.astype(np.float32)).to(DEV).to(t)
    return up(x, t), up(g, t), up(b, t), up(dy, torch.float32), None if lens is None else torch.from_numpy(lens).to(DEV)


def valid_rows(lens, B, L):
    n = np.full(B, L) if lens is None else lens.cpu().numpy()
    return np.arange(L)[None, :] < n[:, None]


def np64(t):
    return t.double().cpu().numpy()


class Ref:
    """The formulas, straight, and the error bounds of the docstring."""

    def __init__(self, x, g, b, dy, lens):
        self.d = d = x.shape[2]
        self.ok = valid_rows(lens, x.shape[0], x.shape[1])
        x, g, dy = np.where(self.ok[..., None], np64(x), 0.0), np64(g), np.where(self.ok[..., None], np64(dy), 0.0)
        mean = x.mean(-1, keepdims=True)
        r = 1 / np.sqrt(((x - mean) ** 2).mean(-1, keepdims=True) + EPS)
        xh = (x - mean) * r
        k = (d / 64 + 48) * U * (1 + np.abs(x).max(-1, keepdims=True) * r)
        q = dy * g
        self.dx = r * (q - q.mean(-1, keepdims=True) - xh * (q * xh).mean(-1, keepdims=True))
        aq = np.abs(q).mean(-1, keepdims=True)
        # each of the two means is off by k of its magnitudes, and xh by k (1 + |xh|)
        self.dx_tol = 2 * k * r * (np.abs(q) + aq + (1 + np.abs(xh)) ** 2 * (np.abs(q * (1 + np.abs(xh)))).mean(-1, keepdims=True))
        rows = self.ok.sum()
        chain = rows / 64 + 64               # no column is added up in longer chains than this
        self.dg = (dy * xh).sum((0, 1))
        self.dg_tol = (np.abs(dy) * (1 + np.abs(xh)) * (2 * k + chain * U)).sum((0, 1))
        self.db = dy.sum((0, 1))
        self.db_tol = chain * U * np.abs(dy).sum((0, 1))
        if b is not None:
            self.y = xh * g + np64(b)
            self.y_tol = 2 * k * ((1 + np.abs(xh)) * np.abs(g) + np.abs(np64(b)))
            self.y[~self.ok] = 0
        self.dx[~self.ok] = 0

    def near(self, got, want, tol, what, half=False):
        got = np64(got)
        tol = tol + (np.abs(want) * 2.0 ** -8 * 1.01 + 2.0 ** -130 if half else 0) + 1e-300
        off = np.abs(got - want)
        assert np.isfinite(got).all(), what
        assert (off <= tol).all(), "%s: worst %.3g of its bound" % (what, (off / tol).max())
        if got.ndim == 3:
            assert (got[~self.ok] == 0).all(), what + ": padding"


def workspace(B, L, d):
    n = lg.longer_layer_norm_backward_workspace_bytes(B, L, d)
    assert n > 0, lg.longer_last_error()
    return guarded_empty(DEV, (n,), torch.uint8)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,L,d", SHAPES)
def test_forward(B, L, d, dtype):
    print("  longer_layer_norm", B, L, d, dtype, flush=True)
    for ragged in (False, True):
        x, g, b, dy, lens = draw(B, L, d, dtype, B * 7 + L + d, ragged)
        ref = Ref(x, g, b, dy, lens)
        x[~torch.from_numpy(ref.ok).to(DEV)] = float("nan")
        y, guard = guarded_empty(DEV, (B, L, d), x.dtype)
        lg.longer_layer_norm(x, g, b, lens, EPS, y)
        torch.cuda.synchronize()
        guard.check("y")
        ref.near(y, ref.y, ref.y_tol, "y", dtype == "bf16")


@pytest.mark.parametrize("dtype,grad", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("B,L,d", SHAPES)
def test_backward(B, L, d, dtype, grad):
    print("  longer_layer_norm_backward", B, L, d, dtype, grad, flush=True)
    for ragged in (False, True):
        x, g, b, dy, lens = draw(B, L, d, dtype, B * 5 + L + d, ragged)
        dy = dy.to(DTYPES[grad])
        ref = Ref(x, g, None, dy, lens)
        pad = ~torch.from_numpy(ref.ok).to(DEV)
        x[pad], dy[pad] = float("nan"), float("nan")
        dx, g1 = guarded_empty(DEV, (B, L, d), dy.dtype)
        grads, g2 = guarded_empty(DEV, (2, d), torch.float32)
        ws, g3 = workspace(B, L, d)
        lg.longer_layer_norm_backward(x, g, dy, lens, EPS, dx, grads, ws)
        torch.cuda.synchronize()
        for k in (g1, g2, g3):
            k.check("backward")
        ref.near(dx, ref.dx, ref.dx_tol, "dx", grad == "bf16")
        ref.near(grads[0], ref.dg, ref.dg_tol, "ln_g's gradient")
        ref.near(grads[1], ref.db, ref.db_tol, "ln_b's gradient")
        # the same call again, its workspace dirty: the same bits
        dx2, grads2 = torch.empty_like(dx), torch.empty_like(grads)
        lg.longer_layer_norm_backward(x, g, dy, lens, EPS, dx2, grads2, ws)
        assert torch.equal(dx, dx2) and torch.equal(grads, grads2)


def strided(t, of, wide, shift):
    """The same rows inside a larger buffer of NaN: `of` rows a user, `wide` values a row, `shift` values from its start."""
    B, L, d = t.shape
    buf = torch.full((shift + B * of * wide,), float("nan"), dtype=t.dtype, device=t.device)
    view = buf[shift:].view(B, of, wide)[:, :L, :d]
    view.copy_(t)
    return view, buf


@pytest.mark.parametrize("B,L,d,of,wide,shift", [(3, 5, 64, 9, 64, 0), (3, 5, 64, 5, 65, 1), (2, 8, 128, 108, 128, 3), (4, 3, 77, 4, 80, 5), (2, 2, 1030, 3, 1031, 7),
                                                 (2, 3, 6, 4, 9, 1), (1, 4, 5000, 4, 5003, 1)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_and_alignment(B, L, d, of, wide, shift, dtype):
    print("  strided", B, L, d, of, wide, shift, dtype, flush=True)
    x, g, b, dy, lens = draw(B, L, d, dtype, 3, True)
    ref = Ref(x, g, b, dy, lens)
    xv, _ = strided(x, of, wide, shift)
    out = torch.full_like(x, 7.0)
    yv, ybuf = strided(out, of, wide, shift)
    before = ybuf.clone()
    gv, bv = torch.cat([g[:1], g])[1:], torch.cat([b[:1], b])[1:]            # parameters off alignment
    lg.longer_layer_norm(xv, gv, bv, lens, EPS, yv)
    ref.near(yv, ref.y, ref.y_tol, "y", dtype == "bf16")
    yv.fill_(7.0)
    assert torch.equal(ybuf.view(torch.uint8), before.view(torch.uint8))      # nothing between the rows was written
    dyv, _ = strided(dy, of, wide, shift)
    dxv, dxbuf = strided(torch.full_like(dy, 7.0), of, wide, shift)
    before = dxbuf.clone()
    grads = torch.empty(2 * d + 1, device=DEV)[1:].view(2, d)
    lg.longer_layer_norm_backward(xv, gv, dyv, lens, EPS, dxv, grads, workspace(B, L, d)[0])
    ref.near(dxv, ref.dx, ref.dx_tol, "dx")
    ref.near(grads[0], ref.dg, ref.dg_tol, "ln_g's gradient")
    ref.near(grads[1], ref.db, ref.db_tol, "ln_b's gradient")
    dxv.fill_(7.0)
    assert torch.equal(dxbuf.view(torch.uint8), before.view(torch.uint8))


def test_rows_of_users_side_by_side_and_broadcast_inputs():
    """[L, B, d] memory seen as [B, L, d], and one row that every row of the input is a view of."""
    B, L, d = 3, 6, 96
    x, g, b, dy, lens = draw(B, L, d, "bf16", 11, True)
    ref = Ref(x, g, b, dy, lens)
    xt, yt = x.transpose(0, 1).contiguous().transpose(0, 1), torch.empty(L, B, d, dtype=x.dtype, device=DEV).transpose(0, 1)
    lg.longer_layer_norm(xt, g, b, lens, EPS, yt)
    ref.near(yt, ref.y, ref.y_tol, "y", True)
    one = x[:1, :1].expand(B, L, d)
    ones = dy[:1, :1].expand(B, L, d)
    ref = Ref(one, g, b, ones, lens)
    y, dx, grads = torch.empty_like(x), torch.empty_like(dy), torch.empty(2, d, device=DEV)
    lg.longer_layer_norm(one, g, b, lens, EPS, y)
    ref.near(y, ref.y, ref.y_tol, "y", True)
    lg.longer_layer_norm_backward(one, g, ones, lens, EPS, dx, grads, workspace(B, L, d)[0])
    ref.near(dx, ref.dx, ref.dx_tol, "dx")
    ref.near(grads[0], ref.dg, ref.dg_tol, "ln_g's gradient")


@pytest.mark.parametrize("d", [32, 128, 203, 1024, 4099, 16383])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place(d, dtype):
    x, g, b, dy, lens = draw(3, 4, d, dtype, 5, True)
    y = torch.empty_like(x)
    lg.longer_layer_norm(x, g, b, lens, EPS, y)
    dx, grads, ws = torch.empty_like(dy), torch.empty(2, d, device=DEV), workspace(3, 4, d)[0]
    lg.longer_layer_norm_backward(x, g, dy, lens, EPS, dx, grads, ws)
    grads2 = torch.empty_like(grads)
    lg.longer_layer_norm_backward(x, g, dy, lens, EPS, dy, grads2, ws)
    lg.longer_layer_norm(x, g, b, lens, EPS, x)
    assert torch.equal(x, y) and torch.equal(dx, dy) and torch.equal(grads, grads2)


@pytest.mark.parametrize("d", [64, 8191])
def test_constant_rows_and_large_values(d):
    """A row of one value has no variance: y = ln_b, dx as the formula has it; values near the type's end stay finite."""
    x, g, b, dy, _ = draw(2, 2, d, "f32", 6)
    x[0, 0] = 0.75
    x[0, 1] = 0.0
    x[1, 0] *= 1e15
    x[1, 1] *= 1e-15
    ref = Ref(x, g, b, dy, None)
    y, dx, grads = torch.empty_like(x), torch.empty_like(x), torch.empty(2, d, device=DEV)
    lg.longer_layer_norm(x, g, b, None, EPS, y)
    ref.near(y, ref.y, ref.y_tol, "y")
    lg.longer_layer_norm_backward(x, g, dy, None, EPS, dx, grads, workspace(2, 2, d)[0])
    ref.near(dx, ref.dx, ref.dx_tol, "dx")
    ref.near(grads[0], ref.dg, ref.dg_tol, "ln_g's gradient")


def test_a_row_with_nan_or_infinity_keeps_it_to_itself():
    x, g, b, dy, _ = draw(2, 5, 130, "f32", 8)
    x[0, 1, 129], x[1, 2, 0] = float("nan"), float("inf")
    y = torch.empty_like(x)
    lg.longer_layer_norm(x, g, b, None, EPS, y)
    bad = torch.zeros(2, 5, dtype=torch.bool, device=DEV)
    bad[0, 1], bad[1, 2] = True, True
    assert torch.isnan(y[bad]).all() and torch.isfinite(y[~bad]).all()


def test_offsets_beyond_32_bits():
    """Two users more than 2^31 values apart."""
    B, L, d, apart = 2, 3, 136, (1 << 31) + 40
    x, g, b, dy, _ = draw(B, L, d, "bf16", 9)
    dy = dy.to(torch.bfloat16)
    ref = Ref(x, g, b, dy, None)
    buf = torch.empty(apart + L * d, dtype=torch.bfloat16, device=DEV)
    out = torch.empty(apart + L * d, dtype=torch.bfloat16, device=DEV)
    xv, yv = (t.as_strided((B, L, d), (apart, d, 1)) for t in (buf, out))
    xv.copy_(x)
    lg.longer_layer_norm(xv, g, b, None, EPS, yv)
    ref.near(yv, ref.y, ref.y_tol, "y", True)
    grads = torch.empty(2, d, device=DEV)
    lg.longer_layer_norm_backward(xv, g, dy, None, EPS, yv, grads, workspace(B, L, d)[0])
    ref.near(yv, ref.dx, ref.dx_tol, "dx", True)
    ref.near(grads[0], ref.dg, ref.dg_tol, "ln_g's gradient")


def test_more_than_2_to_the_30_rows():
    """Rows of one value: y = ln_b and dx = 0 whatever x is; ln_b's gradient counts the rows that are there (dy = 1: shares below 2^24
    are exact, and they meet in fewer than 128 additions, u of the total each)."""
    B, L = 600, 2_000_000
    r = torch.Generator(device=DEV).manual_seed(3)
    lens = torch.randint(0, L + 1, (B,), generator=r, device=DEV, dtype=torch.int32)
    there = (torch.arange(L, device=DEV) < lens[:, None])
    x = torch.randn(B, L, 1, generator=r, device=DEV, dtype=torch.bfloat16)
    g, b = torch.full((1,), 0.5, device=DEV, dtype=torch.bfloat16), torch.full((1,), 3.0, device=DEV, dtype=torch.bfloat16)
    y = torch.full_like(x, 7.0)
    for n in (None, lens):
        print("  longer_layer_norm", B, L, 1, n is not None, flush=True)
        lg.longer_layer_norm(x, g, b, n, EPS, y)
        assert bool((y[..., 0] == (3.0 if n is None else torch.where(there, 3.0, 0.0))).all())
    dy, grads = torch.ones(B, L, 1, device=DEV), torch.empty(2, 1, device=DEV)
    lg.longer_layer_norm_backward(x, g, dy, lens, EPS, dy, grads, workspace(B, L, 1)[0])
    assert not bool(dy.any()) and float(grads[0]) == 0.0
    rows = int(lens.sum(dtype=torch.int64))
    assert abs(float(grads[1]) - rows) <= 128 * U * rows


def test_on_another_stream_and_in_a_graph():
    x, g, b, dy, lens = draw(40, 50, 128, "bf16", 10, True)
    want, dx, grads, ws = torch.empty_like(x), torch.empty_like(dy), torch.empty(2, 128, device=DEV), workspace(40, 50, 128)[0]
    lg.longer_layer_norm(x, g, b, lens, EPS, want)
    lg.longer_layer_norm_backward(x, g, dy, lens, EPS, dx, grads, ws)
    y, dx2, grads2 = torch.zeros_like(x), torch.zeros_like(dx), torch.zeros_like(grads)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    lg.longer_layer_norm(x, g, b, lens, EPS, y, stream=s)
    lg.longer_layer_norm_backward(x, g, dy, lens, EPS, dx2, grads2, ws, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(y, want) and torch.equal(dx, dx2) and torch.equal(grads, grads2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lg.longer_layer_norm(x, g, b, lens, EPS, y)
        lg.longer_layer_norm_backward(x, g, dy, lens, EPS, dx2, grads2, ws)
    for _ in range(3):
        for t in (y, dx2, grads2):
            t.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(dx, dx2) and torch.equal(grads, grads2)


@pytest.mark.parametrize("d", [5, 64, 200])
def test_gradient_against_differences(d):
    """Central differences of sum(w y), y from the formula in 64 bits, step h: off by h^2 / 6 of the third derivative, which for
    rows of order 1 is of the order of the first; h = 1e-4 leaves 1e-8 of it beside 1e-12 / h of rounding, far below the kernel's bound."""
    B, L = 2, 3
    r = np.random.default_rng(d)
    x, g, b, w = (r.standard_normal(s).astype(np.float32) for s in ((B, L, d), d, d, (B, L, d)))
    up = lambda a: torch.from_numpy(a).to(DEV)
    dx, grads = torch.empty(B, L, d, device=DEV), torch.empty(2, d, device=DEV)
    lg.longer_layer_norm_backward(up(x), up(g), up(w), None, EPS, dx, grads, workspace(B, L, d)[0])
    ref = Ref(up(x), up(g), up(b), up(w), None)

    def loss(x, g, b):
        c = x - x.mean(-1, keepdims=True)
        return (w.astype(np.float64) * (c / np.sqrt((c * c).mean(-1, keepdims=True) + EPS) * g + b)).sum()

    h = 1e-4
    args = [a.astype(np.float64) for a in (x, g, b)]
    for which, got, tol in ((0, np64(dx), ref.dx_tol), (1, np64(grads[0]), ref.dg_tol), (2, np64(grads[1]), ref.db_tol)):
        flat, got, tol = args[which].reshape(-1), got.reshape(-1), tol.reshape(-1)
        for i in r.choice(flat.size, min(12, flat.size), replace=False):
            keep, ends = flat[i], []
            for s in (h, -h):
                flat[i] = keep + s
                ends.append(loss(*args))
            flat[i] = keep
            assert abs((ends[0] - ends[1]) / (2 * h) - got[i]) <= tol[i] + 1e-5 * (1 + np.abs(got).max()), (which, i)

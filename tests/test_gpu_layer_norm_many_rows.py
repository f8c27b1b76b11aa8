"""longer_layer_norm and longer_layer_norm_backward with more rows than the chip takes at once, so that every workgroup goes on to second,
third and later turns: at a width of every class (lanes of a row, pieces of a lane, whether the row ends with the lanes, with a piece or
inside one), dense and ragged, against the formulas in 64 bits on the GPU; and rows that are not finite beside rows that are.

Tolerances.  u = 2^-24.  k = (d / 64 + 48) u (1 + max|x| r) bounds a row's sums relative to their magnitudes, as no sum over a row has a longer
chain of additions than d / 64 + 16; dx takes it of both of its means and of xh.  bf16 results add half an ulp, 2^-8.  Column sums: a lane
adds one row a turn; a turn of 256 workgroups or more takes at least 2^18 / lanes rows, a row has at most d / 2 + 1 lanes, 6 + 16 + 16 + 32 additions
join the lanes' sums: chains of at most rows (d / 2 + 1) / 2^18 + 80 additions."""
import pytest
import torch

import paper_2505_04421_amd as lg
from gpu_util import guarded_empty

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
EPS = 1e-5
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
WIDTHS = {
    "f32": [1, 4, 7, 8, 11, 12, 16, 20, 26, 32, 36, 51, 64, 116, 119, 128, 145, 192, 256, 356, 389, 512, 659, 716, 768, 824, 975, 1024, 1026,
            1276, 1536, 1552, 2011, 2048, 2832, 3033, 3385, 3860, 4096, 4375, 5012, 6144, 6692, 7011, 8192, 8359, 10616, 12288, 12410, 16160, 16384],
    "bf16": [5, 8, 15, 16, 24, 30, 32, 40, 42, 64, 100, 120, 128, 144, 223, 256, 288, 317, 512, 529, 904, 1024, 1256, 1513, 1536, 1764, 1784,
             2048, 2440, 2940, 3880, 3970, 4096, 4101, 4296, 6144, 7144, 7773, 8192, 9968, 10277, 12288, 13534, 14784, 16384],
}


def rows_for(dtype, d):
    """Rows of width d of which every workgroup has more than three turns: lanes of 16 bytes of the row, up to four (bf16, fp32) such
    pieces a lane, against the 2048 threads (1280 with three pieces or four) that a compute unit holds at most."""
    v = 4 if dtype == "f32" else 8
    pieces = -(-d // v)
    lanes = 1
    while lanes < pieces and lanes < 64:
        lanes *= 2
    if d < v:
        lanes = 8
    if pieces <= 128:
        return -(-1_700_000 // lanes)
    return -(-1_300_000 // max(64, pieces // 4))


def drawn(B, L, d, dtype, seed):
    """x, gain, bias, dy (of x's type's values, in fp32) and lengths: none, all and more than all of the rows among them."""
    r = torch.Generator(device=DEV).manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=r, device=DEV)
    t = DTYPES[dtype]
    z = randn(B, L, d)
    dy = (0.5 + 0.5 * z + randn(B, L, d).mul_(randn(B, L, 1).exp_())).to(t).float()       # (column sums far from zero)
    x = z.mul_(randn(B, L, 1).exp_()).add_(0.25).to(t)
    g, b = (0.9 + 0.2 * torch.rand(d, generator=r, device=DEV)).to(t), (0.1 * torch.rand(d, generator=r, device=DEV) - 0.05).to(t)
    lens = torch.randint(-L // 3, L + L // 3, (B,), generator=r, device=DEV, dtype=torch.int32).clamp_(min=0)
    lens[0] = 0
    lens[-1] = L
    return x, g, b, dy, lens


def near(got, want, tol, what, half=False):
    if half:
        tol = tol + want.abs() * (2.0 ** -8 * 1.01) + 2.0 ** -130
    off = (got.double() - want).abs()
    assert bool((off <= tol + 1e-300).all()), "%s: worst %.3g of its bound" % (what, float((off / (tol + 1e-300)).max()))     # (NaN is not <=)


def expected(x, g, b, dy):
    """y, dx and the columns' terms of rows x [n, d], each with its bound."""
    d = x.shape[-1]
    x, g, b, dy = x.double(), g.double(), b.double(), dy.double()
    c = x - x.mean(-1, keepdim=True)
    r = ((c * c).mean(-1, keepdim=True) + EPS).rsqrt()
    xh = c * r
    k = (d / 64 + 48) * U * (1 + x.abs().amax(-1, keepdim=True) * r)
    one = 1 + xh.abs()
    q = dy * g
    dx = r * (q - q.mean(-1, keepdim=True) - xh * (q * xh).mean(-1, keepdim=True))
    dx_tol = 2 * k * r * (q.abs() + q.abs().mean(-1, keepdim=True) + one * one * (q.abs() * one).mean(-1, keepdim=True))
    y, y_tol = xh * g + b, 2 * k * (one * g.abs() + b.abs())
    return y, y_tol, dx, dx_tol, dy * xh, dy.abs() * one, k


def check_rows(x, g, b, dy, there, y, dxs, grads, what):
    """y [B, L, d] and every dx of `dxs` (by type), row by row, and grads [2, d] of each; `there` [B, L]: rows that are no padding."""
    d = x.shape[2]
    flat = lambda t: t.reshape(-1, d)
    at = there.reshape(-1).nonzero()[:, 0]
    dg, db, db_tol, dg_tol = (torch.zeros(d, dtype=torch.float64, device=DEV) for _ in range(4))
    chain = at.numel() * (d / 2 + 1) / 2 ** 18 + 80
    step = max(1, (1 << 24) // d)
    for rows in at.split(step):
        v = flat(dy)[rows]
        want, tol, dx, dx_tol, terms, sizes, k = expected(flat(x)[rows], g, b, v)
        near(flat(y)[rows], want, tol, what + " y", y.dtype == torch.bfloat16)
        for t in dxs:
            near(flat(t)[rows], dx, dx_tol, what + " dx", t.dtype == torch.bfloat16)
        dg += terms.sum(0)
        dg_tol += (sizes * (2 * k + chain * U)).sum(0)
        db += v.double().sum(0)
        db_tol += chain * U * v.double().abs().sum(0)
    for t in [y] + dxs:
        assert not bool((t.ne(0).any(-1) & ~there).any()), what + ": padding"
    for s in grads:
        near(s[0], dg, dg_tol, what + " ln_g's gradient")
        near(s[1], db, db_tol, what + " ln_b's gradient")


@pytest.mark.parametrize("dtype,d", [(t, d) for t in WIDTHS for d in WIDTHS[t]])
def test_many_turns(dtype, d):
    rows = rows_for(dtype, d)
    L = 101 if rows > 5000 else 13
    B = -(-rows // L)
    print("  layer norm, many turns", B, L, d, dtype, flush=True)
    x, g, b, dy, some = drawn(B, L, d, dtype, d)
    for lens in (None, some):
        there = torch.ones(B, L, dtype=torch.bool, device=DEV) if lens is None else torch.arange(L, device=DEV) < lens[:, None]
        if lens is not None:
            x[~there], dy[~there] = float("nan"), float("nan")
        y, guard = guarded_empty(DEV, (B, L, d), x.dtype)
        lg.longer_layer_norm(x, g, b, lens, EPS, y)
        guards, dxs, grads = [guard], [], []
        n = lg.longer_layer_norm_backward_workspace_bytes(B, L, d)
        for t in sorted({dtype, "f32"}):
            for again in (False, True):
                dx, g1 = guarded_empty(DEV, (B, L, d), DTYPES[t])
                sums, g2 = guarded_empty(DEV, (2, d), torch.float32)
                ws, g3 = guarded_empty(DEV, (n,), torch.uint8)
                lg.longer_layer_norm_backward(x, g, dy.to(DTYPES[t]), lens, EPS, dx, sums, ws)
                guards += [g1, g2, g3]
                if again:                                        # the same bits in another buffer
                    assert torch.equal(dx, dxs[-1]) and torch.equal(sums, grads[-1])
                else:
                    dxs.append(dx)
                    grads.append(sums)
        for k in guards:
            k.check("layer norm")
        check_rows(x, g, b, dy, there, y, dxs, grads, "ragged" if lens is not None else "dense")


@pytest.mark.parametrize("B,L,d,dtype", [(1201, 1009, 128, "bf16"), (1301, 1009, 64, "f32"), (1013, 67, 2500, "f32"), (1409, 97, 2100, "bf16")])
def test_ragged_users_in_shares(B, L, d, dtype):
    """So many ragged rows that the forward pass deals them to workgroups in shares of eight turns: one, several and part of a wave a row."""
    print("  layer norm, shares", B, L, d, dtype, flush=True)
    x, g, b, _, lens = drawn(B, L, d, dtype, 5)
    there = torch.arange(L, device=DEV) < lens[:, None]
    x[~there] = float("nan")
    y, guard = guarded_empty(DEV, (B, L, d), x.dtype)
    lg.longer_layer_norm(x, g, b, lens, EPS, y)
    torch.cuda.synchronize()
    guard.check("y")
    check_rows(x, g, b, torch.zeros(1, 1, 1, device=DEV).expand(B, L, d), there, y, [], [], "y")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [24, 64, 130, 1030, 4099])
def test_rows_that_are_not_finite_keep_it_to_themselves(d, dtype):
    """Rows that share a wave, a workgroup or a turn with a row of NaN or infinities, or with one whose gradient has them."""
    B, L = 30, 101
    x, g, b, dy, _ = drawn(B, L, d, dtype, 17)
    bad, bad_dy = torch.zeros(2, B, L, dtype=torch.bool, device=DEV)
    for i, v in enumerate((float("nan"), float("inf"), -float("inf"))):
        for u in (0, 3, 11):
            x[u, 7 * i + u, (d - 1) * i // 2] = v
            bad[u, 7 * i + u] = True
            dy[u + 1, 5 * i + u, (d - 1) * i // 2] = v
            bad_dy[u + 1, 5 * i + u] = True
    y = torch.empty_like(x)
    lg.longer_layer_norm(x, g, b, None, EPS, y)
    ws = torch.empty(lg.longer_layer_norm_backward_workspace_bytes(B, L, d), dtype=torch.uint8, device=DEV)
    good_x, good = ~bad, ~bad & ~bad_dy
    want, tol, _, _, _, _, _ = expected(x[good_x], g, b, dy[good_x])
    near(y[good_x], want, tol, "y", dtype == "bf16")
    assert not bool(torch.isfinite(y[bad]).any())
    _, _, want, tol, _, _, _ = expected(x[good], g, b, dy[good])
    for t in sorted({dtype, "f32"}):
        dx, sums = torch.empty(B, L, d, dtype=DTYPES[t], device=DEV), torch.empty(2, d, device=DEV)
        lg.longer_layer_norm_backward(x, g, dy.to(DTYPES[t]), None, EPS, dx, sums, ws)
        near(dx[good], want, tol, "dx", t == "bf16")
        assert not bool(torch.isfinite(dx[bad]).any())

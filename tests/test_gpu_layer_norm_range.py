"""Layer norm of rows near the end of fp32's range: values up to 1e18 from their row's mean, as the header allows at every width.

Tolerances as for ordinary rows, u = 2^-24: k = (d / 64 + 48) u (1 + max|x| r) of the magnitudes, bf16 results half an ulp (2^-8) more."""
import pytest
import torch

import paper_2505_04421_amd as lg
from test_gpu_layer_norm_many_rows import DEV, DTYPES, EPS, expected, near

pytestmark = pytest.mark.gpu


def far_rows(d, dtype, seed):
    """Rows of deviations up to 1e18: normal, all at the ends, one value apart, one wave's or lane's values apart."""
    r = torch.Generator(device=DEV).manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=r, device=DEV)
    x = randn(8, d).mul_(3e17).clamp_(-6e17, 6e17)
    x[1] = torch.where(randn(d) > 0, 4.9e17, -4.9e17)
    x[2] = 0.0
    x[2, d // 2] = 9.9e17
    x[3] = 4.5e17
    x[3, : (d + 3) // 4] = -4.5e17
    x[4] = 4.5e17
    x[4, -min(d, 8):] = -4.5e17
    x[5] = x[1].sort().values
    x[6] = 1e15 * randn(d)
    return x.view(2, 4, d).to(DTYPES[dtype])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [7, 128, 203, 1024, 4099, 8192, 16383, 16384])
def test_values_far_from_the_mean(d, dtype):
    x = far_rows(d, dtype, d)
    assert float((x.double() - x.double().mean(-1, keepdim=True)).abs().max()) <= 1e18
    r = torch.Generator(device=DEV).manual_seed(1)
    g, b = (0.9 + 0.2 * torch.rand(d, generator=r, device=DEV)).to(x.dtype), torch.rand(d, generator=r, device=DEV).to(x.dtype)
    dy = torch.randn(2, 4, d, generator=r, device=DEV)
    y, dx, grads = torch.empty_like(x), torch.empty_like(dy), torch.empty(2, d, device=DEV)
    lg.longer_layer_norm(x, g, b, None, EPS, y)
    ws = torch.empty(lg.longer_layer_norm_backward_workspace_bytes(2, 4, d), dtype=torch.uint8, device=DEV)
    lg.longer_layer_norm_backward(x, g, dy, None, EPS, dx, grads, ws)
    want, tol, dx_want, dx_tol, terms, sizes, k = expected(x, g, b, dy)
    near(y, want, tol, "y", dtype == "bf16")
    near(dx, dx_want, dx_tol, "dx")
    near(grads[0], terms.sum((0, 1)), (sizes * (2 * k + 128 * 2.0 ** -24)).sum((0, 1)), "ln_g's gradient")

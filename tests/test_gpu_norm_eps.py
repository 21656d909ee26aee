"""GPU: head norms with the smallest eps.  Each test prints its case before any GPU step."""
import math

import pytest

from tests.test_gpu_exact import D, PK, U, _dt, _g, _gpu, _i32, _randn, log  # noqa: F401
from tests.test_gpu_pages import normed64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("eps", [5e-324, 1e-310, 1e-200, 2.0 ** -457, 2.0 ** -455, 1e-60, 1e-12])
def test_norm_rotate_of_zeros_with_a_tiny_eps(eps, dtype):
    """A head of zeros is 0 / sqrt(eps) = 0, of either sign; the others, of float32's smallest numbers and
    ordinary ones, have their norm: three roundings and the result's, and 2^-149 where it is below the normal range."""
    import torch
    log(f"case: norm_rotate of zeros, eps {eps} {dtype}")
    pk, g = PK(), _g(34)
    dt = _dt(dtype)
    q = _randn(g, 6, 3, D, dtype=dt)
    q[1] = 0
    q[2] = -0.0
    q[3] = torch.randint(-9, 10, (3, D), generator=g, device="cuda").to(dt) * 2.0 ** -133   # exact in bfloat16 too
    q[4, 1] = 0
    q[5, 0, :-1] = 0
    w = (1 + _randn(g, D, dtype=torch.float32, scale=0.3)).to(dt)
    out, _ = pk.norm_rotate(q, None, _i32([0] * 6), pk.pair_axes((64,)), 1e4, w, None, eps)
    torch.cuda.synchronize()
    want = normed64(q, w, eps)
    r = 2.0 ** -8 if dtype == "bf16" else U
    assert bool((out[1:3] == 0).all()) and bool((out[4, 1] == 0).all())
    assert bool(((out.double() - want).abs() <= (4 * U + r) * want.abs() + 2.0 ** -149).all())


def test_norm_rotate_of_zeros_without_eps():
    import torch
    log("case: norm_rotate of zeros, eps 0")
    pk = PK()
    out, _ = pk.norm_rotate(torch.zeros(2, 1, D, device="cuda"), None, _i32([0] * 2), pk.pair_axes((64,)), 1e4, None, None, 0.0)
    torch.cuda.synchronize()
    assert bool(out.isnan().all()) and math.isnan(float(normed64(torch.zeros(1, D), None, 0.0)[0, 0]))

"""Gradients that are sums over many rows, in float: the error of the sum stays a few roundings of the result, however many rows there are.

Independent terms of variance v: a sum of M of them has the variance M v.  A rounding to 32 bits of a value x is off by at most 2^-24 |x|, evenly, so by U |x| in the root mean
square, with U = 2^-24 / sqrt(3).  Partial sums that cover the rows once and are rounded once each add U^2 M v to the variance of the error, as the
rounding of the result does, and terms with an error of k roundings of their own k^2 U^2 M v.  A float sum of n terms in a row adds about n / 2 times U^2 M v."""
import math

import pytest

torch = pytest.importorskip("torch")
from test_gpu_dropout import Drop  # noqa: E402

pytestmark = pytest.mark.gpu
FLOAT = torch.float32
U = 2.0 ** -24 / math.sqrt(3)


def _rms(x):
    return x.double().square().mean().sqrt().item()


# The terms are the kernel's own din, float as they were added.  Four of them in 32 bits (sums of two, three and four: 9 / 4), a partial sum for every
# workgroup, the result: sqrt(9 / 4 + 2) = 2.1 roundings, and a quarter more for the columns that there are.
@pytest.mark.parametrize("M,N", [(65536, 12288), (131072, 4096), (200000, 520)])
def test_bias_gradient(M, N):
    d = Drop(3, N, 0.1, FLOAT, bias=False, resid=False)
    g = torch.Generator(device="cuda").manual_seed(M)
    dout = torch.randn(M, N, generator=g, device="cuda")
    din, ws = torch.empty_like(dout), torch.empty(d.pkg.tp_layer_dropout_workspace_bytes(M, N), dtype=torch.uint8, device="cuda")
    d.pkg.tp_layer_dropout_bwd(d.dt, M, N, 0.1, d.rng, 7, 0, 0, N, dout, din, d.dbias, ws, stream=torch.cuda.current_stream())
    want = torch.zeros(N, dtype=torch.float64, device="cuda")
    for m in range(0, M, 8192):
        want += din[m:m + 8192].double().sum(0)
    off = _rms(d.dbias.double() - want) / (U * _rms(want))
    assert off <= 1.25 * math.sqrt(9 / 4 + 2), off

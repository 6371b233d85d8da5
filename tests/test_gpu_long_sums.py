"""Gradients that are sums over many rows, in float: the error of the sum stays a few roundings of the result, however many rows there are.

Independent terms of variance v: a sum of M of them has the variance M v.  A rounding to 32 bits of a value x is off by at most 2^-24 |x|, evenly, so by U |x| in the root mean
square, with U = 2^-24 / sqrt(3).  Partial sums that cover the rows once and are rounded once each add U^2 M v to the variance of the error, as the
rounding of the result does, and terms with an error of k roundings of their own k^2 U^2 M v.  A float sum of n terms in a row adds about n / 2 times U^2 M v."""
import math

import pytest

torch = pytest.importorskip("torch")
from test_gpu_dropout import Drop  # noqa: E402
from test_gpu_qk_norm_rope import Norm  # noqa: E402

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


# A term g xh: rstd (half the error of the mean of squares, one rounding, and 1 / sqrt to a step, so two), xh and the product one each, g a sum of two products with
# a sine and a cosine to two roundings each (4 + 1 + 1): k^2 <= 1 + 4 + 1 + 1 + 6 = 13.  Partial sums of a thread and of a workgroup, the result: sqrt(13 + 3) = 4
# roundings, and a quarter more.
@pytest.mark.parametrize("per_head", [True, False])
def test_weight_gradients(per_head):
    M, nq, nkv, dh, rot = 200000, 16, 16, 64, 32
    n = Norm(8, nq, nkv, dh, rot, False, per_head, FLOAT)
    g = torch.Generator(device="cuda").manual_seed(5)
    n.shape = (M, nq, nkv, dh, rot)
    n.qkv, n.dqkv = (torch.randn(M, (nq + 2 * nkv) * dh, generator=g, device="cuda") for _ in range(2))
    n.pos_gpu = torch.randint(0, 4096, (M,), generator=g, device="cuda", dtype=torch.int32)
    n.dout = torch.empty_like(n.dqkv)
    n.ws = torch.empty(n.pkg.tp_layer_qk_norm_rope_workspace_bytes(n.dt, M, nq, nkv, dh), dtype=torch.uint8, device="cuda")
    n.backward()
    heads, h = nq + nkv, rot // 2
    want = torch.zeros(heads, dh, dtype=torch.float64, device="cuda")
    for m in range(0, M, 5000):
        x, up = (t[m:m + 5000].view(-1, heads + nkv, dh)[:, :heads].double() for t in (n.qkv, n.dqkv))
        a = n.pos_gpu[m:m + 5000].double()[:, None] * n.on_gpu
        c, s = n.factor * a.cos()[:, None], n.factor * a.sin()[:, None]
        u, v = up[..., :h].clone(), up[..., h:rot].clone()
        up[..., :h], up[..., h:rot] = u * c + v * s, v * c - u * s
        want += (up * x / (x.square().mean(-1, keepdim=True) + n.eps).sqrt()).sum(0)
    for got, part in ((n.dq, want[:nq]), (n.dk, want[nq:])):
        part = part if per_head else part.sum(0, keepdim=True)
        off = _rms(got.double() - part) / (U * _rms(part))
        assert off <= 1.25 * 4, off

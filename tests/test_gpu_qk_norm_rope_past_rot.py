"""Norms of heads with the rotation: columns past the turned ones are not turned by an angle of zero but left alone, whatever is beside them."""
import math

import pytest

torch = pytest.importorskip("torch")
from test_gpu_qk_norm_rope import Norm  # noqa: E402

pytestmark = pytest.mark.gpu
BF16, FLOAT = torch.bfloat16, torch.float32
# the last turned pair ends a unit of 16 bytes, lies inside one, is alone in the head; heads that are no power of two of units
SIZES = [(64, 32), (64, 36), (128, 2), (80, 20), (24, 10), (104, 96)]


def _run(dh, rot, adjacent, per_head, dtype):
    n = Norm(30, 2, 1, dh, rot, adjacent, per_head, dtype)
    n.run()
    n.check()
    return n


# An infinity in a head: rstd is 0, so the head's other columns are 0 and only its own is NaN.
@pytest.mark.parametrize("dtype", [BF16, FLOAT])
@pytest.mark.parametrize("adjacent", [True, False])
@pytest.mark.parametrize("dh,rot", SIZES)
def test_forward(dh, rot, adjacent, dtype):
    n = _run(dh, rot, adjacent, False, dtype)
    for col in sorted({rot, rot + 1, dh - 2, dh - 1}):
        want = n.out.clone().view(30, 4, dh)
        keep = n.qkv.view(30, 4, dh)[7, 1, col].item()
        n.qkv.view(30, 4, dh)[7, 1, col] = math.inf
        n.forward()
        n.qkv.view(30, 4, dh)[7, 1, col] = keep
        want[7, 1] = 0.0
        got = n.out.view(30, 4, dh)
        assert torch.isnan(got[7, 1, col]), col
        got[7, 1, col] = 0.0
        assert torch.equal(got, want), col
        n.forward()


# An infinite upstream gradient of a column reaches dgamma of that column and of no other (g of the others is as it was).
@pytest.mark.parametrize("dtype", [BF16, FLOAT])
@pytest.mark.parametrize("adjacent,per_head", [(True, False), (True, True), (False, False)])
@pytest.mark.parametrize("dh,rot", SIZES)
def test_backward(dh, rot, adjacent, per_head, dtype):
    n = _run(dh, rot, adjacent, per_head, dtype)
    dq, dk, dout = n.dq.clone(), n.dk.clone(), n.dout.clone().view(30, 4, dh)
    for bad in (math.inf, math.nan):
        for col in sorted({rot, rot + 1, dh - 2, dh - 1}):
            keep = n.dqkv.view(30, 4, dh)[9, 1, col].item()
            n.dqkv.view(30, 4, dh)[9, 1, col] = bad
            n.backward()
            n.dqkv.view(30, 4, dh)[9, 1, col] = keep
            others = torch.arange(dh, device="cuda") != col
            assert torch.equal(n.dq[:, others], dq[:, others]) and torch.equal(n.dk, dk), (bad, col)
            assert not torch.isfinite(n.dq[-1, col]), (bad, col)
            heads = torch.ones(30, 4, dtype=torch.bool, device="cuda")
            heads[9, 1] = False
            assert torch.equal(n.dout.view(30, 4, dh)[heads], dout[heads]), (bad, col)


# A weight that is not finite, in a column that is not turned: that column of every head, and no other.
@pytest.mark.parametrize("dtype", [BF16, FLOAT])
@pytest.mark.parametrize("dh,rot", SIZES)
def test_weights(dh, rot, dtype):
    n = _run(dh, rot, True, False, dtype)
    want = n.out.clone().view(30, 4, dh)
    for col in sorted({rot, dh - 1}):
        keep = n.gq[0, col].item()
        n.gq[0, col] = math.nan
        n.forward()
        n.gq[0, col] = keep
        others = torch.arange(dh, device="cuda") != col
        got = n.out.view(30, 4, dh)
        assert torch.equal(got[:, :, others], want[:, :, others]) and torch.isnan(got[:, :2, col]).all(), col

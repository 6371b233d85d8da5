"""Loss of a vocabulary shard: what lies beside x and w in memory, and what a workspace held, does not come into the results; a token that is not finite
stays with itself (but for dw, a sum over all)."""
import math

import pytest

torch = pytest.importorskip("torch")
from test_gpu_lm_loss import Shards  # noqa: E402

pytestmark = pytest.mark.gpu
SIZES = [(1, 8, 1), (37, 72, 1001), (130, 520, 257), (300, 136, 2055), (129, 64, 65)]


def _among_nan(t):
    """The same values, with a row of NaN before and behind them."""
    big = torch.full((t.shape[0] + 2, t.shape[1]), math.nan, dtype=t.dtype, device=t.device)
    big[1:-1] = t
    return big[1:-1]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,H,V", SIZES)
def test_neighbours(M, H, V, dtype):
    s = Shards(M, H, V, 1, dtype, ignored=0.2 if M > 1 else 0.0)
    s.run()
    first = [t.clone() for t in (s.loss, s.lse, s.dx[0], s.dw)]
    s.x, s.w, s.dw, s.dx = _among_nan(s.x), _among_nan(s.w), _among_nan(s.dw), [_among_nan(s.dx[0])]
    s.ws.fill_(255)
    s.run()
    torch.cuda.synchronize()
    assert all(torch.isfinite(t).all() for t in first)
    assert all(torch.equal(a, b) for a, b in zip(first, (s.loss, s.lse, s.dx[0], s.dw)))
    for t, n in ((s.dx[0], M), (s.dw, V)):                             # and what is beside the outputs is left alone
        assert torch.isnan(t.as_strided((H,), (1,), t.storage_offset() - H)).all() and torch.isnan(t.as_strided((H,), (1,), t.storage_offset() + n * H)).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,H,V", SIZES[1:])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_one_token_that_is_not_finite(bad, M, H, V, dtype):
    s = Shards(M, H, V, 1, dtype, ignored=0.0)
    s.run()
    first = [t.clone() for t in (s.loss, s.lse, s.dx[0])]
    s.x[5] = bad
    s.run()
    torch.cuda.synchronize()
    others = torch.arange(M, device="cuda") != 5
    assert not torch.isfinite(s.loss[5]) and not torch.isfinite(s.dx[0][5].float()).any()
    assert all(torch.equal(a[others], b[others]) for a, b in zip(first, (s.loss, s.lse, s.dx[0])))

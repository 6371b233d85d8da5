"""Float attention of many short sequences beside a longer one whose strips are cut: its chunks, of as few tiles as a short strip, go through the
workgroups that have a wavefront to each quarter, and leave sums that are joined afterwards.  Against the definition in 64 bits; the workspace is
filled with 0xFF (NaN) before."""
import math

import pytest

torch = pytest.importorskip("torch")
import packed_ref as ref  # noqa: E402
from test_gpu_packed_attention import Batch, _run  # noqa: E402

pytestmark = pytest.mark.gpu


# Enough short sequences that a wavefront has a quarter to itself (sequences * key heads over three quarters of 256, 512, 1024 units at once), few
# enough tiles that strips of five or more are cut into chunks of three.
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("count,short,longer,nq,nkv,dh", [
    (7, 64, 320, 32, 32, 128), (25, 40, 300, 8, 8, 128), (200, 30, 300, 1, 1, 128), (28, 20, 300, 8, 8, 128), (60, 30, 320, 8, 8, 96), (48, 15, 300, 8, 8, 64),
    (26, 20, 290, 16, 8, 128)])
def test_one_longer_sequence(count, short, longer, nq, nkv, dh, causal):
    _run([short] * count + [longer], nq, nkv, dh, causal, torch.float32, behind=1)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dh,count", [(64, 50), (96, 27), (128, 26)])
@pytest.mark.parametrize("longer", [257, 319, 321, 384, 385, 449, 513, 577, 640])
def test_lengths_of_the_longer_one(dh, count, longer, causal):
    _run([31] * (count // 2) + [longer] + [24] * (count - count // 2), 8, 8, dh, causal, torch.float32)


# What the causal mask hides in the longer sequence: chunks are worked out again row by row before they are joined.
@pytest.mark.parametrize("dh,count", [(64, 50), (96, 27), (128, 26)])
@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_hidden_values_in_the_longer_one(dh, count, bad):
    nq, nkv, longer, cut = 8, 8, 320, 290
    b = Batch([20] * count + [longer], nq, nkv, dh, True, torch.float32)
    val, tol = ref.attention(b.qkv, b.offsets, nq, nkv, dh, True, b.d_o)
    a = 20 * count
    b.qkv.view(b.M, nq + 2 * nkv, dh)[a + cut:, nq:] = bad              # K and V of the later tokens
    b.make_plan()
    b.run()
    for k in ("o", "lse"):
        ref.check(b.outputs()[k][:a + cut], val[k][:a + cut], tol[k][:a + cut], k)
    ref.check(b.dqkv[:a], val["dqkv"][:a], tol["dqkv"][:a], "dqkv")
    ref.check(b.dqkv[a:a + cut, :nq * dh], val["dqkv"][a:a + cut, :nq * dh], tol["dqkv"][a:a + cut, :nq * dh], "dq")

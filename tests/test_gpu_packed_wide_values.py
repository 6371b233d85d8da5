"""The backward pass of packed attention in bf16 with four wavefronts to a strip above head size 64: every element of a full chip's batch against 64 bits, and values that
are not finite behind a window's edges.  Batches have 342 strips and more, from which on this form is taken."""
import math

import pytest

torch = pytest.importorskip("torch")
import window_ref as ref  # noqa: E402
from test_gpu_packed_attention import _run  # noqa: E402
from test_gpu_packed_wide_forms import _strips  # noqa: E402
from test_gpu_window_attention import Batch, check  # noqa: E402
from test_gpu_window_attention import _run as _run_window  # noqa: E402

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
FULL = [700, 129, 3, 1000, 64]


# Several workgroups share a unit: the last rows of a sequence, whose gradients are small, have bounds of their own.
@pytest.mark.parametrize("nq,nkv,dh,causal", [(32, 32, 128, True), (32, 8, 96, True), (32, 32, 128, False)])
def test_a_full_chip(nq, nkv, dh, causal):
    assert _strips(FULL, nq, nkv) >= 342
    _run(FULL, nq, nkv, dh, causal, BF16, behind=2)


@pytest.mark.parametrize("window,sinks", [(200, 4), (64, 0)])
def test_a_full_chip_with_a_window(window, sinks):
    _run_window(FULL, 32, 8, 128, window, sinks, BF16, behind=2)


# Keys that no row of a tile's other half sees: rows that do not see them are as they were.
@pytest.mark.parametrize("dh", [96, 128])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("window,sinks,spoilt", [(30, 4, range(40, 50)), (100, 0, range(0, 20)), (20, 70, range(100, 110)), (64, 1, range(1, 64)), (5, 0, range(130, 131))])
def test_hidden_keys_do_not_matter(dh, bad, window, sinks, spoilt):
    nq, nkv, n, lengths = 32, 8, 200, [200, 90, 800]
    assert _strips(lengths, nq, nkv) >= 342
    b = Batch(lengths, nq, nkv, dh, window, sinks, BF16, behind=2)
    val, tol = b.expected()
    b.qkv.view(b.M, nq + 2 * nkv, dh)[spoilt.start:spoilt.stop, nq:] = bad          # K and V
    b.make_plan()
    b.run()
    reach = ref.sees(n, window, sinks)[:, list(spoilt)].any(1)                      # queries that see one of them
    well = torch.cat([(~reach).nonzero()[:, 0], torch.arange(n, b.used)])
    assert b.used - n < well.numel() < b.used
    for k in ("o", "lse"):
        check(b.outputs()[k][well], val[k][well], tol[k][well], k)
    check(b.dqkv[well][:, :nq * dh], val["dqkv"][well][:, :nq * dh], tol["dqkv"][well][:, :nq * dh], "dq")
    check(b.dqkv[n:b.used], val["dqkv"][n:b.used], tol["dqkv"][n:b.used], "dqkv")


# A query leaves the keys that it does not see alone, whatever its dO and Q hold.
@pytest.mark.parametrize("dh", [96, 128])
@pytest.mark.parametrize("window,sinks,spoilt", [(30, 0, range(40, 50)), (30, 4, range(100, 140)), (100, 0, range(0, 20)), (5, 0, range(130, 131))])
def test_hidden_queries_do_not_matter(dh, window, sinks, spoilt):
    nq, nkv, n, lengths = 32, 8, 200, [200, 5, 900]
    assert _strips(lengths, nq, nkv) >= 342
    b = Batch(lengths, nq, nkv, dh, window, sinks, BF16)
    val, tol = b.expected()
    b.d_o[spoilt.start:spoilt.stop] = math.inf
    b.qkv.view(b.M, nq + 2 * nkv, dh)[spoilt.start:spoilt.stop, :nq] = math.nan
    b.make_plan()
    b.run()
    reached = ref.sees(n, window, sinks)[list(spoilt)].any(0)                       # keys that one of them sees
    well = torch.cat([(~reached).nonzero()[:, 0], torch.arange(n, b.used)])
    assert b.used - n + 50 < well.numel() < b.used
    kv = slice(nq * dh, None)
    check(b.dqkv[well][:, kv], val["dqkv"][well][:, kv], tol["dqkv"][well][:, kv], "dk, dv")


# The same where strips are cut into chunks: those of long windows, and of first keys that all later rows see.
@pytest.mark.parametrize("dh", [96, 128])
@pytest.mark.parametrize("window,sinks", [(900, 4), (20, 300)])
def test_hidden_values_in_cut_strips(dh, window, sinks):
    nq, nkv, n = 32, 8, 1400
    assert _strips([n, 60], nq, nkv) >= 342
    b = Batch([n, 60], nq, nkv, dh, window, sinks, BF16, behind=2)
    val, tol = b.expected()
    spoilt = slice(400, 430)
    b.qkv.view(b.M, nq + 2 * nkv, dh)[spoilt, nq:] = math.inf
    b.make_plan()
    b.run()
    well = torch.ones(b.M, dtype=torch.bool)
    well[spoilt.start:spoilt.stop + window] = False
    well[b.used:] = False
    assert well.sum() > 400
    for k in ("o", "lse"):
        check(b.outputs()[k][well.cuda()], val[k][well], tol[k][well], k)
    check(b.dqkv[well.cuda()][:, :nq * dh], val["dqkv"][well][:, :nq * dh], tol["dqkv"][well][:, :nq * dh], "dq")

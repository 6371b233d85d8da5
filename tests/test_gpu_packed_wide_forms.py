"""The backward pass of packed attention in bf16 with heads of more than 64 where strips fill the chip: four wavefronts to a strip instead of eight.  Batches
here have 342 strips and more, those of the other tests of packed attention fewer."""
import math

import pytest

torch = pytest.importorskip("torch")
import packed_ref as ref  # noqa: E402
import test_gpu_window_attention as window_tests  # noqa: E402
from test_gpu_packed_attention import Batch, _run  # noqa: E402

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
SHORT, LONG = [1, 0, 63, 64, 65, 1, 130, 0], [1, 0, 63, 64, 65, 1, 130, 0, 1300]


def _strips(lengths, nq, nkv):
    return sum(lengths) * (nq + nkv) // 128 + len(lengths) * nkv


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dh", [72, 96, 104, 120, 128])
@pytest.mark.parametrize("lengths,nq,nkv", [(SHORT, 40, 40), (SHORT, 96, 16), (LONG, 24, 3)])
def test_edges(lengths, nq, nkv, dh, causal):
    assert _strips(lengths, nq, nkv) >= 342
    _run(lengths, nq, nkv, dh, causal, BF16, behind=3)


# Strips that are cut, with one long document among many short ones, and groups that are no power of two.
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("nq,nkv,dh", [(16, 2, 128), (14, 2, 96), (25, 5, 128)])
def test_cut_strips_among_many_short_ones(nq, nkv, dh, causal):
    assert _strips([1500] + [9] * 60, nq, nkv) >= 342
    _run([1500] + [9] * 60, nq, nkv, dh, causal, BF16, behind=1)


@pytest.mark.parametrize("window,sinks", [(1, 0), (63, 1), (64, 0), (65, 70), (129, 64), (500, 1), (2000, 0)])
@pytest.mark.parametrize("nq,nkv,dh", [(24, 3, 128), (20, 5, 96), (24, 3, 104)])
def test_windows(nq, nkv, dh, window, sinks):
    lengths = [1, 0, 63, 300, 65, 0, 1, 1300]
    assert _strips(lengths, nq, nkv) >= 342
    window_tests._run(lengths, nq, nkv, dh, window, sinks, BF16, behind=3)


# Keys that are hidden, and queries that do not see, in whole and in cut strips.
@pytest.mark.parametrize("dh", [96, 128])
@pytest.mark.parametrize("more", [[9] * 60, [1400]])
@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_hidden_values_do_not_matter(more, bad, dh):
    nq, nkv, n, cut = 32, 8, 1400, 40
    b = Batch([n, 90] + more, nq, nkv, dh, True, BF16)
    assert _strips([n, 90] + more, nq, nkv) >= 342
    val, tol = ref.attention(b.qkv, b.offsets, nq, nkv, dh, True, b.d_o)
    rows = b.qkv.view(b.M, nq + 2 * nkv, dh)
    rows[n - cut:n, nq:] = bad                                       # K and V of the first sequence's last tokens
    b.d_o[n:n + cut] = bad                                           # dO of the second one's first
    rows[n:n + cut, :nq] = math.nan
    b.make_plan()
    b.run()
    for k in ("o", "lse"):
        ref.check(b.outputs()[k][:n - cut], val[k][:n - cut], tol[k][:n - cut], k)
    ref.check(b.dqkv[:n - cut, :nq * dh], val["dqkv"][:n - cut, :nq * dh], tol["dqkv"][:n - cut, :nq * dh], "dq")
    ref.check(b.dqkv[n + cut:], val["dqkv"][n + cut:], tol["dqkv"][n + cut:], "dqkv")


@pytest.mark.parametrize("dh", [96, 128])
def test_results_do_not_change_from_run_to_run(dh):
    b = _run(LONG, 24, 3, dh, True, BF16)
    first = b.dqkv.clone()
    for _ in range(3):
        b.make_plan()
        b.run()
        assert torch.equal(b.dqkv, first)


# All strips at once, where several workgroups share a unit: every row against the same batch of one key head after the other.
def test_a_full_chip():
    lengths, nq, nkv, dh = [700, 129, 3, 1000, 64], 32, 32, 128
    b = Batch(lengths, nq, nkv, dh, True, BF16)
    b.make_plan()
    b.run()
    one = Batch(lengths, 1, 1, dh, True, BF16)
    one.make_plan()
    for h in range(nkv):
        one.qkv.copy_(torch.cat([b.qkv[:, (j * nq + h) * dh:(j * nq + h + 1) * dh] for j in range(3)], 1))
        one.d_o.copy_(b.d_o[:, h * dh:(h + 1) * dh])
        one.run()
        for j, name in enumerate(("dq", "dk", "dv")):
            got, want = b.dqkv[:, (j * nq + h) * dh:(j * nq + h + 1) * dh].float(), one.dqkv[:, j * dh:(j + 1) * dh].float()
            # Both are off the exact gradients by their own roundings: P and dS as operands (2^-8 each) and the result's (2^-8 of itself), of sums over up to
            # 1000 terms of either sign: 8 roundings' worth of the largest value of the head bounds the difference of two of them.
            assert (got - want).abs().max() <= 8 * 2 ** -8 * want.abs().max(), (name, h)

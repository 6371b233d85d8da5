"""Both forms of the backward pass of packed attention in bf16 with heads of up to 64: four wavefronts to a strip where strips are short, eight
where they are long, by the average length of the batch's sequences."""
import math

import pytest

torch = pytest.importorskip("torch")
import packed_ref as ref  # noqa: E402
from test_gpu_packed_attention import Batch, _run  # noqa: E402

pytestmark = pytest.mark.gpu
SHORT, LONG = [1, 0, 63, 64, 65, 1, 130, 0], [1, 0, 63, 64, 65, 1, 130, 0, 1300]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lengths", [SHORT, LONG])
@pytest.mark.parametrize("nq,nkv,dh", [(8, 1, 64), (12, 2, 32), (8, 1, 24), (16, 2, 56)])
def test_edges(nq, nkv, dh, lengths, causal):
    _run(lengths, nq, nkv, dh, causal, torch.bfloat16, behind=3)


@pytest.mark.parametrize("causal", [True, False])
def test_strips_that_fill_the_chip(causal):
    _run([520, 0, 300, 270], 64, 64, 64, causal, torch.bfloat16, behind=2)


# Strips that are cut, with one long document among many short ones: the average is short.
@pytest.mark.parametrize("causal", [True, False])
def test_cut_strips_among_many_short_ones(causal):
    _run([1500] + [9] * 60, 2, 1, 64, causal, torch.bfloat16, behind=1)


# Keys that are hidden, and queries that do not see, in whole and in cut strips of either form.
@pytest.mark.parametrize("more", [[], [9] * 60, [1400]])
@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_hidden_values_do_not_matter(more, bad):
    nq, nkv, dh, n, cut = 8, 1, 64, 1400 if more else 70, 40
    b = Batch([n, 90] + more, nq, nkv, dh, True, torch.bfloat16)
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


@pytest.mark.parametrize("lengths", [SHORT, LONG])
def test_results_do_not_change_from_run_to_run(lengths):
    b = _run(lengths, 8, 1, 64, True, torch.bfloat16)
    first = b.dqkv.clone()
    for _ in range(3):
        b.make_plan()
        b.run()
        assert torch.equal(b.dqkv, first)

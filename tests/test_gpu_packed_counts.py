"""Packed attention in bf16 counts every pair of a query and a key once.  With Q (or K) zero all scores are zero and every weight is one over the keys that
a query sees, so results are sums of a few equal terms: one left out, or taken twice, is far outside the rounding."""
import pytest

torch = pytest.importorskip("torch")
import packed_ref as ref  # noqa: E402
from test_gpu_packed_attention import Batch  # noqa: E402

pytestmark = pytest.mark.gpu
STEP = ref.HALF[torch.bfloat16]


def _one_hot(index, dh):
    return torch.nn.functional.one_hot(index % dh, dh).float()


def _batch(lengths, nq, nkv, dh, causal, q, k, v, d_o):
    """q, k, v, d_o: [n, dh] of a sequence of n tokens (every head alike; d_o: [n, group, dh])."""
    b = Batch(lengths, nq, nkv, dh, causal, torch.bfloat16)
    G = nq // nkv
    rows, up = b.qkv.view(b.M, nq + 2 * nkv, dh), b.d_o.view(b.M, nkv, G, dh)
    for a, n in zip(b.offsets, lengths):
        if n:
            rows[a:a + n, :nq], rows[a:a + n, nq:nq + nkv], rows[a:a + n, nq + nkv:] = (f(n)[:, None].to(rows) for f in (q, k, v))
            up[a:a + n] = d_o(n, G)[:, None].to(up)
    b.make_plan()
    b.run()
    torch.cuda.synchronize()
    val, _ = ref.attention(b.qkv, b.offsets, nq, nkv, dh, causal, b.d_o)
    return b, val


def _close(got, want, rel, off):
    got = got.double().cpu().reshape(want.shape)
    assert torch.isfinite(got).all() and ((got - want).abs() <= rel * want.abs() + off).all(), ((got - want).abs() / (want.abs() + 1e-9)).max()


CASES = [([1300, 5, 330, 64, 65, 1], 2, 1, 64), ([2300, 700, 129, 1], 2, 1, 128), ([1500, 31, 300], 2, 2, 80), ([900, 257, 256], 1, 1, 32), ([200] * 12, 8, 2, 64)]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lengths,nq,nkv,dh", CASES)
def test_outputs_and_values(lengths, nq, nkv, dh, causal):
    zero, hot = lambda n: torch.zeros(n, dh), lambda n: _one_hot(torch.arange(n), dh)                        # noqa: E731

    def d_o(n, G):
        # flattened row r of a group in column r, with the largest power of two in the weight's denominator: terms between 1/2 and 1
        seen = torch.arange(1, n + 1) if causal else torch.full((n,), n)
        return _one_hot(torch.arange(n * G), dh).view(n, G, dh) * (2.0 ** seen.log2().floor())[:, None, None]
    b, val = _batch(lengths, nq, nkv, dh, causal, zero, zero, hot, d_o)
    n = max(lengths)
    # O: weights 1, their sum and those of V exact, one quotient and one rounding.  dV: the weight's rounding as an operand and the output's.
    # A weight from its LSE: 2^(-l log2 e), off by 4 roundings of a number below 12.
    _close(b.o, val["o"], STEP + 8 * ref.F32, 0.0)
    _close(b.lse, val["lse"], 4 * ref.F32, 4 * ref.F32)
    dv = (nq + nkv) * dh
    _close(b.dqkv[:, dv:], val["dqkv"][:, dv:], 2 * STEP + STEP * STEP + (64 + n) * ref.F32, 0.0)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lengths,nq,nkv,dh", CASES)
@pytest.mark.parametrize("of", ["dq", "dk"])
def test_gradients_of_queries_and_keys(of, lengths, nq, nkv, dh, causal):
    first = torch.zeros(dh)
    first[0] = 1.0
    zero, hot = lambda n: torch.zeros(n, dh), lambda n: _one_hot(torch.arange(n), dh)                        # noqa: E731
    sign = lambda n: (1.0 - 2.0 * (torch.arange(n) % 2))[:, None] * first                                    # noqa: E731

    def d_o(n, G):
        seen = torch.arange(1, n + 1) if causal else torch.full((n,), n)
        return ((2.0 ** seen.log2().floor())[:, None] * first)[:, None].expand(n, G, dh)
    # dP of key j is (-1)^j times dO's scale (terms between 1/2 and 1 with the weight), D what is left of their mean: at most that of one key
    q, k = (zero, hot) if of == "dq" else (hot, zero)
    b, val = _batch(lengths, nq, nkv, dh, causal, q, k, sign, d_o)
    cols = slice(0, nq * dh) if of == "dq" else slice(nq * dh, (nq + nkv) * dh)
    n, most, G = max(lengths), 2.0 / dh ** 0.5, nq // nkv
    # dS as an operand and the output: half a step each.  D from O, which is rounded, or from weights: off by half a step of 1 / seen of its scale, so that a
    # row adds at most 2 half steps / seen of a term; over the rows of a column (dK) and its heads below 2 (1 + log n) G / dh of them, each sequence apart.
    off = most * STEP * 2 * (1 if of == "dq" else (2 + torch.tensor(float(n)).log().item()) * G) + most * (64 + n) * ref.F32 * (n / dh + 1) * G
    _close(b.dqkv[:, cols], val["dqkv"][:, cols], 2 * STEP + STEP * STEP + (64 + n) * ref.F32, off)

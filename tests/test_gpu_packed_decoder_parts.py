"""The decoder step of test_gpu_packed_decoder.py, operator by operator: every tensor against 64 bits from the tensors that it was made from, within a bound for
each element.  So an error in one gradient does not hide behind a larger one that it is added to.  Eagerly, and captured and replayed, in both types."""
import pytest

torch = pytest.importorskip("torch")
import packed_ref as ref  # noqa: E402
from test_gpu_packed_decoder import BATCHES, DH, H, M, NKV, NQ, RANKS, ROT, V, Decoder  # noqa: E402

pytestmark = pytest.mark.gpu


def _product(a, b, t, resid=None):
    """(value, bound) of a b (+ resid) with float sums and one rounding to type t."""
    a, b = a.double().cpu(), b.double().cpu()
    val, tol = a @ b, (a.shape[1] + 8) * ref.F32 * (a.abs() @ b.abs())
    if resid is not None:
        val, tol = val + resid.double().cpu(), tol + ref.F32 * resid.double().cpu().abs()
    return val, tol + ref.HALF[t] * (val.abs() + tol)


def _turned(val, tol, t, positions, freq, back):
    """(value, bound) of rows of a given value and bound, turned and rounded to type t: see ref.rotary."""
    out, e = val.view(M, NQ + 2 * NKV, DH).clone(), tol.view(M, NQ + 2 * NKV, DH).clone()
    angle = positions.double()[:, None] * torch.tensor(freq, dtype=torch.float64)
    c, s = angle.cos()[:, None], (angle.sin() * (-1 if back else 1))[:, None]
    first, second = slice(0, ROT // 2), slice(ROT // 2, ROT)
    heads = slice(0, NQ + NKV)
    u, v = out[:, heads, first].clone(), out[:, heads, second].clone()
    more = e[:, heads, first] + e[:, heads, second] + 8 * ref.F32 * (u.abs() + v.abs())
    out[:, heads, first], out[:, heads, second] = u * c - v * s, u * s + v * c
    e[:, heads, first], e[:, heads, second] = more, more
    e[:, heads, :ROT] += ref.HALF[t] * (out[:, heads, :ROT].abs() + e[:, heads, :ROT])
    return out.reshape(M, -1), e.reshape(M, -1)


def _check_parts(d):
    t, used = d.dtype, sum(d.lengths)
    at, offsets = 0, [0]
    positions = torch.zeros(M, dtype=torch.int32)
    for n in d.lengths:
        positions[at:at + n] = torch.arange(n, dtype=torch.int32)
        at += n
        offsets.append(at)
    assert torch.equal(d.positions.cpu(), positions)
    val, tol = _turned(*_product(d.x, d.w_qkv, t), t, positions, d.freq_list, False)
    ref.check(d.qkv, val, tol, "qkv")
    val, tol = ref.attention(d.qkv, offsets, NQ, NKV, DH, True, d.do)
    ref.check(d.o, val["o"], tol["o"], "o")
    ref.check(d.lse, val["lse"], tol["lse"], "lse")
    assert (d.o[used:] == 0).all() and (d.dqkv[used:] == 0).all()
    g, e = _turned(torch.nan_to_num(val["dqkv"]), torch.nan_to_num(tol["dqkv"]), t, positions, d.freq_list, True)
    ref.check(d.dqkv[:used], g[:used], e[:used], "dqkv")
    ref.check(d.y, *_product(d.o, d.w_o, t, d.x), "y")
    for r in range(RANKS):
        rows = slice(r * V, (r + 1) * V)
        val, tol = ref.loss(d.y, d.w_out[rows], d.labels, r * V, RANKS * V, d.zlse, d.dloss)
        ref.check(d.stats[r, :, 0], val["lse"], tol["lse"], "stats")
        ref.check(d.dy_part[r], val["dx"], tol["dx"], "dy_part")
        ref.check(d.dw_out[rows], val["dw"], tol["dw"], "dw_out")
    both = d.dy_part.double().cpu()
    ref.check(d.dy, both.sum(0), ref.F32 * both.abs().sum(0) + ref.HALF[t] * both.sum(0).abs() * (1 + ref.F32), "dy")
    ref.check(d.dw_o, *_product(d.o.t(), d.dy, t), "dw_o")
    ref.check(d.do, *_product(d.dy, d.w_o.t(), t), "do")
    ref.check(d.dw_qkv, *_product(d.x.t(), d.dqkv, t), "dw_qkv")
    ref.check(d.dx, *_product(d.dqkv, d.w_qkv.t(), t, d.dy), "dx")


@pytest.mark.parametrize("lengths", BATCHES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_parts(dtype, lengths):
    d = Decoder(dtype)
    d.batch(lengths, seed=1 + sum(lengths))
    d.step()
    torch.cuda.synchronize()
    _check_parts(d)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_captured_parts(dtype):
    d = Decoder(dtype)
    d.batch(BATCHES[0], seed=1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        d.step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        d.step()
    for seed, lengths in enumerate(BATCHES):
        d.batch(lengths, seed)
        graph.replay()
        torch.cuda.synchronize()
        _check_parts(d)
        d.check()
        got = {k: x.clone() for k, x in d.outputs().items()}
        d.step()
        torch.cuda.synchronize()
        assert all(torch.equal(got[k], x) for k, x in d.outputs().items())

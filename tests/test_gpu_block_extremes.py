"""Norms with the rotation at the largest numbers of heads, and dropout of rows so wide that one workgroup has all rows of its columns."""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_dropout import Drop  # noqa: E402
from test_gpu_qk_norm_rope import _run  # noqa: E402

pytestmark = pytest.mark.gpu
BF16, FLOAT = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF16, FLOAT])
@pytest.mark.parametrize("per_head", [False, True])
@pytest.mark.parametrize("M,nq,nkv,dh,rot,adjacent", [(2, 4096, 4096, 8, 8, True), (2, 4096, 3, 16, 6, False), (1, 4096, 1, 512, 512, False), (3, 1, 4096, 64, 30, True)])
def test_many_heads(M, nq, nkv, dh, rot, adjacent, per_head, dtype):
    _run(M, nq, nkv, dh, rot, adjacent, per_head, dtype)


# dbias without a workspace's sums: the rows of a strip of columns in one workgroup.  din is checked by its mask in the other tests, and is what dbias adds: sums of
# 70 terms, of float in 64 bits after four in 32 and rounded once (4 roundings of sums of up to four terms, one of the result), of bf16 in 32 (its terms unrounded, din rounded).
@pytest.mark.parametrize("dtype", [BF16, FLOAT])
def test_wide_rows(dtype):
    M, N = 70, (1 << 20) + 512
    d = Drop(2, 8, 0.25, dtype, width=N)
    g = torch.Generator(device="cuda").manual_seed(1)
    dout = torch.randn(M, N, generator=g, device="cuda").to(dtype)
    din, dbias = torch.empty_like(dout), torch.empty(N, dtype=dtype, device="cuda")
    ws = torch.empty(d.pkg.tp_layer_dropout_workspace_bytes(M, N), dtype=torch.uint8, device="cuda")
    assert ws.numel() < 2 * 4 * N
    d.pkg.tp_layer_dropout_bwd(d.dt, M, N, 0.25, d.rng, 1, 0, 0, N, dout, din, dbias, ws, stream=torch.cuda.current_stream())
    x = torch.where(din != 0, dout.double() / 0.75, 0.0)
    want, size = x.sum(0), x.abs().sum(0)
    f32, half = 2.0 ** -24, 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
    # a product and, of float, three sums of four terms; of bf16 a chain of 70
    e = (5 if dtype == FLOAT else 72) * f32 * size
    assert ((dbias.double() - want).abs() <= e + half * (want.abs() + e)).all()
    parts = [(0, 520), (N // 2, 1032), (N - 512, 512)]
    for c, n in parts:                                             # the mask of the whole, by columns
        o = torch.empty(M, n, dtype=dtype, device="cuda")
        d.pkg.tp_layer_dropout_bwd(d.dt, M, n, 0.25, d.rng, 1, 0, c, N, dout[:, c:c + n].contiguous(), o, stream=torch.cuda.current_stream())
        assert torch.equal(o, din[:, c:c + n])

"""Rotary positions against their definition in 64 bits."""
import pytest

torch = pytest.importorskip("torch")
import packed_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu


def _case(seed, M, nq, nkv, dh, dtype):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(M, (nq + 2 * nkv) * dh, generator=g).to(dtype).cuda()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("M,nq,nkv,dh,rot", [(1, 1, 1, 64, 64), (5, 3, 1, 80, 32), (130, 8, 2, 128, 128), (2500, 4, 4, 64, 16), (33, 2, 2, 8, 2),
                                             (7, 2, 1, 20, 10), (3, 2, 1, 4, 4), (9, 1, 1, 256, 256), (64, 40, 8, 96, 48)])
def test_both_directions(M, nq, nkv, dh, rot, adjacent, dtype):
    import paper_2111_05972_amd as pkg
    dt = pkg.TPL_BF16 if dtype == torch.bfloat16 else pkg.TPL_F32
    pairs = pkg.TPL_ROPE_ADJACENT if adjacent else pkg.TPL_ROPE_HALF
    x = _case(M, M, nq, nkv, dh, dtype)
    freq, factor = pkg.tp_layer_rope_frequencies(rot, 10000.0, pkg.TPL_ROPE_PARTS, 8.0, 4096.0)
    on_gpu = torch.tensor(freq, dtype=torch.float64, device="cuda")
    pos = torch.randint(-2 ** 31, 2 ** 31 - 1, (M,), generator=torch.Generator().manual_seed(3)).to(torch.int32)
    pos[::2] = torch.arange(M, dtype=torch.int32)[::2]
    st = torch.cuda.current_stream()
    # the angle: position (31 bits) times frequency and its whole turns in 64 bits, 2^31 * 2^-52 of a radian off at most
    far = 2.0 ** -20
    for back, call in ((False, pkg.tp_layer_rope_fwd), (True, pkg.tp_layer_rope_bwd)):
        out = torch.full_like(x, 7.0)
        call(dt, M, nq, nkv, dh, rot, pairs, on_gpu, factor, pos.cuda(), x, out, stream=st)
        val, tol = ref.rotary(x, nq, nkv, dh, rot, adjacent, pos, freq, factor, back)
        ref.check(out, val, tol + far * factor * 8, "out")
        plain = torch.ones(nq + 2 * nkv, dh, dtype=torch.bool)
        plain[:nq + nkv, :rot] = False
        assert torch.equal(out[:, plain.view(-1).cuda()], x[:, plain.view(-1).cuda()])
        again = x.clone()
        call(dt, M, nq, nkv, dh, rot, pairs, on_gpu, factor, pos.cuda(), again, again, stream=st)
        assert torch.equal(again, out), "in place"


def test_rows_of_a_batch_are_positions():
    import paper_2111_05972_amd as pkg
    B, S, nq, nkv, dh = 3, 50, 4, 4, 64
    x = _case(1, B * S, nq, nkv, dh, torch.bfloat16)
    freq, factor = pkg.tp_layer_rope_frequencies(dh)
    on_gpu = torch.tensor(freq, dtype=torch.float64, device="cuda")
    a, b = torch.empty_like(x), torch.empty_like(x)
    st = torch.cuda.current_stream()
    pkg.tp_layer_rope_fwd(pkg.TPL_BF16, B * S, nq, nkv, dh, dh, pkg.TPL_ROPE_HALF, on_gpu, factor, None, x, a, seq=S, stream=st)
    pos = torch.arange(B * S, dtype=torch.int32, device="cuda") % S
    pkg.tp_layer_rope_fwd(pkg.TPL_BF16, B * S, nq, nkv, dh, dh, pkg.TPL_ROPE_HALF, on_gpu, factor, pos, x, b, stream=st)
    assert torch.equal(a, b)


# backward is the transpose of forward: <turn x, y> = <x, turn back y>
def test_backward_is_the_transpose():
    import paper_2111_05972_amd as pkg
    M, nq, nkv, dh, rot = 20, 3, 1, 64, 48
    x, y = _case(1, M, nq, nkv, dh, torch.float32), _case(2, M, nq, nkv, dh, torch.float32)
    freq, factor = pkg.tp_layer_rope_frequencies(rot, 1e4, pkg.TPL_ROPE_PARTS, 4.0, 2048.0)
    on_gpu = torch.tensor(freq, dtype=torch.float64, device="cuda")
    u, v = torch.empty_like(x), torch.empty_like(y)
    args = (pkg.TPL_F32, M, nq, nkv, dh, rot, pkg.TPL_ROPE_ADJACENT, on_gpu, factor, None)
    pkg.tp_layer_rope_fwd(*args, x, u, seq=M, stream=torch.cuda.current_stream())
    pkg.tp_layer_rope_bwd(*args, y, v, seq=M, stream=torch.cuda.current_stream())
    a, b = (u.double() * y.double()), (x.double() * v.double())
    assert abs(a.sum() - b.sum()) <= 16 * ref.F32 * factor * 2 * a.abs().sum().item()

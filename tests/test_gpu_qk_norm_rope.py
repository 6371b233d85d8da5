"""Norms of query and key heads with the rotation against their definition in 64 bits, forward and backward."""
import math

import pytest

torch = pytest.importorskip("torch")
import block_ref  # noqa: E402
from packed_ref import F32, check  # noqa: E402

pytestmark = pytest.mark.gpu
BF16, FLOAT = torch.bfloat16, torch.float32


class Norm:
    """Inputs of a call, outputs filled with 7."""

    def __init__(self, M, nq, nkv, dh, rot, adjacent, per_head, dtype, seed=0, eps=1e-6, factor=1.25, far=False):
        import paper_2111_05972_amd as pkg
        g = torch.Generator().manual_seed(seed + M + 1000 * dh)
        make = lambda *s, sigma=1.0, mean=0.0: (torch.randn(*s, generator=g) * sigma + mean).to(dtype).cuda()     # noqa: E731
        self.pkg, self.dt = pkg, pkg.TPL_BF16 if dtype == BF16 else pkg.TPL_F32
        self.shape, self.per_head, self.eps, self.factor = (M, nq, nkv, dh, rot), per_head, eps, factor
        self.adjacent = adjacent
        self.qkv, self.dqkv = make(M, (nq + 2 * nkv) * dh, sigma=1.7), make(M, (nq + 2 * nkv) * dh)
        self.gq, self.gk = (make(n if per_head else 1, dh, sigma=0.3, mean=1.0) for n in (nq, nkv))
        self.freq = [10000.0 ** (-2.0 * i / rot) for i in range(rot // 2)]
        self.on_gpu = torch.tensor(self.freq, dtype=torch.float64, device="cuda")
        top = 2 ** 31 - 1 if far else 100000
        self.pos = torch.randint(-top if far else 0, top, (M,), generator=g).to(torch.int32)
        self.pos_gpu = self.pos.cuda()
        self.out, self.dout = torch.full_like(self.qkv, 7.0), torch.full_like(self.qkv, 7.0)
        self.dq, self.dk = torch.full_like(self.gq, 7.0), torch.full_like(self.gk, 7.0)
        self.ws = torch.full((pkg.tp_layer_qk_norm_rope_workspace_bytes(self.dt, M, nq, nkv, dh),), 255, dtype=torch.uint8, device="cuda")

    def args(self):
        p = self.pkg
        return (self.dt, *self.shape, p.TPL_ROPE_ADJACENT if self.adjacent else p.TPL_ROPE_HALF, self.on_gpu, self.factor, self.pos_gpu, self.gq, self.gk,
                self.per_head, self.eps)

    def forward(self, out=None):
        self.pkg.tp_layer_qk_norm_rope_fwd(*self.args(), self.qkv, self.out if out is None else out, stream=torch.cuda.current_stream())

    def backward(self, up=None, out=None):
        self.pkg.tp_layer_qk_norm_rope_bwd(*self.args(), self.qkv, self.dqkv if up is None else up, self.dout if out is None else out, self.dq, self.dk, self.ws,
                                           stream=torch.cuda.current_stream())

    def run(self):
        self.forward()
        self.backward()

    def outputs(self):
        return {"out": self.out, "dout": self.dout, "dgamma_q": self.dq, "dgamma_k": self.dk}

    def check(self):
        M, nq, nkv, dh, rot = self.shape
        val, tol = block_ref.norm(self.qkv, nq, nkv, dh, rot, self.adjacent, self.pos, self.freq, self.factor, self.gq, self.gk, self.per_head, self.eps, self.dqkv)
        for k, x in self.outputs().items():
            check(x.view(val[k].shape), val[k], tol[k], k)


def _run(*args, **kw):
    n = Norm(*args, **kw)
    n.run()
    n.check()
    v = n.shape[3] * (n.shape[1] + n.shape[2])
    assert torch.equal(n.out[:, v:], n.qkv[:, v:]) and torch.equal(n.dout[:, v:], n.dqkv[:, v:])
    return n


# whole units of 16 bytes in the halves of a rotation, and others; one lane to a head up to a wavefront
SIZES = [(1, 1, 1, 64, 64), (5, 3, 1, 80, 32), (130, 8, 2, 128, 128), (700, 4, 4, 64, 16), (33, 2, 2, 8, 2), (33, 2, 1, 8, 8), (7, 2, 1, 24, 10), (9, 1, 1, 256, 256),
         (64, 40, 8, 96, 48), (31, 5, 1, 104, 104), (31, 5, 5, 104, 26), (17, 3, 3, 80, 20), (3, 1, 1, 512, 512), (3, 2, 1, 512, 36), (2000, 1, 1, 32, 8), (600, 12, 12, 32, 32)]


@pytest.mark.parametrize("dtype", [BF16, FLOAT])
@pytest.mark.parametrize("adjacent,per_head", [(False, False), (True, False), (False, True), (True, True)])
@pytest.mark.parametrize("M,nq,nkv,dh,rot", SIZES)
def test_both_directions(M, nq, nkv, dh, rot, adjacent, per_head, dtype):
    _run(M, nq, nkv, dh, rot, adjacent, per_head, dtype)


@pytest.mark.parametrize("dtype", [BF16, FLOAT])
@pytest.mark.parametrize("adjacent", [False, True])
def test_far_positions(adjacent, dtype):
    _run(50, 2, 1, 64, 48, adjacent, False, dtype, far=True)


# many heads to a row: several passes over them, in which a workgroup's heads do not divide
@pytest.mark.parametrize("dtype", [BF16, FLOAT])
@pytest.mark.parametrize("rot", [128, 20])
@pytest.mark.parametrize("nq,nkv", [(64, 8), (37, 37), (100, 1), (129, 3)])
def test_many_heads(nq, nkv, rot, dtype):
    _run(40, nq, nkv, 128, rot, False, True, dtype)
    _run(41, nq, nkv, 128, rot, False, False, dtype, seed=1)


# more rows than a workgroup has angles for at a time; in one pass over the heads and in several
@pytest.mark.parametrize("per_head", [False, True])
@pytest.mark.parametrize("M,nq,dh,rot,adjacent", [(80000, 1, 64, 64, True), (80000, 1, 64, 60, False), (8300, 7, 512, 500, True), (8300, 7, 512, 500, False)])
def test_angles_in_chunks(M, nq, dh, rot, adjacent, per_head):
    _run(M, nq, 1, dh, rot, adjacent, per_head, FLOAT)


@pytest.mark.parametrize("dtype", [BF16, FLOAT])
@pytest.mark.parametrize("rot,adjacent", [(64, False), (64, True), (20, False)])
def test_in_place(rot, adjacent, dtype):
    n = _run(70, 6, 2, 64, rot, adjacent, False, dtype)
    a, b, dq = n.qkv.clone(), n.dqkv.clone(), n.dq.clone()
    n.backward(b, b)
    assert torch.equal(b, n.dout) and torch.equal(n.dq, dq)
    n.qkv = a
    n.forward(a)
    assert torch.equal(a, n.out)


def test_rows_of_a_batch_are_positions():
    B, S = 3, 50
    n = Norm(B * S, 4, 4, 64, 64, False, False, BF16)
    n.pos_gpu = torch.arange(B * S, dtype=torch.int32, device="cuda") % S
    n.run()
    got = {k: x.clone() for k, x in n.outputs().items()}
    n.pos_gpu = None
    n.pkg.tp_layer_qk_norm_rope_fwd(*n.args(), n.qkv, n.out, seq=S, stream=torch.cuda.current_stream())
    n.pkg.tp_layer_qk_norm_rope_bwd(*n.args(), n.qkv, n.dqkv, n.dout, n.dq, n.dk, n.ws, seq=S, stream=torch.cuda.current_stream())
    assert all(torch.equal(x, got[k]) for k, x in n.outputs().items())


# A row of zeros has an rstd of 1 / sqrt(eps); values that are not finite stay in their head.
@pytest.mark.parametrize("dtype", [BF16, FLOAT])
def test_zeros_and_other_heads(dtype):
    n = Norm(20, 3, 1, 64, 64, False, True, dtype)
    n.qkv[4] = 0.0
    n.run()
    n.check()
    val, tol = n.out.clone(), n.dout.clone()
    n.qkv.view(20, 5, 64)[7, 1] = math.inf
    n.dqkv.view(20, 5, 64)[8, 0] = math.nan
    n.run()
    same = torch.ones(20, 5, dtype=torch.bool, device="cuda")
    same[7, 1] = False
    assert torch.equal(n.out.view(20, 5, 64)[same], val.view(20, 5, 64)[same])
    same[8, 0] = False
    assert torch.equal(n.dout.view(20, 5, 64)[same], tol.view(20, 5, 64)[same])
    assert torch.isnan(n.dq[0]).all() and torch.isnan(n.dq[1]).any() and torch.isfinite(n.dq[2]).all() and torch.isfinite(n.dk).all()


def test_results_do_not_change_from_run_to_run():
    n = _run(3000, 5, 1, 64, 64, True, False, BF16)
    first = {k: x.clone() for k, x in n.outputs().items()}
    for _ in range(3):
        n.ws.fill_(255)
        n.run()
        assert all(torch.equal(x, first[k]) for k, x in n.outputs().items())


@pytest.mark.parametrize("rot,adjacent,per_head", [(16, False, False), (16, True, True), (6, False, True)])
def test_gradient_against_differences(rot, adjacent, per_head):
    n = Norm(3, 2, 1, 16, rot, adjacent, per_head, FLOAT)
    n.run()
    step, up = 2.0 ** -6, n.dqkv.double()

    def value():
        n.forward()
        return (n.out.double() * up).sum().item()
    # values of about one, slopes of rstd of about one: fifth derivatives below 1000; float outputs' rounding over the step
    tol = 1000 * step ** 4 / 30 + 64 * F32 * float((n.out.double().abs() * up.abs()).sum()) / step
    for x, d, at in ((n.qkv, n.dout, [(0, 0), (1, 17), (2, 33), (2, 47), (0, 60)]), (n.gq, n.dq, [(0, 3), (0, 15)]), (n.gk, n.dk, [(0, 9)])):
        for i, j in at:
            keep, f = x[i, j].item(), []
            for k in (1, -1, 2, -2):
                x[i, j] = keep + k * step
                f.append(value())
            x[i, j] = keep
            diff = (8 * (f[0] - f[1]) - (f[2] - f[3])) / (12 * step)
            assert abs(diff - d[i, j].item()) <= tol, (i, j, diff, d[i, j].item())


def test_captured_and_on_another_stream():
    n = Norm(300, 4, 2, 64, 64, False, False, BF16)
    n.run()
    want = {k: x.clone() for k, x in n.outputs().items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        n.run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        n.run()
    for i in range(3):
        for x in n.outputs().values():
            x.fill_(7.0)
        n.ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, want[k]) for k, x in n.outputs().items())
        n.run()


# Rows past 2^31 bytes and 2^31 elements
def test_a_long_batch():
    M, nq, nkv, dh, tail = 700000, 24, 4, 128, 40
    n = Norm(tail, nq, nkv, dh, dh, False, False, BF16)
    rows = torch.zeros(M, (nq + 2 * nkv) * dh, dtype=BF16, device="cuda")
    up = torch.zeros_like(rows)
    rows[-tail:], up[-tail:] = n.qkv, n.dqkv
    n.qkv, n.dqkv, n.pos_gpu = rows, up, torch.cat([torch.zeros(M - tail, dtype=torch.int32), n.pos]).cuda()
    n.shape = (M, nq, nkv, dh, dh)
    n.out, n.dout = torch.empty_like(rows), torch.empty_like(rows)
    n.ws = torch.empty(n.pkg.tp_layer_qk_norm_rope_workspace_bytes(n.dt, M, nq, nkv, dh), dtype=torch.uint8, device="cuda")
    n.run()
    torch.cuda.synchronize()
    assert not n.out[:-tail].any() and not n.dout[:-tail].any()
    n.qkv, n.dqkv, n.out, n.dout = rows[-tail:], up[-tail:], n.out[-tail:], n.dout[-tail:]
    n.check()

"""Loss of a vocabulary shard against its definition in 64 bits: sizes that divide by nothing, pieces, shards joined, ignored labels."""
import math

import pytest

torch = pytest.importorskip("torch")
import packed_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu


def _tensors(seed, M, H, V, dtype, sigma=0.1):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(M, H, generator=g).to(dtype).cuda(), (torch.randn(V, H, generator=g) * sigma).to(dtype).cuda(), g


class Shards:
    """All shards of a vocabulary on the one GPU."""

    def __init__(self, M, H, V, ranks, dtype, seed=0, ignored=0.2):
        import paper_2111_05972_amd as pkg
        self.pkg, self.dt = pkg, pkg.TPL_BF16 if dtype == torch.bfloat16 else pkg.TPL_F32
        self.M, self.H, self.V, self.ranks = M, H, V, ranks
        self.x, self.w, g = _tensors(seed, M, H, V * ranks, dtype)
        labels = torch.randint(0, V * ranks, (M,), generator=g)
        labels[torch.rand(M, generator=g) < ignored] = -100
        if M > 2:
            labels[0], labels[1], labels[2] = V * ranks - 1, 0, V * ranks          # the last and the first of the vocabulary, one past it
        self.labels = labels.to(torch.int32).cuda()
        self.dloss = torch.rand(M, generator=g).cuda()
        self.stats = torch.full((ranks, M, 2), 7.0, device="cuda")
        self.loss, self.lse = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
        self.ws = torch.full((max(pkg.tp_layer_lm_loss_workspace_bytes(self.dt, M, H, V, b) for b in (0, 1)),), 255, dtype=torch.uint8, device="cuda")
        self.dx = [torch.full_like(self.x, 7.0) for _ in range(ranks)]
        self.dw = torch.full_like(self.w, 7.0)

    def run(self):
        st, M, H, V, T, p = torch.cuda.current_stream(), self.M, self.H, self.V, self.ranks, self.pkg
        for r in range(T):
            p.tp_layer_lm_loss_fwd(self.dt, M, H, V, r * V, self.x, self.w[r * V:], self.labels, self.stats[r], self.ws, stream=st)
        p.tp_layer_lm_loss_join(M, T, T * V, self.stats, self.labels, self.loss, self.lse, stream=st)
        for r in range(T):
            p.tp_layer_lm_loss_bwd(self.dt, M, H, V, r * V, T * V, self.x, self.w[r * V:], self.labels, self.lse, self.dloss, self.dx[r],
                                   self.dw[r * V:], self.ws, stream=st)

    def check(self):
        V, T = self.V, self.ranks
        z = self.x.double().cpu() @ self.w.double().cpu().t()
        lse = z.logsumexp(1)
        y = self.labels.long().cpu()
        known = (y >= 0) & (y < T * V)
        for r in range(T):
            val, tol = ref.loss(self.x, self.w[r * V:(r + 1) * V], self.labels, r * V, T * V, lse, self.dloss)
            ref.check(self.stats[r, :, 0], val["lse"], tol["lse"], "lse")
            here = torch.isfinite(val["target"])
            ref.check(self.stats[r, :, 1][here.cuda()], val["target"][here], tol["target"][here], "target")
            assert (self.stats[r, :, 1].cpu()[~here] == -math.inf).all()
            more = tol["lse"].max().item() + 8 * ref.F32 * (1 + lse.abs().max().item())      # what is off in the lse that backward is given
            ref.check(self.dx[r], val["dx"], tol["dx"] + more * self._scale(val, r)[0], "dx")
            ref.check(self.dw[r * V:(r + 1) * V], val["dw"], tol["dw"] + more * self._scale(val, r)[1], "dw")
        want = torch.where(known, lse - z.gather(1, y.clamp(0, T * V - 1)[:, None])[:, 0], torch.zeros_like(lse))
        assert (self.loss.double().cpu() - want).abs().max() <= 4 * (tol["lse"].max() + tol["target"].max() + 16 * ref.F32 * (1 + lse.abs().max()))
        assert (self.loss.cpu()[~known] == 0).all()

    def _scale(self, val, r):
        """sum |p| d |w| and sum |p| d |x|: what a relative error of the probabilities does."""
        w, x = self.w[r * self.V:(r + 1) * self.V].double().cpu(), self.x.double().cpu()
        z = x @ self.w.double().cpu().t()
        p = (x @ w.t() - z.logsumexp(1)[:, None]).exp() * self.dloss.double().cpu()[:, None]
        return p @ w.abs(), p.t() @ x.abs()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,H,V,ranks", [(1, 64, 1, 1), (1, 256, 1000, 1), (37, 128, 1001, 2), (130, 72, 257, 3), (300, 520, 2055, 1), (257, 64, 8, 4), (64, 1024, 511, 2)])
def test_shards(M, H, V, ranks, dtype):
    s = Shards(M, H, V, ranks, dtype)
    s.run()
    torch.cuda.synchronize()
    s.check()
    first = [t.clone() for t in (s.loss, s.lse, *s.dx, s.dw)]
    s.run()
    assert all(torch.equal(a, b) for a, b in zip(first, (s.loss, s.lse, *s.dx, s.dw)))


# more than one piece of the vocabulary: dx is added up over them (bf16: 128 MiB a piece; 16391 tokens, 4096 rows a piece)
@pytest.mark.parametrize("dtype,M,V", [(torch.bfloat16, 16391, 9001), (torch.float32, 8195, 9001)])
def test_pieces(dtype, M, V):
    s = Shards(M, 64, V, 1, dtype)
    s.run()
    torch.cuda.synchronize()
    s.check()


# Weights of more than 2 GiB: more than one piece also in forward.  Against 64 bits on the GPU, a slice of the vocabulary at a time.
@pytest.mark.parametrize("dtype,M,H,V", [(torch.bfloat16, 24, 8192, 140000), (torch.float32, 9, 4096, 140000)])
def test_many_weights(dtype, M, H, V):
    import paper_2111_05972_amd as pkg
    dt, st = pkg.TPL_BF16 if dtype == torch.bfloat16 else pkg.TPL_F32, torch.cuda.current_stream()
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(M, H, device="cuda", generator=g).to(dtype)
    w = (torch.randn(V, H, device="cuda", generator=g) * 0.02).to(dtype)
    labels = torch.randint(0, V, (M,), device="cuda", generator=g, dtype=torch.int32)
    labels[0] = V - 1
    dloss = torch.rand(M, device="cuda", generator=g)
    stats, loss, lse = torch.empty(1, M, 2, device="cuda"), torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    ws = torch.empty(max(pkg.tp_layer_lm_loss_workspace_bytes(dt, M, H, V, b) for b in (0, 1)), dtype=torch.uint8, device="cuda")
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    pkg.tp_layer_lm_loss_fwd(dt, M, H, V, 0, x, w, labels, stats, ws, stream=st)
    pkg.tp_layer_lm_loss_join(M, 1, V, stats, labels, loss, lse, stream=st)
    pkg.tp_layer_lm_loss_bwd(dt, M, H, V, 0, V, x, w, labels, lse, dloss, dx, dw, ws, stream=st)
    torch.cuda.synchronize()
    X, z, most = x.double(), torch.empty(M, V, dtype=torch.float64, device="cuda"), 0.0
    for i in range(0, V, 10000):
        t = w[i:i + 10000].double().t().contiguous()
        z[:, i:i + 10000] = X @ t
        most = max(most, (X.abs() @ t.abs()).max().item())
    want = z.logsumexp(1)
    off = (H + 8) * ref.F32 * most + (V + 32) * ref.F32 * (1 + want.abs().max().item())           # of a logit, of the sum
    rows = torch.arange(M, device="cuda")
    assert (lse.double() - want).abs().max().item() <= off
    assert (loss.double() - (want - z[rows, labels.long()])).abs().max().item() <= 2 * off
    dz = (z - want[:, None]).exp()
    dz[rows, labels.long()] -= 1
    dz *= dloss.double()[:, None]
    # dz as an operand and what is stored: half a step each, as norms; float sums add far less
    tol = 2 * ref.HALF[dtype] + (2 * off if dtype == torch.float32 else 0.0)
    got_x, diff, norm = torch.zeros(M, H, dtype=torch.float64, device="cuda"), 0.0, 0.0
    for i in range(0, V, 10000):
        got_x += dz[:, i:i + 10000].contiguous() @ w[i:i + 10000].double()
        t = dz[:, i:i + 10000].t().contiguous() @ X
        diff, norm = diff + (dw[i:i + 10000].double() - t).norm().item() ** 2, norm + t.norm().item() ** 2
    assert (dx.double() - got_x).norm() <= tol * got_x.norm()
    assert diff ** 0.5 <= tol * norm ** 0.5


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_all_ignored(dtype):
    s = Shards(40, 64, 100, 1, dtype)
    s.labels.fill_(-1)
    s.run()
    assert (s.loss == 0).all() and all((d == 0).all() for d in s.dx) and (s.dw == 0).all()


# logits far apart: the maximum is taken off before the exponential
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_large_logits(dtype):
    s = Shards(20, 64, 300, 2, dtype, ignored=0.0)
    s.w.mul_(64)
    s.run()
    torch.cuda.synchronize()
    s.check()
    assert torch.isfinite(s.loss).all()


# The options that force the tiles of a layer's products leave the loss right, whatever they are set to.
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("name,value", [("gemm_group", g) for g in ("0", "64", "128", "192", "256", "384", "512")] + [("gemm_tile", "8"), ("gemm_shares", "3"), ("gemm_band", "2")])
def test_options(tune, name, value, dtype):
    tune.set(name, value)
    s = Shards(300, 520, 2055, 1, dtype)
    s.run()
    torch.cuda.synchronize()
    s.check()


def test_captured_and_replayed():
    s = Shards(150, 128, 1003, 1, torch.bfloat16)
    s.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
    for seed in (1, 2, 3):
        other = Shards(150, 128, 1003, 1, torch.bfloat16, seed=seed)
        for a, b in ((s.x, other.x), (s.w, other.w), (s.labels, other.labels), (s.dloss, other.dloss)):
            a.copy_(b)
        graph.replay()
        other.run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((s.loss, s.lse, s.dx[0], s.dw), (other.loss, other.lse, other.dx[0], other.dw)))


# dx and dw against differences of the loss in float
def test_gradient_against_differences():
    s = Shards(6, 8, 11, 1, torch.float32, ignored=0.0)
    s.run()
    st, step = torch.cuda.current_stream(), 2.0 ** -5

    def value(x, w):
        s.pkg.tp_layer_lm_loss_fwd(s.dt, 6, 8, 11, 0, x, w, s.labels, s.stats[0], s.ws, stream=st)
        s.pkg.tp_layer_lm_loss_join(6, 1, 11, s.stats, s.labels, s.loss, s.lse, stream=st)
        return (s.loss.double() * s.dloss.double()).sum().item()
    for which, grad in ((0, s.dx[0].clone()), (1, s.dw.clone())):
        for i, j in [(0, 0), (3, 5), (5, 7)]:
            f = []
            for k in (1, -1, 2, -2):
                t = [s.x.clone(), s.w.clone()]
                t[which][i, j] += k * step
                f.append(value(*t))
            diff = (8 * (f[0] - f[1]) - (f[2] - f[3])) / (12 * step)
            # fifth derivative of log-sum-exp (below 100 for unit inputs) times step^4 / 30, rounding of six losses below 8 over the step
            tol = 100 * step ** 4 / 30 + 6 * 8 * 8 * ref.F32 / step
            assert abs(diff - grad[i, j].item()) <= tol, (which, i, j)

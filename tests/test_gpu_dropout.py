"""Dropout with a mask that is not stored: the generator, the mask of slices, values and gradients against their definition in 64 bits."""
import math

import pytest

torch = pytest.importorskip("torch")
import block_ref  # noqa: E402
from packed_ref import check  # noqa: E402

pytestmark = pytest.mark.gpu
BF16, FLOAT = torch.bfloat16, torch.float32
SEED, STEP, SITE = 0x89ABCDEF01234567, 0x0000000712345678, 0xABCDE


class Drop:
    def __init__(self, M, N, p, dtype, first_row=0, first_col=0, width=None, seed=SEED, step=STEP, site=SITE, bias=True, resid=True):
        import paper_2111_05972_amd as pkg
        g = torch.Generator().manual_seed(M + N)
        make = lambda *s: torch.randn(*s, generator=g).to(dtype).cuda()          # noqa: E731
        self.pkg, self.dt = pkg, pkg.TPL_BF16 if dtype == BF16 else pkg.TPL_F32
        self.signed = lambda x: x - 2 ** 64 if x >= 2 ** 63 else x               # noqa: E731
        self.rng = torch.tensor([self.signed(seed), self.signed(step)], dtype=torch.int64, device="cuda")
        self.place, self.words = (site, first_row, first_col, width or N), (seed, step)
        self.dims = (M, N, p)
        self.x, self.bias, self.resid, self.dout = make(M, N), make(N) if bias else None, make(M, N) if resid else None, make(M, N)
        self.out, self.din, self.dbias = torch.full_like(self.x, 7.0), torch.full_like(self.x, 7.0), torch.full((N,), 7.0, dtype=dtype, device="cuda")
        self.ws = torch.full((pkg.tp_layer_dropout_workspace_bytes(M, N),), 255, dtype=torch.uint8, device="cuda")

    def args(self):
        return (self.dt, *self.dims, self.rng, *self.place)

    def run(self):
        st = torch.cuda.current_stream()
        self.pkg.tp_layer_dropout_fwd(*self.args(), self.x, self.bias, self.resid, self.out, stream=st)
        self.pkg.tp_layer_dropout_bwd(*self.args(), self.dout, self.din, self.dbias, self.ws, stream=st)

    def check(self):
        keep, scale = block_ref.kept(*self.dims, *self.words, *self.place)
        check(self.out, *block_ref.dropout(self.x, self.bias, self.resid, keep, scale), "out")
        d, ed, s, es = block_ref.dropout_bwd(self.dout, keep, scale)
        check(self.din, d, ed, "din")
        check(self.dbias, s, es, "dbias")
        assert torch.equal(self.din.cpu() == 0, ~keep | (self.dout.cpu() == 0))
        return keep


@pytest.mark.parametrize("dtype", [BF16, FLOAT])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.999, 1.0 - 2.0 ** -40, 1e-7])
@pytest.mark.parametrize("M,N", [(1, 8), (3, 64), (37, 520), (5, 1032), (130, 16)])
def test_values_and_gradients(M, N, p, dtype):
    d = Drop(M, N, p, dtype)
    d.run()
    d.check()


@pytest.mark.parametrize("dtype", [BF16, FLOAT])
@pytest.mark.parametrize("bias,resid", [(False, False), (True, False), (False, True)])
def test_without_bias_or_residual(bias, resid, dtype):
    d = Drop(19, 72, 0.25, dtype, bias=bias, resid=resid)
    d.run()
    d.check()
    din = d.din.clone()
    d.pkg.tp_layer_dropout_bwd(*d.args(), d.dout, d.din, stream=torch.cuda.current_stream())
    assert torch.equal(d.din, din)


# counters past 32 bits, the largest site, seeds and steps with their highest bits set
@pytest.mark.parametrize("seed,step,site,first_row", [(2 ** 64 - 1, 2 ** 64 - 1, 2 ** 20 - 1, 2 ** 44 - 7), (2 ** 63, 2 ** 32, 0, 2 ** 32 - 3), (1, 2 ** 63, 1, 2 ** 40)])
def test_far_counters(seed, step, site, first_row):
    d = Drop(7, 8, 0.5, FLOAT, first_row=first_row, seed=seed, step=step, site=site)
    d.run()
    d.check()


# Slices draw what the whole tensor draws, whatever their sizes.
@pytest.mark.parametrize("dtype", [BF16, FLOAT])
def test_slices_have_the_mask_of_the_whole(dtype):
    M, N = 50, 640
    whole = Drop(M, N, 0.3, dtype, bias=False, resid=False)
    whole.run()
    for r0, r1, c0, c1 in [(0, 50, 0, 320), (0, 50, 320, 640), (13, 14, 8, 16), (20, 50, 72, 600)]:
        part = Drop(r1 - r0, c1 - c0, 0.3, dtype, first_row=r0, first_col=c0, width=N, bias=False, resid=False)
        part.x, part.dout = whole.x[r0:r1, c0:c1].contiguous(), whole.dout[r0:r1, c0:c1].contiguous()
        part.run()
        assert torch.equal(part.out, whole.out[r0:r1, c0:c1]) and torch.equal(part.din, whole.din[r0:r1, c0:c1])


# Another seed, step or site is another mask: of 32768 elements half differ, within 6 standard deviations (sqrt(32768) / 2).
def test_masks_differ():
    masks = []
    for kw in (dict(), dict(seed=SEED + 1), dict(step=STEP + 1), dict(site=SITE + 1), dict(seed=SEED ^ 1 << 40), dict(step=STEP ^ 1 << 40), dict(first_row=64)):
        d = Drop(64, 512, 0.5, FLOAT, bias=False, resid=False, **kw)
        d.run()
        masks.append(d.out != 0)
    for i in range(len(masks)):
        for j in range(i):
            assert abs((masks[i] != masks[j]).sum().item() - 16384) <= 6 * math.sqrt(32768) / 2, (i, j)


# Kept with probability 1 - t / 65536 in every column and place of an eight, within 6 standard deviations.
@pytest.mark.parametrize("p", [0.1, 0.5, 0.9])
def test_share_that_is_kept(p):
    M, N = 4096, 1024
    d = Drop(M, N, p, BF16, bias=False, resid=False)
    d.x.fill_(1.0)
    d.run()
    q = 1.0 - min(65535, math.floor(65536 * p + 0.5)) / 65536
    keep = (d.out != 0).double()
    assert abs(keep.sum().item() - M * N * q) <= 6 * math.sqrt(M * N * q * (1 - q))
    for part in (keep.view(-1, 8).sum(0), ):
        assert (part - M * N / 8 * q).abs().max().item() <= 6 * math.sqrt(M * N / 8 * q * (1 - q))
    assert (keep.sum(0) - M * q).abs().max().item() <= 7 * math.sqrt(M * q * (1 - q))
    assert (keep.sum(1) - N * q).abs().max().item() <= 7 * math.sqrt(N * q * (1 - q))


# What is dropped does not matter.
@pytest.mark.parametrize("dtype", [BF16, FLOAT])
@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_dropped_values_do_not_matter(dtype, bad):
    d = Drop(20, 64, 0.5, dtype)
    d.run()
    keep = d.check().cuda()
    out, din, dbias = d.out.clone(), d.din.clone(), d.dbias.clone()
    d.x[~keep] = bad
    d.dout[~keep] = bad
    d.run()
    assert torch.equal(d.out, out) and torch.equal(d.din, din) and torch.equal(d.dbias, dbias)


@pytest.mark.parametrize("dtype", [BF16, FLOAT])
def test_in_place(dtype):
    d = Drop(70, 136, 0.2, dtype)
    d.run()
    st = torch.cuda.current_stream()
    a, b, g = d.x.clone(), d.resid.clone(), d.dout.clone()
    d.pkg.tp_layer_dropout_fwd(*d.args(), a, d.bias, d.resid, a, stream=st)
    d.pkg.tp_layer_dropout_fwd(*d.args(), d.x, d.bias, b, b, stream=st)
    d.pkg.tp_layer_dropout_bwd(*d.args(), g, g, d.dbias, d.ws, stream=st)
    assert torch.equal(a, d.out) and torch.equal(b, d.out) and torch.equal(g, d.din)


# Sums over many rows: the same from run to run, whatever the workspace holds.
@pytest.mark.parametrize("M,N", [(5000, 8), (3000, 520), (1000, 4096)])
def test_bias_gradient_over_many_rows(M, N):
    d = Drop(M, N, 0.1, FLOAT)
    d.run()
    # the mask from the kernel's own din: that is checked above
    keep = d.din != 0
    x = torch.where(keep, d.dout.double() * (65536.0 / (65536 - 6554)), 0.0)
    assert ((d.dbias.double() - x.sum(0)).abs() <= (M + 8) * 2.0 ** -24 * x.abs().sum(0)).all()
    first = d.dbias.clone()
    for fill in (0, 255):
        d.ws.fill_(fill)
        d.run()
        assert torch.equal(d.dbias, first)


# A captured step draws anew whenever a replay finds another step in memory.
def test_graph_follows_the_step():
    d = Drop(40, 256, 0.4, BF16)
    d.run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        d.run()
    seen = []
    for step in (STEP, 5, 6, 5):
        d.words = (SEED, step)
        d.rng[1] = d.signed(step)
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (d.out, d.din, d.dbias)]
        d.check()
        d.run()
        assert all(torch.equal(a, b) for a, b in zip(got, (d.out, d.din, d.dbias)))
        seen.append(got[0])
    assert torch.equal(seen[1], seen[3]) and not torch.equal(seen[1], seen[2])


# Elements past 2^32: the last rows of a tensor of 8 GiB
def test_a_large_tensor():
    M, N, tail = 350000, 12288, 3
    d = Drop(tail, N, 0.1, BF16, first_row=M - tail, bias=False, resid=False)
    d.run()
    x = torch.zeros(M, N, dtype=BF16, device="cuda")
    x[-tail:] = d.x
    d.pkg.tp_layer_dropout_fwd(d.dt, M, N, 0.1, d.rng, d.place[0], 0, 0, N, x, None, None, x, stream=torch.cuda.current_stream())
    assert torch.equal(x[-tail:], d.out) and not x[:-tail].any()

"""The rotary, packed-attention and loss entry points together, as a decoder uses them: a batch of packed documents through an attention block with
grouped heads and a residual, the loss of a vocabulary in two shards, and back to every weight; eagerly, and captured once for all batches."""
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
H, NQ, NKV, DH, ROT, V, RANKS, M = 96, 4, 2, 32, 16, 152, 2, 224


class Decoder:
    def __init__(self, dtype):
        import paper_2111_05972_amd as pkg
        self.pkg, self.dtype, self.dt = pkg, dtype, pkg.TPL_BF16 if dtype == torch.bfloat16 else pkg.TPL_F32
        g = torch.Generator().manual_seed(11)
        new = lambda *s, sigma=1.0: (torch.randn(*s, generator=g) * sigma).to(dtype).cuda()     # noqa: E731
        row, wide = (NQ + 2 * NKV) * DH, NQ * DH
        self.x, self.w_qkv, self.w_o, self.w_out = new(M, H), new(H, row, sigma=H ** -0.5), new(wide, H, sigma=wide ** -0.5), new(RANKS * V, H, sigma=0.2)
        freq, self.factor = pkg.tp_layer_rope_frequencies(ROT)
        self.freq_list, self.freq = freq, torch.tensor(freq, dtype=torch.float64, device="cuda")
        self.offsets = torch.zeros(4, dtype=torch.int32, device="cuda")
        self.labels = torch.zeros(M, dtype=torch.int32, device="cuda")
        self.dloss = torch.zeros(M, device="cuda")
        self.plan = torch.empty(pkg.tp_layer_pack_plan_bytes(3, M, NQ, NKV), dtype=torch.uint8, device="cuda")
        self.positions = self.plan[:4 * M].view(torch.int32)
        self.dims = (self.dt, 3, M, NQ, NKV, DH, True)
        like = lambda *s, t=dtype: torch.full(s, math.nan, dtype=t, device="cuda")             # noqa: E731
        self.qkv, self.o, self.y = like(M, row), torch.zeros(M, wide, dtype=dtype, device="cuda"), like(M, H)
        self.lse, self.dsum = like(M, NQ, t=torch.float32), like(M, NQ, t=torch.float32)
        self.stats, self.loss, self.zlse = (like(*s, t=torch.float32) for s in ((RANKS, M, 2), (M,), (M,)))
        self.dy_part, self.dy, self.do = like(RANKS, M, H), like(M, H), like(M, wide)
        self.dqkv = torch.zeros(M, row, dtype=dtype, device="cuda")
        self.dx, self.dw_qkv, self.dw_o, self.dw_out = like(M, H), like(H, row), like(wide, H), like(RANKS * V, H)
        sizes = [pkg.tp_layer_attn_packed_workspace_bytes(*self.dims, b) for b in (0, 1)] + [pkg.tp_layer_lm_loss_workspace_bytes(self.dt, M, H, V, b) for b in (0, 1)]
        sizes += [pkg.tp_layer_gemm_workspace_bytes(self.dt, *s) for s in ((M, row, H), (M, H, wide), (M, wide, H), (wide, H, M), (M, H, row), (H, row, M))]
        self.ws = torch.empty(max(sizes), dtype=torch.uint8, device="cuda")

    def batch(self, lengths, seed):
        g = torch.Generator().manual_seed(seed)
        self.lengths, used = lengths, sum(lengths)
        labels = torch.randint(0, RANKS * V, (M,), generator=g)
        labels[torch.rand(M, generator=g) < 0.1] = -100
        labels[used:] = -100
        self.x.copy_((torch.randn(M, H, generator=g)).to(self.dtype))
        self.offsets.copy_(torch.tensor([0, lengths[0], lengths[0] + lengths[1], used], dtype=torch.int32))
        self.labels.copy_(labels.to(torch.int32))
        self.dloss.fill_(1.0 / max(1, int((labels >= 0).sum())))

    def step(self):
        p, st = self.pkg, torch.cuda.current_stream()
        row, wide = (NQ + 2 * NKV) * DH, NQ * DH
        rope = (self.dt, M, NQ, NKV, DH, ROT, p.TPL_ROPE_HALF, self.freq, self.factor, self.positions)
        product = lambda *a, **k: p.tp_layer_gemm(self.dt, *a, ws=self.ws, stream=st, **k)      # noqa: E731
        self.o.zero_()                                                                          # rows of no sequence
        self.dqkv.zero_()
        p.tp_layer_pack_plan(3, M, self.offsets, NQ, NKV, True, self.plan, stream=st)
        product(0, 0, M, row, H, self.x, self.w_qkv, self.qkv)
        p.tp_layer_rope_fwd(*rope, self.qkv, self.qkv, stream=st)
        p.tp_layer_attn_packed_fwd(*self.dims, self.plan, self.qkv, self.o, self.lse, self.ws, stream=st)
        product(0, 0, M, H, wide, self.o, self.w_o, self.y, resid=self.x)
        for r in range(RANKS):
            p.tp_layer_lm_loss_fwd(self.dt, M, H, V, r * V, self.y, self.w_out[r * V:], self.labels, self.stats[r], self.ws, stream=st)
        p.tp_layer_lm_loss_join(M, RANKS, RANKS * V, self.stats, self.labels, self.loss, self.zlse, stream=st)
        for r in range(RANKS):
            p.tp_layer_lm_loss_bwd(self.dt, M, H, V, r * V, RANKS * V, self.y, self.w_out[r * V:], self.labels, self.zlse, self.dloss, self.dy_part[r],
                                   self.dw_out[r * V:], self.ws, stream=st)
        torch.add(self.dy_part[0], self.dy_part[1], out=self.dy)                                # what the ranks would all-reduce
        product(1, 0, wide, H, M, self.o, self.dy, self.dw_o)
        product(0, 1, M, wide, H, self.dy, self.w_o, self.do)
        p.tp_layer_attn_packed_bwd(*self.dims, self.plan, self.qkv, self.o, self.lse, self.do, self.dqkv, self.dsum, self.ws, stream=st)
        p.tp_layer_rope_bwd(*rope, self.dqkv, self.dqkv, stream=st)
        product(1, 0, H, row, M, self.x, self.dqkv, self.dw_qkv)
        product(0, 1, M, H, row, self.dqkv, self.w_qkv, self.dx, resid=self.dy)

    def outputs(self):
        return {k: getattr(self, k) for k in ("loss", "dx", "dw_qkv", "dw_o", "dw_out")}

    def expected(self):
        """The same in 64 bits on the host, gradients by differentiation of its operations."""
        x, w_qkv, w_o, w_out = (t.double().cpu().requires_grad_() for t in (self.x, self.w_qkv, self.w_o, self.w_out))
        used = sum(self.lengths)
        qkv = (x @ w_qkv).view(M, NQ + 2 * NKV, DH)
        o = []
        at = 0
        for n in self.lengths:
            a = torch.arange(n, dtype=torch.float64)[:, None] * torch.tensor(self.freq_list, dtype=torch.float64)
            c, s = a.cos()[:, None], a.sin()[:, None]
            rows = qkv[at:at + n]
            u, v = rows[..., :ROT // 2], rows[..., ROT // 2:ROT]
            turned = torch.cat([u * c - v * s, u * s + v * c, rows[..., ROT:]], -1)
            turned = torch.cat([turned[:, :NQ + NKV], rows[:, NQ + NKV:]], 1)
            hide = torch.ones(n, n, dtype=torch.bool).triu(1)
            heads = []
            for h in range(NQ):
                k, v = turned[:, NQ + h // (NQ // NKV)], turned[:, NQ + NKV + h // (NQ // NKV)]
                heads.append((turned[:, h] @ k.t() / math.sqrt(DH)).masked_fill(hide, -math.inf).softmax(-1) @ v)
            o.append(torch.stack(heads, 1).reshape(n, NQ * DH))
            at += n
        o = torch.cat(o + [torch.zeros(M - used, NQ * DH, dtype=torch.float64)])
        y = x + o @ w_o
        z = y @ w_out.t()
        labels = self.labels.long().cpu()
        known = (labels >= 0) & (labels < RANKS * V)
        loss = torch.where(known, z.logsumexp(1) - z.gather(1, labels.clamp(min=0)[:, None])[:, 0], torch.zeros(M, dtype=torch.float64))
        (loss * self.dloss.double().cpu()).sum().backward()
        return {"loss": loss.detach(), "dx": x.grad, "dw_qkv": w_qkv.grad, "dw_o": w_o.grad, "dw_out": w_out.grad}

    def check(self):
        # Twelve operations lie between the inputs and the last gradient.  float: each sums at most n = 304 terms (the vocabulary) and is off by
        # (n + 32) 2^-24 of the sum of their absolute values, which for terms of random sign is below 16 ~ sqrt(n) times the sum.
        # bf16: each stores its result, off by half a step (2^-8 at most, of one value), and uses what the one before stored; as norms the errors of twelve
        # add up, and a difference of two (dP - D, dz) may double what is relative to it, twice on the way: 4 x 12 x 2^-8.
        tol = 12 * (304 + 32) * 16 * 2.0 ** -24 if self.dtype == torch.float32 else 4 * 12 * 2.0 ** -8
        for k, want in self.expected().items():
            got = getattr(self, k).double().cpu()
            assert torch.isfinite(got).all(), k
            assert (got - want).norm() <= tol * want.norm(), k


BATCHES = [[100, 60, 40], [1, 0, 223], [0, 130, 7], [64, 64, 96]]


@pytest.mark.parametrize("lengths", BATCHES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_step(dtype, lengths):
    d = Decoder(dtype)
    d.batch(lengths, seed=sum(lengths))
    d.step()
    torch.cuda.synchronize()
    d.check()


def test_captured_step_takes_any_batch():
    d = Decoder(torch.bfloat16)
    d.batch(BATCHES[0], seed=1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        d.step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        d.step()
    for seed, lengths in enumerate(BATCHES + BATCHES[:1]):
        d.batch(lengths, seed)
        graph.replay()
        torch.cuda.synchronize()
        d.check()
        got = {k: x.clone() for k, x in d.outputs().items()}
        d.step()
        torch.cuda.synchronize()
        assert all(torch.equal(got[k], x) for k, x in d.outputs().items())

"""Attention of packed sequences with grouped heads against its definition in 64 bits: lengths, head sizes, groups, cut strips, what a mask
hides, rows of no sequence, plans, graphs."""
import math

import pytest

torch = pytest.importorskip("torch")
import packed_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu
EDGES = [1, 0, 63, 64, 65, 1, 130, 0]


def _pkg():
    import paper_2111_05972_amd as pkg
    return pkg


def _rows(seed, *shape, dtype, sigma=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * sigma).to(dtype).cuda()


class Batch:
    """A packed batch with its plan and workspace; rows behind the last sequence hold `behind`."""

    def __init__(self, lengths, nq, nkv, dh, causal, dtype, behind=0, seed=0, fill=math.nan):
        pkg = _pkg()
        self.pkg, self.dt = pkg, pkg.TPL_BF16 if dtype == torch.bfloat16 else pkg.TPL_F32
        self.offsets = [0]
        for n in lengths:
            self.offsets.append(self.offsets[-1] + n)
        self.M, self.used = self.offsets[-1] + behind, self.offsets[-1]
        self.dims = (self.dt, len(lengths), self.M, nq, nkv, dh, causal)
        self.shape, self.dtype = (nq, nkv, dh, causal), dtype
        self.qkv = _rows(seed, self.M, (nq + 2 * nkv) * dh, dtype=dtype)
        self.d_o = _rows(seed + 1, self.M, nq * dh, dtype=dtype)
        self.qkv[self.used:] = fill
        self.d_o[self.used:] = fill
        self.on_gpu = torch.tensor(self.offsets, dtype=torch.int32, device="cuda")
        self.plan = torch.full((pkg.tp_layer_pack_plan_bytes(len(lengths), self.M, nq, nkv),), 255, dtype=torch.uint8, device="cuda")
        self.ws = torch.full((max(pkg.tp_layer_attn_packed_workspace_bytes(*self.dims, b) for b in (0, 1)),), 255, dtype=torch.uint8, device="cuda")
        self.o = torch.full((self.M, nq * dh), 7.0, dtype=dtype, device="cuda")
        self.lse = torch.full((self.M, nq), 7.0, device="cuda")
        self.dsum = torch.empty(self.M, nq, device="cuda")
        self.dqkv = torch.full_like(self.qkv, 7.0)

    def make_plan(self):
        self.pkg.tp_layer_pack_plan(self.dims[1], self.M, self.on_gpu, *self.dims[3:5], self.dims[6], self.plan, stream=torch.cuda.current_stream())

    def run(self):
        st = torch.cuda.current_stream()
        self.pkg.tp_layer_attn_packed_fwd(*self.dims, self.plan, self.qkv, self.o, self.lse, self.ws, stream=st)
        self.pkg.tp_layer_attn_packed_bwd(*self.dims, self.plan, self.qkv, self.o, self.lse, self.d_o, self.dqkv, self.dsum, self.ws, stream=st)

    def outputs(self):
        return {"o": self.o, "lse": self.lse, "dqkv": self.dqkv}

    def check(self):
        nq, nkv, dh, causal = self.shape
        val, tol = ref.attention(self.qkv, self.offsets, nq, nkv, dh, causal, self.d_o)
        for k, x in self.outputs().items():
            ref.check(x, val[k], tol[k], k)
            assert (x[self.used:] == 7.0).all(), f"{k}: rows behind the last sequence"


def _run(*args, **kw):
    b = Batch(*args, **kw)
    b.make_plan()
    b.run()
    torch.cuda.synchronize()
    b.check()
    return b


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("nq,nkv", [(2, 2), (6, 2), (8, 1)])
@pytest.mark.parametrize("dh", [64, 128, 80])
def test_edges(dh, nq, nkv, causal):
    _run(EDGES, nq, nkv, dh, causal, torch.bfloat16, behind=3)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dh", [8, 32, 40, 96, 104])
def test_head_sizes(dh, dtype):
    _run([33, 1, 100], 5, 1, dh, True, dtype, behind=1)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("nq,nkv,dh", [(2, 2, 64), (6, 2, 64), (3, 1, 128)])
def test_float(dh, nq, nkv, causal):
    _run(EDGES, nq, nkv, dh, causal, torch.float32, behind=3)


@pytest.mark.parametrize("lengths,nq", [([1], 1), ([1], 128), ([2, 1, 1, 3], 7), ([0, 0, 5], 2), ([1] * 70, 3), ([17] * 40, 4)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_few_tokens(lengths, nq, dtype):
    _run(lengths, nq, 1, 64, True, dtype)


# strips long enough to be cut on both sides: in chunks of 16 tiles and a shorter last one
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,dh,nq", [(torch.bfloat16, 128, 1), (torch.bfloat16, 64, 3), (torch.bfloat16, 80, 2), (torch.float32, 64, 2), (torch.float32, 32, 1)])
def test_cut_strips(dtype, dh, nq, causal):
    _run([2300, 5, 700], nq, 1, dh, causal, dtype, behind=2)


def test_results_do_not_change_from_run_to_run():
    b = _run([1500, 3, 800], 4, 2, 64, True, torch.bfloat16)
    first = {k: x.clone() for k, x in b.outputs().items()}
    for _ in range(3):
        b.make_plan()
        b.run()
        assert all(torch.equal(x, first[k]) for k, x in b.outputs().items())


def test_positions_begin_the_plan():
    b = Batch([3, 0, 70, 1], 2, 1, 64, True, torch.bfloat16, behind=4)
    b.make_plan()
    want = [i for n in (3, 0, 70, 1) for i in range(n)] + [0] * 4
    assert b.plan.view(torch.int32)[:b.M].tolist() == want


# What a mask hides is as if it were not there: later tokens of the sequence under the causal mask, other sequences, rows of none.
@pytest.mark.parametrize("dtype,dh", [(torch.bfloat16, 64), (torch.bfloat16, 128), (torch.float32, 64)])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_hidden_values_do_not_matter(dtype, dh, bad):
    nq, nkv, cut = 4, 2, 40
    b = Batch([70, 90], nq, nkv, dh, True, dtype, behind=2)
    val, tol = ref.attention(b.qkv, b.offsets, nq, nkv, dh, True, b.d_o)
    b.qkv.view(b.M, nq + 2 * nkv, dh)[cut:70, nq:] = bad             # K and V of the first sequence's later tokens
    b.make_plan()
    b.run()
    for k in ("o", "lse"):
        ref.check(b.outputs()[k][:cut], val[k][:cut], tol[k][:cut], k)
    for k, x in b.outputs().items():
        ref.check(x[70:160], val[k][70:160], tol[k][70:160], k)


# Backward: a query that does not see a key leaves it alone, whatever its dO and Q hold.
@pytest.mark.parametrize("dtype,dh", [(torch.bfloat16, 64), (torch.bfloat16, 128), (torch.float32, 64)])
def test_hidden_queries_do_not_matter(dtype, dh):
    cut = 40
    b = Batch([70, 5], 2, 1, dh, True, dtype)
    val, tol = ref.attention(b.qkv, b.offsets, 2, 1, dh, True, b.d_o)
    b.d_o[:cut] = math.inf
    b.qkv.view(b.M, 4, dh)[:cut, :2] = math.nan
    b.make_plan()
    b.run()
    ref.check(b.dqkv[cut:75], val["dqkv"][cut:75], tol["dqkv"][cut:75], "dqkv")   # keys that no spoilt query sees, and their own queries


# The same where strips are cut into chunks: a chunk that holds a spoilt key or query is worked out again before it is joined.
@pytest.mark.parametrize("dtype,dh", [(torch.bfloat16, 64), (torch.bfloat16, 128), (torch.float32, 64)])
def test_hidden_values_in_cut_strips(dtype, dh):
    nq, nkv, cut = 4, 2, 1370
    b = Batch([1400, 60], nq, nkv, dh, True, dtype, behind=2)
    val, tol = ref.attention(b.qkv, b.offsets, nq, nkv, dh, True, b.d_o)
    b.qkv.view(b.M, nq + 2 * nkv, dh)[cut:1400, nq:] = math.inf
    b.make_plan()
    b.run()
    for k in ("o", "lse"):
        ref.check(b.outputs()[k][:cut], val[k][:cut], tol[k][:cut], k)
    ref.check(b.dqkv[:cut, :nq * dh], val["dqkv"][:cut, :nq * dh], tol["dqkv"][:cut, :nq * dh], "dq")
    for k, x in b.outputs().items():
        ref.check(x[1400:1460], val[k][1400:1460], tol[k][1400:1460], k)


@pytest.mark.parametrize("dtype,dh", [(torch.bfloat16, 64), (torch.bfloat16, 128), (torch.float32, 64)])
def test_hidden_queries_in_cut_strips(dtype, dh):
    nq, nkv, cut = 4, 2, 700
    b = Batch([1400, 60], nq, nkv, dh, True, dtype)
    val, tol = ref.attention(b.qkv, b.offsets, nq, nkv, dh, True, b.d_o)
    b.d_o[:cut] = math.inf
    b.qkv.view(b.M, nq + 2 * nkv, dh)[:cut, :nq] = math.nan
    b.make_plan()
    b.run()
    ref.check(b.dqkv[cut:], val["dqkv"][cut:], tol["dqkv"][cut:], "dqkv")


# Sequences of every length around a tile and a strip, all at once: chunks, whole strips, strips of one row
def test_many_lengths():
    _run(list(range(0, 70)) + [127, 128, 129, 255, 257, 1025], 3, 1, 64, True, torch.bfloat16, behind=1)


# Rows and values past 2^31 bytes and 2^31 elements: the last documents of a batch of a million tokens
def test_a_long_batch():
    pkg = _pkg()
    nq, nkv, dh, each, tail = 16, 2, 128, 500, 1000
    M = 1000000
    n = M // each
    st = torch.cuda.current_stream()
    g = torch.Generator(device="cuda").manual_seed(4)
    qkv = torch.empty(M, (nq + 2 * nkv) * dh, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    d_o = torch.empty(M, nq * dh, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    before = qkv[-tail:].clone()
    offsets = torch.arange(0, M + 1, each, dtype=torch.int32, device="cuda")
    plan = torch.empty(pkg.tp_layer_pack_plan_bytes(n, M, nq, nkv), dtype=torch.uint8, device="cuda")
    dims = (pkg.TPL_BF16, n, M, nq, nkv, dh, True)
    ws = torch.empty(max(pkg.tp_layer_attn_packed_workspace_bytes(*dims, b) for b in (0, 1)), dtype=torch.uint8, device="cuda")
    freq, factor = pkg.tp_layer_rope_frequencies(dh)
    pkg.tp_layer_pack_plan(n, M, offsets, nq, nkv, True, plan, stream=st)
    on_gpu = torch.tensor(freq, dtype=torch.float64, device="cuda")
    pkg.tp_layer_rope_fwd(pkg.TPL_BF16, M, nq, nkv, dh, dh, 0, on_gpu, factor, plan[:4 * M].view(torch.int32), qkv, qkv, stream=st)
    o, lse, dsum, dqkv = torch.empty_like(d_o), torch.empty(M, nq, device="cuda"), torch.empty(M, nq, device="cuda"), torch.empty_like(qkv)
    pkg.tp_layer_attn_packed_fwd(*dims, plan, qkv, o, lse, ws, stream=st)
    pkg.tp_layer_attn_packed_bwd(*dims, plan, qkv, o, lse, d_o, dqkv, dsum, ws, stream=st)
    torch.cuda.synchronize()
    val, tol = ref.rotary(before, nq, nkv, dh, dh, False, torch.arange(tail) % each, freq, factor, False)
    ref.check(qkv[-tail:], val, tol, "turned")
    val, tol = ref.attention(qkv[-tail:], [0, each, tail], nq, nkv, dh, True, d_o[-tail:])
    for k, x in (("o", o), ("lse", lse), ("dqkv", dqkv)):
        ref.check(x[-tail:], val[k], tol[k], k)


# Many short sequences in float, which a wavefront has to itself, beside longer ones; and what a mask hides among them
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dh,nq,nkv", [(64, 16, 8), (128, 4, 4), (32, 6, 2), (32, 12, 12), (96, 16, 4)])
def test_many_short_sequences_in_float(dh, nq, nkv, causal):
    _run(list(range(0, 60)) + [0, 1, 31, 32, 33, 64, 65, 150, 193] * 2, nq, nkv, dh, causal, torch.float32, behind=1)


def test_hidden_values_among_many_short_sequences():
    nq, nkv, dh, n, cut = 4, 4, 128, 70, 20
    b = Batch([30] * n, nq, nkv, dh, True, torch.float32)
    val, tol = ref.attention(b.qkv, b.offsets, nq, nkv, dh, True, b.d_o)
    rows = b.qkv.view(n, 30, nq + 2 * nkv, dh)
    rows[::2, cut:, nq:] = math.inf                                  # K and V of the later tokens of every other sequence
    b.d_o.view(n, 30, nq, dh)[1::4, :cut] = math.nan                 # dO of the earlier ones of some of the others
    b.make_plan()
    b.run()
    shape = lambda x: x.reshape(n, 30, -1)                           # noqa: E731
    for k in ("o", "lse"):
        ref.check(shape(b.outputs()[k])[::2, :cut], shape(val[k])[::2, :cut], shape(tol[k])[::2, :cut], k)
        ref.check(shape(b.outputs()[k])[1::2], shape(val[k])[1::2], shape(tol[k])[1::2], k)
    got, want, off = shape(b.dqkv), shape(val["dqkv"]), shape(tol["dqkv"])
    ref.check(got[::2, :cut, :nq * dh], want[::2, :cut, :nq * dh], off[::2, :cut, :nq * dh], "dq")
    ref.check(got[1::4, cut:], want[1::4, cut:], off[1::4, cut:], "dqkv")
    ref.check(got[3::4], want[3::4], off[3::4], "dqkv")


def test_offsets_that_decrease_stay_in_bounds():
    b = Batch([40, 30, 30], 2, 1, 64, True, torch.bfloat16)
    b.on_gpu = torch.tensor([-5, 60, 20, 1000], dtype=torch.int32, device="cuda")      # taken as 0, 60, 60, 100
    b.make_plan()
    b.run()
    b.offsets = [0, 60, 60, 100]
    b.check()


@pytest.mark.parametrize("causal", [True, False])
def test_offsets_that_decrease_are_their_running_maximum(causal):
    b = Batch([200, 0, 100, 50], 2, 1, 64, causal, torch.bfloat16, behind=3)
    b.on_gpu = torch.tensor([0, 200, 90, 300, 350], dtype=torch.int32, device="cuda")          # 0, 200, 200, 300, 350
    b.dsum.fill_(math.nan)
    b.make_plan()
    assert b.plan.view(torch.int32)[:b.M].tolist() == list(range(200)) + list(range(100)) + list(range(50)) + [0] * 3
    b.run()
    b.check()


# More sequences than a workgroup of the plan has threads, and than it keeps in LDS; empty ones and a decrease among them
@pytest.mark.parametrize("n", [1023, 1024, 1025, 2047, 2048, 2500])
def test_many_sequences(n):
    g = torch.Generator().manual_seed(n)
    lengths = torch.randint(0, 5, (n,), generator=g).tolist()
    lengths[n // 2], lengths[n - 1] = 150, 3
    b = Batch(lengths, 2, 1, 32, True, torch.bfloat16, behind=2)
    b.on_gpu[n // 3] = 1                                            # before it all is larger: the sequence before ends where this one did not
    b.offsets = torch.tensor(b.on_gpu.tolist()).cummax(0)[0].tolist()
    b.make_plan()
    want = [i for a, z in zip(b.offsets[:-1], b.offsets[1:]) for i in range(z - a)] + [0] * 2
    assert b.plan.view(torch.int32)[:b.M].tolist() == want
    b.run()
    b.check()


def test_another_plan_writes_nothing():
    b = Batch([40, 30], 2, 1, 64, True, torch.bfloat16)
    other = Batch([40, 30], 2, 1, 64, False, torch.bfloat16)
    other.make_plan()
    b.plan = other.plan
    b.run()
    assert all((x == 7.0).all() for x in b.outputs().values())


# A captured step follows the offsets that a replay finds, also between the program's own eager work.
def test_graph_follows_the_offsets():
    b = Batch([100, 60, 40], 4, 2, 64, True, torch.bfloat16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.make_plan()
        b.run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.make_plan()
        b.run()
    for lengths in ([100, 60, 40], [1, 198, 1], [0, 77, 123], [100, 60, 40]):
        b.offsets = [0, lengths[0], lengths[0] + lengths[1], sum(lengths)]
        b.on_gpu.copy_(torch.tensor(b.offsets, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        got = {k: x.clone() for k, x in b.outputs().items()}
        b.check()
        b.make_plan()
        b.run()
        assert all(torch.equal(x, got[k]) for k, x in b.outputs().items())


def test_two_batches_on_two_streams():
    a, b = Batch([300, 20], 4, 2, 64, True, torch.bfloat16), Batch([50, 400], 2, 1, 128, False, torch.bfloat16, seed=5)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for s, x in zip(streams, (a, b)):
        with torch.cuda.stream(s):
            x.make_plan()
            x.run()
    torch.cuda.synchronize()
    a.check()
    b.check()


# dQ, dK, dV against differences of the forward pass in float
def test_gradient_against_differences():
    nq, nkv, dh, lengths = 2, 1, 8, [5, 3]
    b = Batch(lengths, nq, nkv, dh, True, torch.float32)
    b.make_plan()
    b.run()
    x, step = b.qkv.clone(), 2.0 ** -6
    d_o = b.d_o.double()

    def value(qkv):
        b.pkg.tp_layer_attn_packed_fwd(*b.dims, b.plan, qkv, b.o, b.lse, b.ws, stream=torch.cuda.current_stream())
        return (b.o.double() * d_o).sum().item()
    for i, j in [(0, 0), (2, 3), (4, 17), (3, 25), (5, 9), (7, 30), (6, 20)]:
        f = []
        for k in (1, -1, 2, -2):
            y = x.clone()
            y[i, j] += k * step
            f.append(value(y))
        diff = (8 * (f[0] - f[1]) - (f[2] - f[3])) / (12 * step)
        # fifth derivative times step^4 / 30 (softmax of unit values: below 100), and the float outputs' rounding over the step
        tol = 100 * step ** 4 / 30 + 64 * ref.F32 * float((b.o.double().abs() * d_o.abs()).sum()) / step
        assert abs(diff - b.dqkv[i, j].item()) <= tol, (i, j)

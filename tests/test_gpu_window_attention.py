"""Attention with a sliding window and first tokens that stay visible against its definition in 64 bits: windows and first tokens around tiles and strips,
lengths, head sizes, groups, cut strips, what a window hides, rows of no sequence, plans, graphs."""
import math

import pytest

torch = pytest.importorskip("torch")
import packed_ref  # noqa: E402
import window_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu
BF16, FLOAT = torch.bfloat16, torch.float32
check = packed_ref.check


def _rows(seed, *shape, dtype):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(*shape, generator=g).to(dtype).cuda()


class Batch:
    """A packed batch with its plan and workspace; rows behind the last sequence hold `fill`, outputs 7."""

    def __init__(self, lengths, nq, nkv, dh, window, sinks, dtype, behind=0, seed=0, fill=math.nan):
        import paper_2111_05972_amd as pkg
        self.pkg, self.dt = pkg, pkg.TPL_BF16 if dtype == BF16 else pkg.TPL_F32
        self.offsets = [0]
        for n in lengths:
            self.offsets.append(self.offsets[-1] + n)
        self.used = self.offsets[-1]
        self.M = self.used + behind
        self.dims = (self.dt, len(lengths), self.M, nq, nkv, dh, window, sinks)
        self.qkv, self.d_o = _rows(seed, self.M, (nq + 2 * nkv) * dh, dtype=dtype), _rows(seed + 1, self.M, nq * dh, dtype=dtype)
        self.qkv[self.used:] = fill
        self.d_o[self.used:] = fill
        self.on_gpu = torch.tensor(self.offsets, dtype=torch.int32, device="cuda")
        self.plan = torch.full((pkg.tp_layer_window_plan_bytes(len(lengths), self.M, nq, nkv),), 255, dtype=torch.uint8, device="cuda")
        need = max(pkg.tp_layer_attn_window_workspace_bytes(*self.dims, b) for b in (0, 1))
        self.ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
        self.o, self.lse = torch.full((self.M, nq * dh), 7.0, dtype=dtype, device="cuda"), torch.full((self.M, nq), 7.0, device="cuda")
        self.dsum, self.dqkv = torch.full((self.M, nq), math.nan, device="cuda"), torch.full_like(self.qkv, 7.0)

    def make_plan(self):
        _, n, M, nq, nkv, _, window, sinks = self.dims
        self.pkg.tp_layer_window_plan(n, M, self.on_gpu, nq, nkv, window, sinks, self.plan, stream=torch.cuda.current_stream())

    def forward(self):
        self.pkg.tp_layer_attn_window_fwd(*self.dims, self.plan, self.qkv, self.o, self.lse, self.ws, stream=torch.cuda.current_stream())

    def run(self):
        self.forward()
        self.pkg.tp_layer_attn_window_bwd(*self.dims, self.plan, self.qkv, self.o, self.lse, self.d_o, self.dqkv, self.dsum, self.ws,
                                          stream=torch.cuda.current_stream())

    def outputs(self):
        return {"o": self.o, "lse": self.lse, "dqkv": self.dqkv}

    def expected(self):
        return ref.attention(self.qkv, self.offsets, *self.dims[3:], self.d_o)

    def check(self):
        val, tol = self.expected()
        for k, x in self.outputs().items():
            check(x, val[k], tol[k], k)
            assert (x[self.used:] == 7.0).all(), f"{k}: rows behind the last sequence"


def _run(*args, **kw):
    b = Batch(*args, **kw)
    b.make_plan()
    b.run()
    torch.cuda.synchronize()
    b.check()
    return b


@pytest.mark.parametrize("lengths,nq", [([1], 1), ([1], 128), ([2, 1, 1, 3], 7), ([0, 0, 5], 2), ([1] * 70, 3)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (2, 1), (100, 100)])
@pytest.mark.parametrize("dtype", [BF16, FLOAT])
def test_few_tokens(lengths, nq, window, sinks, dtype):
    _run(lengths, nq, 1, 64, window, sinks, dtype)


# windows and first tokens that end at, before and behind the ends of tiles (64) and strips (128)
@pytest.mark.parametrize("window", [1, 2, 33, 63, 64, 65, 127, 128, 129, 200])
@pytest.mark.parametrize("sinks", [0, 1, 64, 70])
@pytest.mark.parametrize("dtype,nq,nkv,dh", [(BF16, 2, 2, 64), (BF16, 5, 1, 80), (FLOAT, 3, 1, 64)])
def test_edges(window, sinks, dtype, nq, nkv, dh):
    _run([1, 0, 63, 300, 65, 0], nq, nkv, dh, window, sinks, dtype, behind=3)


# the same beside a long document: heads of up to 64 have a backward form for short strips (what is above) and one for long ones
@pytest.mark.parametrize("window,sinks", [(64, 0), (65, 70), (500, 1), (2000, 0)])
@pytest.mark.parametrize("nq,nkv,dh", [(8, 1, 64), (12, 2, 32), (8, 1, 40)])
def test_edges_beside_a_long_document(nq, nkv, dh, window, sinks):
    _run([1, 0, 63, 300, 65, 0, 1, 1300], nq, nkv, dh, window, sinks, BF16, behind=3)


# and short strips that fill the chip: more than two strips of keys to a compute unit
@pytest.mark.parametrize("window,sinks", [(200, 3), (1, 0), (40, 0)])
def test_short_strips_that_fill_the_chip(window, sinks):
    _run([520, 0, 300, 270], 64, 64, 64, window, sinks, BF16, behind=2)


@pytest.mark.parametrize("dtype", [BF16, FLOAT])
@pytest.mark.parametrize("dh", [8, 32, 40, 96, 104, 128])
def test_head_sizes(dh, dtype):
    _run([33, 1, 260], 5, 1, dh, 70, 3, dtype, behind=1)


@pytest.mark.parametrize("nq,nkv", [(6, 2), (8, 8), (16, 2), (100, 1)])
@pytest.mark.parametrize("window,sinks", [(30, 4), (90, 0), (40, 130)])
def test_groups(nq, nkv, window, sinks):
    _run([200, 7], nq, nkv, 64, window, sinks, BF16)


# first tokens past a strip of keys, and a window smaller than they are
@pytest.mark.parametrize("dtype", [BF16, FLOAT])
@pytest.mark.parametrize("window,sinks", [(1, 150), (10, 257), (64, 128), (100, 127), (3, 5)])
def test_many_first_tokens(window, sinks, dtype):
    _run([500, 150, 30], 2, 1, 32, window, sinks, dtype, behind=2)


# strips long enough to be cut on either side: by the window, and by first keys that every later row sees
@pytest.mark.parametrize("dtype,dh,nq", [(BF16, 128, 1), (BF16, 64, 3), (BF16, 80, 2), (FLOAT, 64, 2), (FLOAT, 32, 1)])
@pytest.mark.parametrize("window,sinks", [(1500, 0), (40, 4), (700, 100), (10, 700)])
def test_cut_strips(dtype, dh, nq, window, sinks):
    _run([2300, 5, 700], nq, 1, dh, window, sinks, dtype, behind=2)


@pytest.mark.parametrize("dtype", [BF16, FLOAT])
def test_many_lengths(dtype):
    _run(list(range(0, 70)) + [127, 128, 129, 255, 257, 1025], 3, 1, 64, 50, 2, dtype, behind=1)


@pytest.mark.parametrize("dh,nq,nkv", [(64, 16, 8), (128, 4, 4), (32, 12, 12), (96, 16, 4)])
@pytest.mark.parametrize("window,sinks", [(20, 3), (100, 0)])
def test_many_short_sequences_in_float(dh, nq, nkv, window, sinks):
    _run(list(range(0, 60)) + [0, 1, 31, 32, 33, 64, 65, 150, 193] * 2, nq, nkv, dh, window, sinks, FLOAT, behind=1)


# A window that no sequence leaves, or first tokens that are all of them, is the causal mask: the same results, bit for bit where strips are the same.
@pytest.mark.parametrize("dtype", [BF16, FLOAT])
@pytest.mark.parametrize("window,sinks", [(300, 0), (2 ** 31, 5), (2 ** 40, 2 ** 40), (1, 300)])
def test_wide_is_causal(dtype, window, sinks):
    b = _run([300, 20, 100], 4, 2, 64, window, sinks, dtype)
    pkg, (dt, n, M, nq, nkv, dh, _, _) = b.pkg, b.dims
    got = {k: x.clone() for k, x in b.outputs().items()}
    st = torch.cuda.current_stream()
    pkg.tp_layer_pack_plan(n, M, b.on_gpu, nq, nkv, True, b.plan, stream=st)
    args = (dt, n, M, nq, nkv, dh, True, b.plan)
    pkg.tp_layer_attn_packed_fwd(*args, b.qkv, b.o, b.lse, b.ws, stream=st)
    pkg.tp_layer_attn_packed_bwd(*args, b.qkv, b.o, b.lse, b.d_o, b.dqkv, b.dsum, b.ws, stream=st)
    assert all(torch.equal(x, got[k]) for k, x in b.outputs().items())


def test_results_do_not_change_from_run_to_run():
    b = _run([1500, 3, 800], 4, 2, 64, 900, 70, BF16)
    first = {k: x.clone() for k, x in b.outputs().items()}
    for _ in range(3):
        b.make_plan()
        b.run()
        assert all(torch.equal(x, first[k]) for k, x in b.outputs().items())


def test_positions_begin_the_plan():
    b = Batch([3, 0, 70, 1], 2, 1, 64, 5, 1, BF16, behind=4)
    b.make_plan()
    want = [i for n in (3, 0, 70, 1) for i in range(n)] + [0] * 4
    assert b.plan.view(torch.int32)[:b.M].tolist() == want


# Keys that have left the window, and later ones, are as if they were not there; other sequences too.
@pytest.mark.parametrize("dtype,dh", [(BF16, 64), (BF16, 128), (FLOAT, 64)])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("window,sinks,spoilt", [(30, 4, range(40, 50)), (100, 0, range(0, 20)), (20, 70, range(100, 110)), (64, 1, range(1, 64)), (5, 0, range(130, 131))])
def test_hidden_keys_do_not_matter(dtype, dh, bad, window, sinks, spoilt):
    nq, nkv, n = 4, 2, 200
    b = Batch([n, 90], nq, nkv, dh, window, sinks, dtype, behind=2)
    val, tol = b.expected()
    b.qkv.view(b.M, nq + 2 * nkv, dh)[spoilt.start:spoilt.stop, nq:] = bad          # K and V
    b.make_plan()
    b.run()
    reach = ref.sees(n, window, sinks)[:, list(spoilt)].any(1)                      # queries that see one of them
    well = torch.cat([(~reach).nonzero()[:, 0], torch.arange(n, n + 90)])
    assert 90 < well.numel() < n + 90
    for k in ("o", "lse"):
        check(b.outputs()[k][well], val[k][well], tol[k][well], k)
    check(b.dqkv[well][:, :nq * dh], val["dqkv"][well][:, :nq * dh], tol["dqkv"][well][:, :nq * dh], "dq")
    check(b.dqkv[n:n + 90], val["dqkv"][n:n + 90], tol["dqkv"][n:n + 90], "dqkv")


# Backward: a query leaves the keys that it does not see alone, whatever its dO and Q hold.
@pytest.mark.parametrize("dtype,dh", [(BF16, 64), (BF16, 128), (FLOAT, 64)])
@pytest.mark.parametrize("window,sinks,spoilt", [(30, 0, range(40, 50)), (30, 4, range(100, 140)), (100, 0, range(0, 20)), (5, 0, range(130, 131))])
def test_hidden_queries_do_not_matter(dtype, dh, window, sinks, spoilt):
    nq, n = 2, 200
    b = Batch([n, 5], nq, 1, dh, window, sinks, dtype)
    val, tol = b.expected()
    b.d_o[spoilt.start:spoilt.stop] = math.inf
    b.qkv.view(b.M, nq + 2, dh)[spoilt.start:spoilt.stop, :nq] = math.nan
    b.make_plan()
    b.run()
    reached = ref.sees(n, window, sinks)[list(spoilt)].any(0)                       # keys that one of them sees
    well = torch.cat([(~reached).nonzero()[:, 0], torch.arange(n, n + 5)])
    assert well.numel() > 50
    kv = slice(nq * dh, None)
    check(b.dqkv[well][:, kv], val["dqkv"][well][:, kv], tol["dqkv"][well][:, kv], "dk, dv")


# The same where strips are cut into chunks.
@pytest.mark.parametrize("dtype,dh", [(BF16, 64), (BF16, 128), (FLOAT, 64)])
@pytest.mark.parametrize("window,sinks", [(900, 4), (20, 300)])
def test_hidden_values_in_cut_strips(dtype, dh, window, sinks):
    nq, nkv, n = 4, 2, 2000
    b = Batch([n, 60], nq, nkv, dh, window, sinks, dtype, behind=2)
    val, tol = b.expected()
    spoilt = slice(500, 530)
    b.qkv.view(b.M, nq + 2 * nkv, dh)[spoilt, nq:] = math.inf
    b.make_plan()
    b.run()
    well = torch.ones(b.M, dtype=torch.bool)
    well[spoilt.start:spoilt.stop + window] = False
    well[b.used:] = False
    for k in ("o", "lse"):
        check(b.outputs()[k][well.cuda()], val[k][well], tol[k][well], k)
    check(b.dqkv[well.cuda()][:, :nq * dh], val["dqkv"][well][:, :nq * dh], tol["dqkv"][well][:, :nq * dh], "dq")


# A key that rows see and that is NaN makes them NaN, in whole and in cut strips.
@pytest.mark.parametrize("dtype", [BF16, FLOAT])
@pytest.mark.parametrize("n,window", [(200, 50), (2000, 900)])
def test_seen_nan(dtype, n, window):
    b = Batch([n], 1, 1, 64, window, 2, dtype)
    b.qkv[100, 64:] = math.nan
    b.make_plan()
    b.run()
    assert torch.isnan(b.o[100:100 + window]).all() and torch.isnan(b.lse[100:100 + window]).all()
    assert torch.isfinite(b.o[:100]).all() and torch.isfinite(b.o[100 + window:]).all()


def test_offsets_that_decrease_stay_in_bounds():
    b = Batch([40, 30, 30], 2, 1, 64, 20, 2, BF16)
    b.on_gpu = torch.tensor([-5, 60, 20, 1000], dtype=torch.int32, device="cuda")      # taken as 0, 60, 60, 100
    b.make_plan()
    b.run()
    b.offsets = [0, 60, 60, 100]
    b.check()


# A plan of another window, other first tokens or another mask: nothing is written, in either direction.
@pytest.mark.parametrize("dtype", [BF16, FLOAT])
@pytest.mark.parametrize("window,sinks", [(21, 2), (20, 3), (None, None)])
def test_another_plan_writes_nothing(dtype, window, sinks):
    b = Batch([40, 30], 2, 1, 64, 20, 2, dtype)
    _, n, M, nq, nkv, dh, _, _ = b.dims
    st = torch.cuda.current_stream()
    if window is None:
        b.pkg.tp_layer_pack_plan(n, M, b.on_gpu, nq, nkv, True, b.plan, stream=st)
    else:
        b.pkg.tp_layer_window_plan(n, M, b.on_gpu, nq, nkv, window, sinks, b.plan, stream=st)
    b.run()
    assert all((x == 7.0).all() for x in b.outputs().values())
    b.make_plan()                                                       # nor does causal attention with this one
    args = (b.dt, n, M, nq, nkv, dh, True, b.plan)
    b.pkg.tp_layer_attn_packed_fwd(*args, b.qkv, b.o, b.lse, b.ws, stream=st)
    b.pkg.tp_layer_attn_packed_bwd(*args, b.qkv, b.o, b.lse, b.d_o, b.dqkv, b.dsum, b.ws, stream=st)
    assert all((x == 7.0).all() for x in b.outputs().values())


# A captured step follows the offsets that a replay finds, also between the program's own eager work.
def test_graph_follows_the_offsets():
    b = Batch([100, 60, 40], 4, 2, 64, 30, 3, BF16)
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
    a, b = Batch([300, 20], 4, 2, 64, 70, 0, BF16), Batch([50, 400], 2, 1, 128, 33, 5, BF16, seed=5)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for s, x in zip(streams, (a, b)):
        with torch.cuda.stream(s):
            x.make_plan()
            x.run()
    torch.cuda.synchronize()
    a.check()
    b.check()


# The window in rows and values past 2^31 bytes: the last documents of a batch of a million tokens
def test_a_long_batch():
    import paper_2111_05972_amd as pkg
    nq, nkv, dh, each, tail, window, sinks, M = 16, 2, 128, 500, 1000, 150, 4, 1000000
    n = M // each
    st = torch.cuda.current_stream()
    g = torch.Generator(device="cuda").manual_seed(4)
    qkv = torch.empty(M, (nq + 2 * nkv) * dh, dtype=BF16, device="cuda").normal_(generator=g)
    d_o = torch.empty(M, nq * dh, dtype=BF16, device="cuda").normal_(generator=g)
    offsets = torch.arange(0, M + 1, each, dtype=torch.int32, device="cuda")
    plan = torch.empty(pkg.tp_layer_window_plan_bytes(n, M, nq, nkv), dtype=torch.uint8, device="cuda")
    dims = (pkg.TPL_BF16, n, M, nq, nkv, dh, window, sinks)
    ws = torch.empty(max(pkg.tp_layer_attn_window_workspace_bytes(*dims, b) for b in (0, 1)), dtype=torch.uint8, device="cuda")
    pkg.tp_layer_window_plan(n, M, offsets, nq, nkv, window, sinks, plan, stream=st)
    o, lse, dsum, dqkv = torch.empty_like(d_o), torch.empty(M, nq, device="cuda"), torch.empty(M, nq, device="cuda"), torch.empty_like(qkv)
    pkg.tp_layer_attn_window_fwd(*dims, plan, qkv, o, lse, ws, stream=st)
    pkg.tp_layer_attn_window_bwd(*dims, plan, qkv, o, lse, d_o, dqkv, dsum, ws, stream=st)
    torch.cuda.synchronize()
    val, tol = ref.attention(qkv[-tail:], [0, each, tail], nq, nkv, dh, window, sinks, d_o[-tail:])
    for k, x in (("o", o), ("lse", lse), ("dqkv", dqkv)):
        check(x[-tail:], val[k], tol[k], k)


# dQ, dK, dV against differences of the forward pass in float
def test_gradient_against_differences():
    nq, nkv, dh = 2, 1, 8
    b = Batch([7, 3], nq, nkv, dh, 3, 1, FLOAT)
    b.make_plan()
    b.run()
    x, step, d_o = b.qkv.clone(), 2.0 ** -6, b.d_o.double()

    def value(qkv):
        b.pkg.tp_layer_attn_window_fwd(*b.dims, b.plan, qkv, b.o, b.lse, b.ws, stream=torch.cuda.current_stream())
        return (b.o.double() * d_o).sum().item()
    for i, j in [(0, 0), (0, 17), (0, 25), (1, 18), (4, 17), (3, 25), (6, 9), (9, 30), (8, 20)]:
        f = []
        for k in (1, -1, 2, -2):
            y = x.clone()
            y[i, j] += k * step
            f.append(value(y))
        diff = (8 * (f[0] - f[1]) - (f[2] - f[3])) / (12 * step)
        # fifth derivative times step^4 / 30 (softmax of unit values: below 100), and the float outputs' rounding over the step
        tol = 100 * step ** 4 / 30 + 64 * packed_ref.F32 * float((b.o.double().abs() * d_o.abs()).sum()) / step
        assert abs(diff - b.dqkv[i, j].item()) <= tol, (i, j)

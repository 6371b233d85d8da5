"""Host side of the rotary, packed-attention and loss entry points: frequencies, sizes, and calls that are refused before any launch."""
import math

import pytest

import paper_2111_05972_amd as pkg

AT = 0x1000                     # never dereferenced: every call below is refused first
BIG = 1 << 40


def test_frequencies():
    for rot, base in ((128, 10000.0), (2, 500000.0), (20, 10000.0)):
        plain, factor = pkg.tp_layer_rope_frequencies(rot, base)
        assert factor == 1.0 and len(plain) == rot // 2
        for i, f in enumerate(plain):
            assert math.isclose(f, base ** (-2.0 * i / rot), rel_tol=1e-14)
        linear, factor = pkg.tp_layer_rope_frequencies(rot, base, pkg.TPL_ROPE_LINEAR, 4.0)
        assert factor == 1.0 and all(math.isclose(a, b / 4, rel_tol=1e-14) for a, b in zip(linear, plain))
        wider, factor = pkg.tp_layer_rope_frequencies(rot, base, pkg.TPL_ROPE_BASE, 4.0)
        assert factor == 1.0 and wider[0] == 1.0
        if rot > 2:
            assert math.isclose(wider[-1], plain[-1] / 4, rel_tol=1e-13)
        parts, factor = pkg.tp_layer_rope_frequencies(rot, base, pkg.TPL_ROPE_PARTS, 4.0, 4096.0)
        assert math.isclose(factor, 0.1 * math.log(4.0) + 1.0, rel_tol=2.0 ** -23)
        for f, g in zip(parts, plain):
            turns = 4096.0 * g / (2 * math.pi)
            want = g if turns >= 32 else g / 4 if turns <= 1 else None
            assert want is None or math.isclose(f, want, rel_tol=1e-13)
            assert g / 4 <= f * (1 + 1e-13) and f <= g * (1 + 1e-13)
    assert pkg.tp_layer_rope_frequencies(8, 10000.0, pkg.TPL_ROPE_PARTS, 0.5, 64.0)[1] == 1.0


@pytest.mark.parametrize("kw", [dict(rot=0), dict(rot=3), dict(rot=-2), dict(base=0.0), dict(base=math.nan), dict(base=math.inf), dict(scaling=4),
                                dict(scaling=-1), dict(scaling=1, stretch=0.0), dict(scaling=1, stretch=math.nan), dict(scaling=2, stretch=math.inf),
                                dict(scaling=3, stretch=2.0, context=0.0), dict(scaling=3, stretch=2.0, context=math.nan)])
def test_frequencies_refused(kw):
    a = {"rot": 8, "base": 10000.0, "scaling": 0, "stretch": 1.0, "context": 0.0, **kw}
    with pytest.raises(pkg.TpLayerError):
        pkg.tp_layer_rope_frequencies(**a)


@pytest.mark.parametrize("call", [pkg.tp_layer_rope_fwd, pkg.tp_layer_rope_bwd])
def test_rotary_refused(call):
    row = (4 + 2 * 2) * 64 * 2

    def rc(dtype=pkg.TPL_BF16, M=8, nq=4, nkv=2, dh=64, rot=64, pairs=0, freq=AT, positions=AT, qkv=AT, out=AT, seq=0):
        return call(dtype, M, nq, nkv, dh, rot, pairs, freq, 1.0, positions, qkv, out, seq=seq, check=False)
    for kw in (dict(dtype=7), dict(M=0), dict(nq=0), dict(nkv=-1), dict(dh=0), dict(rot=0), dict(rot=5), dict(rot=66), dict(pairs=2), dict(freq=None),
               dict(qkv=None), dict(out=None), dict(positions=None), dict(positions=None, seq=-3),
               dict(out=AT + row), dict(out=AT + 8 * row - 16), dict(qkv=AT + 16)):           # parts of one another
        assert rc(**kw) == pkg.TPL_EINVAL, kw
    for kw in (dict(qkv=AT + 8), dict(out=AT + 4), dict(freq=AT + 8), dict(positions=AT + 4)):
        assert rc(**kw) == pkg.TPL_EALIGN, kw
    for kw in (dict(M=1 << 24), dict(nq=1 << 17), dict(nq=1, nkv=1, dh=2, rot=2), dict(dh=8200), dict(nq=1 << 15, nkv=1 << 15, dh=1024)):
        assert rc(**kw) == pkg.TPL_EUNSUPPORTED, kw


# (sequences, M, nq, nkv)
INVALID = [(0, 8, 2, 2), (1, 0, 2, 2), (1, 8, 0, 1), (1, 8, 2, 0), (1, 8, 3, 2), (-1, 8, 2, 2)]
UNSUPPORTED = [((1 << 20) + 1, 8, 2, 2), (1, (1 << 24) + 1, 1, 1), (1, 8, 1 << 13, 1 << 13), (1, 8, 129, 1), (1, 1 << 24, 128, 1), (1, 1 << 24, 128, 64),
               (1 << 20, 1 << 20, 16, 8), (1, 1 << 24, 32, 32)]


def test_plan_sizes():
    for n, M, nq, nkv in [(1, 1, 1, 1), (3, 1000, 8, 2), (64, 65536, 32, 8), (1 << 16, 1 << 20, 1, 1)]:
        got = pkg.tp_layer_pack_plan_bytes(n, M, nq, nkv)
        # positions, keys seen, offsets and counts of both sides, an item of 32 bytes to each strip that there can be
        least = 4 * (2 * M + 3 * (n + 1)) + 32 * (M * (nq // nkv) // 128 + M // 128 + 2 * n)
        assert least <= got <= 2 * least + (1 << 17) and got % 256 == 0
    for a in INVALID + UNSUPPORTED:
        assert pkg.tp_layer_pack_plan_bytes(*a) == 0, a


def test_plan_refused():
    def rc(dims=(2, 100, 4, 2), offsets=AT, plan=AT, nbytes=BIG):
        return pkg.tp_layer_pack_plan(*dims[:2], offsets, *dims[2:], True, plan, plan_bytes=nbytes, check=False)
    for a in INVALID:
        assert rc(a) == pkg.TPL_EINVAL, a
    for a in UNSUPPORTED:
        assert rc(a) == pkg.TPL_EUNSUPPORTED, a
    assert rc(offsets=None) == pkg.TPL_EINVAL and rc(plan=None) == pkg.TPL_EINVAL
    assert rc(offsets=AT + 2) == pkg.TPL_EALIGN and rc(plan=AT + 8) == pkg.TPL_EALIGN
    assert rc(nbytes=pkg.tp_layer_pack_plan_bytes(2, 100, 4, 2) - 1) == pkg.TPL_EWORKSPACE and rc(nbytes=0) == pkg.TPL_EWORKSPACE


@pytest.mark.parametrize("bwd", [False, True])
def test_packed_attention_refused(bwd):
    names = ["qkv", "o", "lse", "d_o", "dqkv", "d_scratch"] if bwd else ["qkv", "o", "lse"]

    def rc(dtype=pkg.TPL_BF16, dims=(2, 100, 4, 2), dh=64, plan=AT, plan_bytes=BIG, ws=AT, ws_bytes=BIG, **kw):
        call = pkg.tp_layer_attn_packed_bwd if bwd else pkg.tp_layer_attn_packed_fwd
        return call(dtype, *dims, dh, True, plan, *[kw.get(k, AT) for k in names], ws, ws_bytes=ws_bytes, plan_bytes=plan_bytes, check=False)
    for a in INVALID:
        assert rc(dims=a) == pkg.TPL_EINVAL, a
        assert pkg.tp_layer_attn_packed_workspace_bytes(pkg.TPL_BF16, *a, 64, True, bwd) == 0
    for a in UNSUPPORTED:
        assert rc(dims=a) == pkg.TPL_EUNSUPPORTED, a
        assert pkg.tp_layer_attn_packed_workspace_bytes(pkg.TPL_BF16, *a, 64, True, bwd) == 0
    assert rc(dtype=2) == pkg.TPL_EINVAL and rc(dh=0) == pkg.TPL_EINVAL
    for dh in (4, 12, 136, 256):
        assert rc(dh=dh) == pkg.TPL_EUNSUPPORTED, dh
    for k in names + ["plan", "ws"]:
        assert rc(**{k: None}) == pkg.TPL_EINVAL, k
        assert rc(**{k: AT + 4}) == pkg.TPL_EALIGN, k
    assert rc(plan_bytes=pkg.tp_layer_pack_plan_bytes(2, 100, 4, 2) - 1) == pkg.TPL_EWORKSPACE
    for dtype in (pkg.TPL_F32, pkg.TPL_BF16):
        dims = (3, 5000, 8, 2)
        need = pkg.tp_layer_attn_packed_workspace_bytes(dtype, *dims, 128, True, bwd)
        assert need >= 256 and rc(dtype=dtype, dims=dims, dh=128, ws_bytes=need - 1) == pkg.TPL_EWORKSPACE


def test_loss_sizes():
    size = pkg.tp_layer_lm_loss_workspace_bytes
    for dtype, es in ((pkg.TPL_F32, 4), (pkg.TPL_BF16, 2)):
        for M, H, V in [(1, 8, 1), (37, 128, 1001), (4096, 1024, 50000)]:
            assert 0 < size(dtype, M, H, V, False) and es * M * min(V, 256) <= size(dtype, M, H, V, True)
    # The logits of a training step are not kept ([8192, 128000] would be 2 GiB).  Forward: 8 bytes for a token and 256 columns (31.25 MiB), its
    # target (32 KiB), and float sums of the tiles that are cut into K shares, a tile of 256 x 256 to each of 256 units at most (64 MiB).
    # Backward: dz of a piece and dx in float (128 MiB each), sums of shares of two products.
    assert size(pkg.TPL_BF16, 8192, 4096, 128000, False) <= 96 << 20
    assert size(pkg.TPL_BF16, 8192, 4096, 128000, True) <= 640 << 20


LOSS_INVALID = [dict(dtype=9), dict(M=0), dict(H=0), dict(V=0), dict(first=-1)]
LOSS_UNSUPPORTED = [dict(H=68), dict(V=(1 << 24) + 1), dict(M=(1 << 20) + 1, H=8), dict(M=1 << 20, H=1024), dict(H=(1 << 20) + 8, M=1), dict(first=1 << 31),
                    dict(M=1 << 20, H=8, V=1 << 18)]


@pytest.mark.parametrize("which", ["fwd", "bwd"])
def test_loss_refused(which):
    base = dict(dtype=pkg.TPL_BF16, M=64, H=128, V=1000, first=0)
    names = ["x", "w", "labels", "stats"] if which == "fwd" else ["x", "w", "labels", "lse", "dloss", "dx", "dw"]

    def rc(vocab=None, ws=AT, ws_bytes=BIG, **kw):
        d = {k: kw.get(k, v) for k, v in base.items()}
        t = [kw.get(k, AT) for k in names]
        if which == "fwd":
            return pkg.tp_layer_lm_loss_fwd(d["dtype"], d["M"], d["H"], d["V"], d["first"], *t, ws, ws_bytes=ws_bytes, check=False)
        vocab = d["first"] + d["V"] if vocab is None else vocab
        return pkg.tp_layer_lm_loss_bwd(d["dtype"], d["M"], d["H"], d["V"], d["first"], vocab, *t, ws, ws_bytes=ws_bytes, check=False)
    for kw in LOSS_INVALID:
        assert rc(**kw) == pkg.TPL_EINVAL, kw
    for kw in LOSS_UNSUPPORTED:
        assert rc(**kw) == pkg.TPL_EUNSUPPORTED, kw
    for k in names + ["ws"]:
        assert rc(**{k: None}) == pkg.TPL_EINVAL, k
        assert rc(**{k: AT + 2}) == pkg.TPL_EALIGN, k
    need = pkg.tp_layer_lm_loss_workspace_bytes(base["dtype"], base["M"], base["H"], base["V"], which == "bwd")
    assert rc(ws_bytes=need - 1) == pkg.TPL_EWORKSPACE
    if which == "bwd":
        assert rc(vocab=999) == pkg.TPL_EINVAL and rc(vocab=(1 << 30) + 1) == pkg.TPL_EUNSUPPORTED


def test_loss_join_refused():
    def rc(M=8, ranks=2, vocab=100, stats=AT, labels=AT, loss=AT, lse=AT):
        return pkg.tp_layer_lm_loss_join(M, ranks, vocab, stats, labels, loss, lse, check=False)
    for kw in (dict(M=0), dict(ranks=0), dict(vocab=0), dict(stats=None), dict(labels=None), dict(loss=None), dict(lse=None)):
        assert rc(**kw) == pkg.TPL_EINVAL, kw
    for kw in (dict(M=(1 << 24) + 1), dict(ranks=(1 << 16) + 1)):
        assert rc(**kw) == pkg.TPL_EUNSUPPORTED, kw
    for kw in (dict(stats=AT + 4), dict(labels=AT + 2), dict(loss=AT + 1), dict(lse=AT + 2)):
        assert rc(**kw) == pkg.TPL_EALIGN, kw

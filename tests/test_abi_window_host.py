"""Host side of attention with a sliding window: sizes, and calls that are refused before any launch."""
import pytest

import paper_2111_05972_amd as pkg

AT = 0x1000                     # never dereferenced: every call below is refused first
BIG = 1 << 40
INVALID = [(0, 8, 2, 2), (1, 0, 2, 2), (1, 8, 0, 1), (1, 8, 2, 0), (1, 8, 3, 2), (-1, 8, 2, 2)]
UNSUPPORTED = [((1 << 20) + 1, 8, 2, 2), (1, (1 << 24) + 1, 1, 1), (1, 8, 1 << 13, 1 << 13), (1, 8, 129, 1), (1, 1 << 24, 128, 1), (1, 1 << 24, 32, 32)]
MASKS = [(0, 0), (-1, 0), (5, -1), (-(1 << 40), 0)]


def test_sizes():
    for n, M, nq, nkv in [(1, 1, 1, 1), (3, 1000, 8, 2), (64, 65536, 32, 8)]:
        assert pkg.tp_layer_window_plan_bytes(n, M, nq, nkv) == pkg.tp_layer_pack_plan_bytes(n, M, nq, nkv) > 0
    for a in INVALID + UNSUPPORTED:
        assert pkg.tp_layer_window_plan_bytes(*a) == 0, a


def test_plan_refused():
    def rc(dims=(2, 100, 4, 2), mask=(10, 2), offsets=AT, plan=AT, nbytes=BIG):
        return pkg.tp_layer_window_plan(*dims[:2], offsets, *dims[2:], *mask, plan, plan_bytes=nbytes, check=False)
    for a in INVALID:
        assert rc(a) == pkg.TPL_EINVAL, a
    for a in UNSUPPORTED:
        assert rc(a) == pkg.TPL_EUNSUPPORTED, a
    for m in MASKS:
        assert rc(mask=m) == pkg.TPL_EINVAL, m
    assert rc(offsets=None) == pkg.TPL_EINVAL and rc(plan=None) == pkg.TPL_EINVAL
    assert rc(offsets=AT + 2) == pkg.TPL_EALIGN and rc(plan=AT + 8) == pkg.TPL_EALIGN
    assert rc(nbytes=pkg.tp_layer_window_plan_bytes(2, 100, 4, 2) - 1) == pkg.TPL_EWORKSPACE and rc(nbytes=0) == pkg.TPL_EWORKSPACE


@pytest.mark.parametrize("bwd", [False, True])
def test_attention_refused(bwd):
    names = ["qkv", "o", "lse", "d_o", "dqkv", "d_scratch"] if bwd else ["qkv", "o", "lse"]
    size = pkg.tp_layer_attn_window_workspace_bytes

    def rc(dtype=pkg.TPL_BF16, dims=(2, 100, 4, 2), dh=64, mask=(10, 2), plan=AT, plan_bytes=BIG, ws=AT, ws_bytes=BIG, **kw):
        call = pkg.tp_layer_attn_window_bwd if bwd else pkg.tp_layer_attn_window_fwd
        return call(dtype, *dims, dh, *mask, plan, *[kw.get(k, AT) for k in names], ws, ws_bytes=ws_bytes, plan_bytes=plan_bytes, check=False)
    for a in INVALID:
        assert rc(dims=a) == pkg.TPL_EINVAL and size(pkg.TPL_BF16, *a, 64, 10, 2, bwd) == 0, a
    for a in UNSUPPORTED:
        assert rc(dims=a) == pkg.TPL_EUNSUPPORTED and size(pkg.TPL_BF16, *a, 64, 10, 2, bwd) == 0, a
    for m in MASKS:
        assert rc(mask=m) == pkg.TPL_EINVAL and size(pkg.TPL_BF16, 2, 100, 4, 2, 64, *m, bwd) == 0, m
    assert rc(dtype=2) == pkg.TPL_EINVAL and rc(dh=0) == pkg.TPL_EINVAL
    for dh in (4, 12, 136, 256):
        assert rc(dh=dh) == pkg.TPL_EUNSUPPORTED, dh
    for k in names + ["plan", "ws"]:
        assert rc(**{k: None}) == pkg.TPL_EINVAL, k
        assert rc(**{k: AT + 4}) == pkg.TPL_EALIGN, k
    assert rc(plan_bytes=pkg.tp_layer_window_plan_bytes(2, 100, 4, 2) - 1) == pkg.TPL_EWORKSPACE
    for dtype in (pkg.TPL_F32, pkg.TPL_BF16):
        dims = (3, 5000, 8, 2)
        need = size(dtype, *dims, 128, 700, 5, bwd)
        assert need >= 256 and rc(dtype=dtype, dims=dims, dh=128, mask=(700, 5), ws_bytes=need - 1) == pkg.TPL_EWORKSPACE

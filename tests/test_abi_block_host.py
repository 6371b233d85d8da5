"""Host side of the norms of heads with the rotation and of dropout: sizes, and calls that are refused before any launch."""
import math

import pytest

import paper_2111_05972_amd as pkg

AT = 0x100000                   # never dereferenced: every call below is refused first
FAR = {k: AT * (i + 2) for i, k in enumerate(["qkv", "dqkv", "out", "x", "resid", "dout", "din"])}
BIG = 1 << 40


@pytest.mark.parametrize("bwd", [False, True])
def test_norm_refused(bwd):
    names = ["qkv", "dqkv", "out", "dgamma_q", "dgamma_k", "ws"] if bwd else ["qkv", "out"]
    row = (4 + 2 * 2) * 64 * 2

    def rc(dtype=pkg.TPL_BF16, M=8, nq=4, nkv=2, dh=64, rot=64, pairs=0, freq=AT, positions=AT, gamma_q=AT, gamma_k=AT, eps=1e-6, seq=0, ws_bytes=BIG, **kw):
        head = (dtype, M, nq, nkv, dh, rot, pairs, freq, 1.0, positions, gamma_q, gamma_k, True, eps)
        rest = [kw.get(k, FAR.get(k, AT)) for k in names]
        if bwd:
            return pkg.tp_layer_qk_norm_rope_bwd(*head, *rest, ws_bytes=ws_bytes, seq=seq, check=False)
        return pkg.tp_layer_qk_norm_rope_fwd(*head, *rest, seq=seq, check=False)
    for kw in (dict(dtype=7), dict(M=0), dict(nq=0), dict(nkv=-1), dict(dh=0), dict(rot=0), dict(rot=5), dict(rot=66), dict(pairs=2), dict(freq=None),
               dict(gamma_q=None), dict(gamma_k=None), dict(positions=None), dict(positions=None, seq=-3), dict(eps=-1e-6), dict(eps=math.nan), dict(eps=math.inf)):
        assert rc(**kw) == pkg.TPL_EINVAL, kw
    for k in names:
        assert rc(**{k: None}) == pkg.TPL_EINVAL, k
        assert rc(**{k: AT + 8}) == pkg.TPL_EALIGN, k
    for k in ("freq", "positions", "gamma_q", "gamma_k"):
        assert rc(**{k: AT + 4}) == pkg.TPL_EALIGN, k
    for kw in (dict(M=1 << 24), dict(nq=4097), dict(nkv=4097), dict(dh=520), dict(dh=68), dict(dh=4, rot=4)):
        assert rc(**kw) == pkg.TPL_EUNSUPPORTED, kw
    # parts of one another; in backward the input of before the norm has to stay
    for kw in ([dict(out=FAR["dqkv"] + row), dict(out=FAR["dqkv"] - 8 * row + 16), dict(out=FAR["qkv"]), dict(out=FAR["qkv"] + row)] if bwd else
               [dict(out=FAR["qkv"] + row), dict(out=FAR["qkv"] - 8 * row + 16)]):
        assert rc(**kw) == pkg.TPL_EINVAL, kw
    if bwd:
        need = pkg.tp_layer_qk_norm_rope_workspace_bytes(pkg.TPL_BF16, 8, 4, 2, 64)
        assert need > 0 and rc(ws_bytes=need - 1) == pkg.TPL_EWORKSPACE
    for a in ((9, 8, 4, 2, 64), (1, 0, 4, 2, 64), (1, 8, 0, 2, 64), (1, 8, 4, 2, 60), (1, 1 << 24, 4, 2, 64)):
        assert pkg.tp_layer_qk_norm_rope_workspace_bytes(*a) == 0


@pytest.mark.parametrize("bwd", [False, True])
def test_dropout_refused(bwd):
    names = ["dout", "din", "dbias", "ws"] if bwd else ["x", "bias", "resid", "out"]

    def rc(dtype=pkg.TPL_BF16, M=8, N=64, p=0.1, rng=AT, site=3, first_row=0, first_col=0, width=64, ws_bytes=BIG, **kw):
        head = (dtype, M, N, p, rng, site, first_row, first_col, width)
        rest = [kw.get(k, FAR.get(k, AT)) for k in names]
        return pkg.tp_layer_dropout_bwd(*head, *rest, ws_bytes=ws_bytes, check=False) if bwd else pkg.tp_layer_dropout_fwd(*head, *rest, check=False)
    for kw in (dict(dtype=2), dict(M=0), dict(N=0), dict(p=-0.1), dict(p=1.0), dict(p=math.nan), dict(rng=None), dict(site=-1), dict(first_row=-1), dict(first_col=-8),
               dict(width=56), dict(first_col=8), dict(first_col=1 << 62), dict(width=72, first_col=16)):
        assert rc(**kw) == pkg.TPL_EINVAL, kw
    for kw in (dict(N=60), dict(width=68), dict(width=80, first_col=4), dict(site=1 << 20), dict(M=1 << 31), dict(width=1 << 31), dict(first_row=1 << 44),
               dict(first_row=(1 << 41) - 7), dict(first_row=(1 << 63) - 1)):
        assert rc(**kw) == pkg.TPL_EUNSUPPORTED, kw
    for k in names[:2] if bwd else ["x", "out"]:
        assert rc(**{k: None}) == pkg.TPL_EINVAL, k
    for k in names:
        assert rc(**{k: AT + 8}) == pkg.TPL_EALIGN, k
    assert rc(rng=AT + 4) == pkg.TPL_EALIGN
    if bwd:
        assert rc(din=FAR["dout"] + 16) == pkg.TPL_EINVAL and rc(ws=None) == pkg.TPL_EINVAL
        need = pkg.tp_layer_dropout_workspace_bytes(8, 64)
        assert need > 0 and rc(ws_bytes=need - 1) == pkg.TPL_EWORKSPACE
    else:
        assert rc(out=FAR["x"] + 16) == pkg.TPL_EINVAL and rc(out=FAR["resid"] - 16) == pkg.TPL_EINVAL
    for a in ((0, 8), (8, 0), (8, 12), (1 << 31, 8), (8, 1 << 31)):
        assert pkg.tp_layer_dropout_workspace_bytes(*a) == 0


# Published known answers of Philox4x32-10: counter and key of zeros, of ones, and of the digits of pi.
def test_the_generator_of_the_definition():
    block_ref = pytest.importorskip("block_ref")
    assert block_ref.philox([0] * 4, [0] * 2) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert block_ref.philox([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert block_ref.philox([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0]) == [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


# Entry points that are called without ctypes: the same arguments, and what is not one of them.
def test_arguments_that_are_none():
    lib = pkg.load_library()
    call = lib.tp_layer_dropout_workspace_bytes
    assert call(8, 64) > 0 and call(True, 64) > 0
    for bad in ((8,), (8, 64, 1), ()):
        with pytest.raises(TypeError):
            call(*bad)
    for bad in ((8.5, 64), ("8", 64), (None, 64)):
        with pytest.raises(TypeError):
            call(*bad)
    with pytest.raises(OverflowError):
        call(1 << 63, 64)
    plan = (2, 100, AT, 4, 2, True, AT)
    with pytest.raises(OverflowError):
        pkg.tp_layer_pack_plan(*plan, plan_bytes=-1)
    with pytest.raises(OverflowError):
        pkg.tp_layer_pack_plan(2, 100, AT, 1 << 31, 2, True, AT, plan_bytes=0)
    with pytest.raises(TypeError):
        pkg.tp_layer_pack_plan(2, 100, "offsets", 4, 2, True, AT, plan_bytes=0)


class _Tensor:
    """Something with an address: aligned or not."""

    def __init__(self, address):
        self.address, self.nbytes = address, 0

    def data_ptr(self):
        return self.address


class _Stream:
    cuda_stream = 0


def test_tensors_and_streams_are_pointers():
    for stream in (None, 0, _Stream(), _Stream()):
        def rc(offsets, plan, stream=stream):
            return pkg.tp_layer_pack_plan(2, 100, offsets, 4, 2, True, plan, stream=stream, check=False)
        assert rc(_Tensor(AT), _Tensor(AT)) == pkg.TPL_EWORKSPACE          # of no bytes
        assert rc(_Tensor(AT), _Tensor(AT + 8)) == pkg.TPL_EALIGN and rc(_Tensor(AT + 2), _Tensor(AT)) == pkg.TPL_EALIGN
        assert rc(_Tensor(0), _Tensor(AT)) == pkg.TPL_EINVAL and rc(None, AT) == pkg.TPL_EINVAL

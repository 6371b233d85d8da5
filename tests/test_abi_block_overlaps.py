"""Norms of heads with the rotation, and dropout: tensors that overlap where they may not are refused before any launch, whichever they are."""
import pytest

import paper_2111_05972_amd as pkg

STEP = 0x100000                 # never dereferenced: every call below is refused first


@pytest.mark.parametrize("dtype,es", [(pkg.TPL_BF16, 2), (pkg.TPL_F32, 4)])
@pytest.mark.parametrize("per_head", [False, True])
@pytest.mark.parametrize("bwd", [False, True])
def test_norm(bwd, per_head, dtype, es):
    M, nq, nkv, dh, rot = 64, 4, 2, 64, 48
    need = pkg.tp_layer_qk_norm_rope_workspace_bytes(dtype, M, nq, nkv, dh)
    rows = M * (nq + 2 * nkv) * dh * es
    size = {"freq": rot // 2 * 8, "positions": 4 * M, "gamma_q": (nq if per_head else 1) * dh * es, "gamma_k": (nkv if per_head else 1) * dh * es, "qkv": rows, "out": rows}
    outs = ["out"]
    if bwd:
        size.update(dqkv=rows, dgamma_q=size["gamma_q"], dgamma_k=size["gamma_k"], ws=need)
        outs += ["dgamma_q", "dgamma_k", "ws"]
    at = {k: STEP * (i + 1) for i, k in enumerate(size)}

    def rc(**kw):
        a = {**at, **kw}
        head = (dtype, M, nq, nkv, dh, rot, 0, a["freq"], 1.0, a["positions"], a["gamma_q"], a["gamma_k"], per_head, 1e-6, a["qkv"])
        if bwd:
            return pkg.tp_layer_qk_norm_rope_bwd(*head, a["dqkv"], a["out"], a["dgamma_q"], a["dgamma_k"], a["ws"], ws_bytes=need, check=False)
        return pkg.tp_layer_qk_norm_rope_fwd(*head, a["out"], check=False)

    for o in outs:
        for k in size:
            if k == o:
                continue
            # the last 16 bytes of the one are the first of the other
            for place in {at[k] - size[o] + 16, at[k] + size[k] - 16} | (set() if (o, k) in (("out", "qkv"), ("out", "dqkv")) else {at[k]}):
                assert rc(**{o: place}) == pkg.TPL_EINVAL, (o, k, place - at[k])
    if bwd:
        assert rc(out=at["qkv"]) == pkg.TPL_EINVAL


@pytest.mark.parametrize("dtype,es", [(pkg.TPL_BF16, 2), (pkg.TPL_F32, 4)])
@pytest.mark.parametrize("bwd", [False, True])
def test_dropout(bwd, dtype, es):
    M, N = 64, 128
    need = pkg.tp_layer_dropout_workspace_bytes(M, N)
    whole = M * N * es
    size = {"rng": 16, "dout": whole, "din": whole, "dbias": N * es, "ws": need} if bwd else {"rng": 16, "x": whole, "bias": N * es, "resid": whole, "out": whole}
    at = {k: STEP * (i + 1) for i, k in enumerate(size)}

    def rc(**kw):
        a = {**at, **kw}
        head = (dtype, M, N, 0.1, a["rng"], 3, 0, 0, N)
        if bwd:
            return pkg.tp_layer_dropout_bwd(*head, a["dout"], a["din"], a["dbias"], a["ws"], ws_bytes=need, check=False)
        return pkg.tp_layer_dropout_fwd(*head, a["x"], a["bias"], a["resid"], a["out"], check=False)

    for o in ("din", "dbias", "ws") if bwd else ("out",):
        for k in size:
            if k == o:
                continue
            for place in {at[k] - size[o] + 16, at[k] + size[k] - 16} | (set() if (o, k) in (("out", "x"), ("out", "resid"), ("din", "dout")) else {at[k]}):
                assert rc(**{o: place}) == pkg.TPL_EINVAL, (o, k, place - at[k])

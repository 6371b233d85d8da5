"""Packed attention: a NaN that a row sees comes out of it, wherever the strip was cut.  A chunk all of whose scores are NaN has no largest score, and
its sum is NaN: joined with the others it may not pass for a chunk that the mask hides."""
import math

import pytest

torch = pytest.importorskip("torch")
import packed_ref as ref  # noqa: E402
from test_gpu_packed_attention import Batch  # noqa: E402

pytestmark = pytest.mark.gpu
NQ, NKV, LONG, OTHER = 4, 2, 2304, 60


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,dh", [(torch.bfloat16, 64), (torch.bfloat16, 128), (torch.float32, 64)])
@pytest.mark.parametrize("first,last", [(0, 576), (576, 1728), (0, 1728), (700, 701)])
def test_keys_that_are_nan(dtype, dh, first, last, causal):
    b = Batch([LONG, OTHER], NQ, NKV, dh, causal, dtype, behind=1)
    val, tol = ref.attention(b.qkv, b.offsets, NQ, NKV, dh, causal)
    b.qkv.view(b.M, NQ + 2 * NKV, dh)[first:last, NQ:NQ + NKV] = math.nan
    b.make_plan()
    b.pkg.tp_layer_attn_packed_fwd(*b.dims, b.plan, b.qkv, b.o, b.lse, b.ws, stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    blind = first if causal else 0                                       # rows that see none of them
    assert torch.isnan(b.o[blind:LONG].float()).all(), "o"
    assert torch.isnan(b.lse[blind:LONG]).all(), "lse"
    for k in ("o", "lse"):
        ref.check(b.outputs()[k][:blind], val[k][:blind], tol[k][:blind], k)
        ref.check(b.outputs()[k][LONG:LONG + OTHER], val[k][LONG:LONG + OTHER], tol[k][LONG:LONG + OTHER], k)

"""Values that a diverging training step meets: what is not finite shows where it is met."""
import math

import pytest
import torch

import train_reference as ref
from test_gpu_train_ops import BF16, F32, attn_inputs, normal

pytestmark = pytest.mark.gpu
TYPES = pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])


@pytest.fixture(scope="module")
def ps():
    import paper_2410_05589_b200 as ps
    assert torch.cuda.is_available()
    return ps


# ---- no score above -inf ------------------------------------------------------------------------------------

@pytest.mark.parametrize("n_ctx, n_groups, heads", [([40], [30], 2), ([700], [3], 2), ([0, 300], [120, 130], 64)],
                         ids=["one part", "several parts", "many tiles"])
@pytest.mark.parametrize("odd", [False, True], ids=["aligned", "odd"])
@TYPES
def test_row_whose_scores_are_all_minus_infinity_is_no_number(ps, n_ctx, n_groups, heads, odd, dtype):
    """exp(-inf - lse) with lse = -inf is no number: on every path, whatever the type, the alignment and the parts of the keys."""
    k, d = 4, 64
    q, kk, v, do = attn_inputs(61, n_ctx, n_groups, k, heads, heads, d, dtype)
    kk[..., 0] = 1.0
    bad = [1, 11]
    q[bad, :, 0] = -math.inf
    if odd:   # (off a 16-byte boundary: the kernels of the FMA units)
        buf = torch.empty(v.numel() + 1, dtype=dtype, device="cuda")
        v = buf[1:].view(v.shape).copy_(v)
    at = dict(n_ctx=n_ctx, n_groups=n_groups, k_masks=k)
    r = ps.group_attention(q, kk, v, **at)
    r |= ps.group_attention_backward(do, q, kk, v, r["out"], r["lse"], **at)
    assert torch.isnan(r["out"][bad]).all() and (r["lse"][:, bad] == -math.inf).all()
    assert torch.isnan(r["dq"][bad]).all()
    good = torch.ones(q.shape[0], dtype=torch.bool, device="cuda")
    good[bad] = False
    assert torch.isfinite(r["out"][good]).all() and torch.isfinite(r["lse"][:, good]).all() and torch.isfinite(r["dq"][good]).all()

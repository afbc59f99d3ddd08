"""The training operators on the GPU against their 64-bit forms (train_reference), at the sizes, masks, strides and
types where a kernel can go wrong."""
import pytest
import torch

import train_reference as ref

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def ps():
    import paper_2410_05589_b200 as ps
    assert torch.cuda.is_available()
    return ps


def normal(seed, shape, sigma=1.0, dtype=F32):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * sigma).to(dtype).cuda()


# ---- attention under the groups' mask -----------------------------------------------------------------

def attn_inputs(seed, n_ctx, n_groups, k, nh, nkv, d, dtype, spread=1.0):
    R = k + 1
    rq, rkv = sum(n_groups) * R, sum(n_ctx) + sum(n_groups) * R
    return (normal(seed, (rq, nh, d), spread, dtype), normal(seed + 1, (rkv, nkv, d), spread, dtype),
            normal(seed + 2, (rkv, nkv, d), 1.0, dtype), normal(seed + 3, (rq, nh, d), 1.0, dtype))


ATTN = [  # n_ctx, n_groups, k_masks, query heads, key heads
    ([0], [1], 0, 1, 1),                      # one token
    ([0], [1], 4, 2, 2),                      # one group, no context
    ([5], [1], 15, 2, 1),                     # all masks
    ([0], [129], 0, 2, 2),                    # causal, a row behind a tile
    ([64], [64], 1, 1, 1),                    # whole tiles
    ([127], [26], 4, 2, 2),                   # one group behind a query tile of 128 rows
    ([129], [25], 4, 3, 1),
    ([300], [2], 4, 2, 2),                    # few rows, long context
    ([0, 7, 0, 130, 1], [3, 0, 0, 61, 128], 2, 4, 2),   # empty sequences, context only, ragged
    ([33, 1], [16, 9], 15, 2, 2),
    ([0, 257], [300, 40], 7, 2, 1),
    ([10] * 20, list(range(20)), 3, 2, 2),
]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("shape", ATTN, ids=lambda s: f"c{sum(s[0])}g{sum(s[1])}k{s[2]}h{s[3]}x{s[4]}b{len(s[0])}")
def test_attention_and_its_gradients(ps, shape, dtype, d):
    n_ctx, n_groups, k, nh, nkv = shape
    q, kk, v, do = attn_inputs(7, n_ctx, n_groups, k, nh, nkv, d, dtype)
    at = dict(n_ctx=n_ctx, n_groups=n_groups, k_masks=k)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = ps.group_attention(q, kk, v, status=status, **at)
    got |= ps.group_attention_backward(do, q, kk, v, got["out"], got["lse"], status=status, **at)
    val, bnd = ref.attention(q, kk, v, do, n_ctx, n_groups, k, d ** -0.5)
    assert status.item() == 0
    ref.check(got, val, bnd, ("out", "lse", "dq", "dk", "dv"))


# ---- loss of the LM head --------------------------------------------------------------------------------

def loss_inputs(seed, rows, H, V, ignored, dtype):
    x, w = normal(seed, (rows, H), 1.0, dtype), normal(seed + 1, (V, H), 0.1, dtype)
    g = torch.Generator().manual_seed(seed + 2)
    labels = torch.randint(0, V, (rows,), generator=g, dtype=torch.int32)
    labels[torch.rand(rows, generator=g) < ignored] = -100
    if rows > 2:
        labels[0], labels[1] = 0, V - 1
    return x, w, labels.cuda(), (torch.rand(rows, generator=g) + 0.1).cuda()


LOSS = [  # rows, hidden, vocab, share of ignored rows
    (1, 8, 1, 0.0), (1, 64, 2, 0.0), (3, 72, 257, 0.0), (5, 256, 1000, 0.3), (64, 64, 64, 0.0), (129, 136, 513, 0.5),
    (257, 320, 1500, 0.1), (300, 768, 5000, 0.2), (513, 264, 255, 0.9), (40, 64, 8, 1.0),
]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("shape", LOSS, ids=lambda s: "x".join(map(str, s)))
def test_loss_and_its_gradients(ps, shape, dtype):
    rows, H, V, ignored = shape
    x, w, labels, up = loss_inputs(3, rows, H, V, ignored, dtype)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = ps.lm_loss(x, w, labels, status=status)
    got |= ps.lm_loss_backward(x, w, labels, got["lse"], up, status=status)
    val, bnd = ref.loss(x, w, labels, up)
    assert status.item() == 0
    ref.check(got, val, bnd, ("loss", "lse", "dx", "dw"))


# ---- embedding rows ---------------------------------------------------------------------------------------

EMBED = [  # rows, hidden, vocab, masks
    (1, 8, 1, 0), (1, 256, 50, 4), (31, 7, 5, 1), (33, 64, 3, 2), (700, 40, 1000, 4), (257, 768, 5000, 15), (2000, 24, 2, 1),
]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("shape", EMBED, ids=lambda s: "x".join(map(str, s)))
def test_embedding_rows_and_their_gradients(ps, shape, dtype):
    rows, H, V, k = shape
    g = torch.Generator().manual_seed(5)
    ids = torch.randint(-1, V + k + 1, (rows,), generator=g, dtype=torch.int32)   # (padded rows on either side)
    ids[rows // 3:rows // 2] = V if k else 0                                      # one id with many rows
    ids = ids.cuda()
    table, masks = normal(1, (V, H), 1.0, dtype), normal(2, (k, H), 1.0, dtype) if k else None
    dout = normal(3, (rows, H), 1.0, dtype)
    got = {"out": ps.embed_rows(ids, table, masks, scale=1.7)}
    got |= ps.embed_rows_backward(ids, dout, V, k, scale=1.7)
    val, bnd = ref.embed(ids, table, masks, 1.7, dout)
    ref.check(got, val, bnd, ("out", "d_table", "d_mask") if k else ("out", "d_table"))


@pytest.mark.parametrize("odd", [False, True], ids=["aligned", "odd"])
@pytest.mark.parametrize("shape", [([0], [1], 1, 4, 1), ([1], [1], 0, 8, 8), ([0], [3], 4, 6, 2), ([0, 60], [2, 2], 3, 4, 4)],
                         ids=lambda s: f"c{sum(s[0])}g{sum(s[1])}k{s[2]}")
def test_gradients_of_rows_with_few_keys(ps, shape, odd):
    """p (dP - delta) is a difference of near numbers where one of a few keys has most of the weight: a delta from the
    rounded out would show in dq and dk with several roundings' size."""
    n_ctx, n_groups, k, nh, nkv = shape
    d = 128
    at = dict(n_ctx=n_ctx, n_groups=n_groups, k_masks=k)
    for seed in range(8):
        q, kk, v, do = attn_inputs(100 + 10 * seed, n_ctx, n_groups, k, nh, nkv, d, BF16, spread=1.5)
        if odd:
            buf = torch.empty(v.numel() + 1, dtype=BF16, device="cuda")
            vv = buf[1:].view(v.shape)
            v = vv.copy_(v)
        got = ps.group_attention(q, kk, v, **at)
        got |= ps.group_attention_backward(do, q, kk, v, got["out"], got["lse"], **at)
        val, bnd = ref.attention(q, kk, v, do, n_ctx, n_groups, k, d ** -0.5)
        ref.check(got, val, bnd, ("out", "lse", "dq", "dk", "dv"))
        for n in ("dq", "dk"):
            # dS and the result are each rounded once: half a step each, no more than twice that over the whole
            off = (got[n].double().cpu() - val[n]).norm() / val[n].norm().clamp_min(1e-30)
            assert off <= 2 * 2.0 ** -8 or val[n].norm() < 1e-6, (n, off.item())

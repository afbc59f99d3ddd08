"""The training operators at sizes whose work does not fit the device at once: blocks that take several units, pairs that take several
tiles, several pieces of the vocabulary, rows numbered in several turns."""
import pytest
import torch

import train_reference as ref
from test_gpu_train_ops import BF16, F32, attn_inputs, loss_inputs, normal

pytestmark = pytest.mark.gpu
TYPES = pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])


@pytest.fixture(scope="module")
def ps():
    import paper_2410_05589_b200 as ps
    assert torch.cuda.is_available()
    return ps


ATTN = [  # n_ctx, n_groups, k_masks, query heads, key heads
    # bf16: 1280 query tiles of a head and 336 key tiles on 148 blocks: nine and three rounds, every other one backwards
    ([5, 130, 0, 64, 129, 1, 33, 90, 128, 77], [100, 90, 77, 101, 96, 80, 99, 51, 76, 93], 4, 32, 16),
    # the steps of a key tile in several parts, which are more than the blocks too
    ([130, 0, 260, 17, 40], [140, 131, 129, 150, 133], 4, 32, 4),
    # causal rows without masks, sequences that end inside tiles
    ([0, 0, 7, 300], [700, 129, 640, 515], 0, 16, 8),
    # eight masks: 14 groups a tile
    ([200, 31], [99, 130], 8, 24, 24),
]


@pytest.mark.parametrize("shape", ATTN, ids=lambda s: f"c{sum(s[0])}g{sum(s[1])}k{s[2]}h{s[3]}x{s[4]}b{len(s[0])}")
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["fp32", "bf16"])
def test_attention_in_several_rounds(ps, shape, dtype):
    n_ctx, n_groups, k, nh, nkv = shape
    d = 64
    q, kk, v, do = attn_inputs(81, n_ctx, n_groups, k, nh, nkv, d, dtype)
    at = dict(n_ctx=n_ctx, n_groups=n_groups, k_masks=k)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = ps.group_attention(q, kk, v, status=status, **at)
    got |= ps.group_attention_backward(do, q, kk, v, got["out"], got["lse"], status=status, **at)
    val, bnd = ref.attention(q, kk, v, do, n_ctx, n_groups, k, d ** -0.5)
    assert status.item() == 0
    ref.check(got, val, bnd, ("out", "lse", "dq", "dk", "dv"))


def test_attention_of_wide_heads_in_several_rounds(ps):
    n_ctx, n_groups, k, nh, nkv, d = [64, 3, 140], [90, 77, 101], 4, 40, 40, 128
    q, kk, v, do = attn_inputs(83, n_ctx, n_groups, k, nh, nkv, d, BF16)
    at = dict(n_ctx=n_ctx, n_groups=n_groups, k_masks=k)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = ps.group_attention(q, kk, v, status=status, **at)
    got |= ps.group_attention_backward(do, q, kk, v, got["out"], got["lse"], status=status, **at)
    val, bnd = ref.attention(q, kk, v, do, n_ctx, n_groups, k, d ** -0.5)
    assert status.item() == 0
    ref.check(got, val, bnd, ("out", "lse", "dq", "dk", "dv"))


LOSS = [  # rows, hidden, vocab, share of ignored rows
    (4200, 72, 33000, 0.75),    # rows numbered in two turns; bf16: three pieces of the vocabulary, the last one short; 645 tiles
    (1025, 64, 33000, 0.0),     # the first size of its own numbering; fp32: two pieces, the last one short
    (2305, 64, 2600, 0.02),     # more row tiles than stand side by side
    (1300, 4104, 1500, 0.05),   # dx and dw in more tiles than pairs
]


@pytest.mark.parametrize("shape", LOSS, ids=lambda s: "x".join(map(str, s)))
@TYPES
def test_loss_in_several_rounds(ps, shape, dtype):
    rows, H, V, ignored = shape
    x, w, labels, up = loss_inputs(85, rows, H, V, ignored, dtype)
    # labels on either side of where a piece may end (multiples of 256), and in the last, short one
    edge = torch.arange(2, min(rows, 2 + 2 * (V // 256)), device="cuda")
    labels[edge] = torch.where(labels[edge] < 0, -100, ((edge // 2) * 256 - edge % 2).int())
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = ps.lm_loss(x, w, labels, status=status)
    got |= ps.lm_loss_backward(x, w, labels, got["lse"], up, status=status)
    val, bnd = ref.loss(x, w, labels, up)
    assert status.item() == 0
    ref.check(got, val, bnd, ("loss", "lse", "dx", "dw"))


@TYPES
def test_embedding_of_a_large_vocabulary(ps, dtype):
    """More ids a block than threads, ids with many rows, padded rows on either side."""
    rows, H, V, k = 3000, 16, 2 ** 18 + 3, 4
    g = torch.Generator().manual_seed(6)
    ids = torch.randint(-1, V + k + 1, (rows,), generator=g, dtype=torch.int32)
    ids[::5] = V + 1
    ids[1::7] = V - 1
    ids[2::50] = 443          # (the first id of a block's range where it has 443)
    ids = ids.cuda()
    table, masks, dout = normal(1, (V, H), 1.0, dtype), normal(2, (k, H), 1.0, dtype), normal(3, (rows, H), 1.0, dtype)
    got = {"out": ps.embed_rows(ids, table, masks, scale=0.7)} | ps.embed_rows_backward(ids, dout, V, k, scale=0.7)
    val, bnd = ref.embed(ids, table, masks, 0.7, dout)
    ref.check(got, val, bnd, ("out", "d_table", "d_mask"))
    # either gradient alone: the same sums, perhaps of pieces that begin elsewhere
    one = ps.embed_rows_backward(ids, dout, V, k, scale=0.7, want_table=False) | ps.embed_rows_backward(ids, dout, V, k, scale=0.7, want_mask=False)
    ref.check(one, val, bnd, ("d_table", "d_mask"))

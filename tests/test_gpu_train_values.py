"""Values that a diverging or a finished training step meets: what is not finite shows where it is met and nowhere else, and at
no other cost to the call; losses of rows that the head is sure of."""
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


# ---- rows that the head is sure of ----------------------------------------------------------------------------

@pytest.mark.parametrize("H, V, logit", [(4096, 1500, 30.0), (1024, 32000, 40.0), (256, 700, 18.0), (64, 1, 5.0), (2048, 257, 60.0)])
@TYPES
def test_loss_of_rows_that_the_head_is_sure_of(ps, H, V, logit, dtype):
    """The label's logit far above the others: loss = log(1 + sum_v exp(s_v - s_label)) is as small as that, and never below zero.

    With d = log sum_{v != label} exp(s_v) - s_label the loss is log(1 + e^d), whose slope e^d / (1 + e^d) is the others' share of
    the probability.  So it may be off by that share of what d is off by (two scores, a sum, an fp32 logarithm and a
    difference of numbers of its parts' size), and by its own roundings."""
    rows = 70
    w = normal(1, (V, H), 0.02, dtype)
    g = torch.Generator().manual_seed(2)
    labels = torch.randint(0, V, (rows,), generator=g, dtype=torch.int32)
    labels[:3] = torch.tensor([0, V - 1, V // 2], dtype=torch.int32)
    own = w[labels.long().cuda()].float()
    x = (own * (logit / own.square().sum(-1, keepdim=True))).to(dtype)
    labels = labels.cuda()
    got = ps.lm_loss(x, w, labels)
    S = x.double().cpu() @ w.double().cpu().T
    lab = labels.long().cpu()
    elem = torch.arange(rows)
    es = (H + 8) * ref.W * (x.double().cpu().abs() @ w.double().cpu().abs().T).amax(-1)
    own_s = S[elem, lab].clone()
    S[elem, lab] = -math.inf
    d = torch.logsumexp(S, -1) - own_s
    want = torch.nn.functional.softplus(d)
    share = torch.sigmoid(d)
    ed = 2 * es + (V + 8) * ref.W + 8 * ref.W * (torch.logsumexp(S, -1).abs().nan_to_num(0, 0, 0) + own_s.abs())
    loss = got["loss"].double().cpu()
    assert (loss >= 0).all(), loss.min().item()
    off = (loss - want).abs()
    assert (off <= share * ed * (1 + ed) + 8 * ref.W * want).all(), (off.max().item(), want.max().item())
    lse = torch.logaddexp(torch.logsumexp(S, -1), own_s)
    assert ((got["lse"].double().cpu() - lse).abs() <= es + (V + 8) * ref.W + 8 * ref.W * lse.abs()).all()


@TYPES
def test_loss_of_extreme_logits(ps, dtype):
    """A label's logit of -inf, of +inf or that is no number, and others of +inf or -inf."""
    V, H = 300, 64
    w = normal(3, (V, H), 0.1, dtype)
    w[:, :4] = 0
    w[7, 0], w[8, 1], w[:, 2], w[9, 3] = 1.0, 1.0, 1.0, math.nan
    x = normal(4, (6, H), 1.0, dtype)
    x[:, :4] = 0
    # rows of which one logit alone is not finite need a w that is: huge products instead of infinite operands
    big = 2.0 ** 127
    x[0, 0], w[7, 0] = big, -2.0     # the label's logit is -inf
    x[1, 0] = -big                   # ... +inf
    x[2, 1], w[8, 1] = big, 2.0      # another one is +inf
    x[3, 1] = -big                   # ... -inf: nothing but one term less
    x[4, 2], w[:, 2] = -big, 2.0     # all of them are -inf
    x[5, 2] = 0
    w[9, 3] = 0
    labels = torch.tensor([7, 7, 5, 5, 5, 5], dtype=torch.int32, device="cuda")
    loss = ps.lm_loss(x, w, labels)["loss"].double().cpu()
    assert loss[0] == math.inf and torch.isnan(loss[[1, 4]]).all() and not torch.isfinite(loss[2])
    S = x[[3, 5]].double().cpu() @ w.double().cpu().T
    want = torch.logsumexp(torch.where(S < -3e38, -math.inf, S), -1) - S[:, 5]
    # (72 roundings of 2^-23 of a sum of 64 products of about 0.06: 3.4e-5 at most for a score, twice that for their difference)
    assert ((loss[[3, 5]] - want).abs() <= 1e-4).all()


@TYPES
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_loss_of_logits_at_the_end_of_single_precision(ps, sign, dtype):
    """Logits of 3e38, whose products with log2(e) are beyond it."""
    V, H = 600, 64
    w, x = torch.zeros((V, H), dtype=dtype, device="cuda"), torch.zeros((4, H), dtype=dtype, device="cuda")
    x[:, 0] = 2.0 ** 126
    w[300, 0] = sign * 3.5          # a logit of +-2.98e38; the others are 0 ...
    w[:, 1] = sign * 3.5
    x[2:, 1] = 2.0 ** 126           # ... or all of them are that
    x[2:, 0] = 0
    labels = torch.tensor([5, 300, 5, 300], dtype=torch.int32, device="cuda")
    r = ps.lm_loss(x, w, labels)
    big = 3.5 * 2.0 ** 126
    want = [math.log(V - 1), big, math.log(V), math.log(V)] if sign < 0 else [big, 0.0, math.log(V), math.log(V)]
    for got, right in zip(r["loss"].tolist(), want):
        # (roundings of an ulp or two of the logit, where the loss is one, or of log(600))
        assert abs(got - right) <= 4 * ref.W * right, (got, right)


def test_logits_of_long_rows(ps):
    """32768 positive terms a logit.  The tensor cores truncate as they add: a part of 4096 terms is 256 steps, each of which takes
    half an ulp of what is there on average, and not more than that again from its terms (an ulp: 2^-23); what is there grows
    evenly to the part's size, so that it is at most 128 ulps of the logit in all, and one for each part that is added (80 in one
    part, 88 in eight; in one chain of 32768 terms 1460)."""
    rows, H, V = 5, 32768, 40
    g = torch.Generator().manual_seed(8)
    x, w = (((torch.rand((n, H), generator=g) + 0.5) * s).bfloat16() for n, s in ((rows, 0.01), (V, 0.02)))
    labels = torch.arange(rows, dtype=torch.int32)
    got = ps.lm_loss(x.cuda(), w.cuda(), labels.cuda())
    S = x.double() @ w.double().T
    lse = torch.logsumexp(S, -1)
    off = (got["lse"].double().cpu() - lse).abs()
    assert (off <= (128 + 8) * ref.W * S.amax(-1) + (V + 8) * ref.W + 4 * ref.W * lse).all(), (off / S.amax(-1) / ref.W).tolist()


@pytest.mark.parametrize("n_ctx, n_groups", [([30], [20]), ([500], [3]), ([0, 60], [70, 40])], ids=["one part", "several parts", "two sequences"])
@pytest.mark.parametrize("d, odd", [(64, False), (128, False), (128, True)], ids=["64", "128", "128 odd"])
@TYPES
def test_scores_far_from_zero(ps, n_ctx, n_groups, d, odd, dtype):
    """Scores of 1e10 to 1e12, more than 2^28 apart: the largest one that a row sees has all of the weight."""
    k, nh = 1, 2
    R = k + 1
    q, kk, v, do = attn_inputs(91, n_ctx, n_groups, k, nh, nh, d, dtype)
    q.zero_(), kk.zero_()
    q[..., 0] = 2.0 ** 20
    if odd:
        v = torch.empty(v.numel() + 1, dtype=dtype, device="cuda")[1:].view(v.shape).copy_(v)
    n = kk.shape[0]
    sizes = (128 + torch.arange(128)[None, :]).double() * 2.0 ** torch.arange(5)[:, None]     # 640 different ones
    order = torch.randperm(640, generator=torch.Generator().manual_seed(4))[:n]
    kk[..., 0] = (sizes.flatten()[order] * 2.0 ** 5).to(dtype).cuda()[:, None]
    for sign in (1.0, -1.0):
        kk *= sign
        r = ps.group_attention(q, kk, v, n_ctx=n_ctx, n_groups=n_groups, k_masks=k)
        q0 = k0 = 0
        for c, g in zip(n_ctx, n_groups):
            sees = ref.group_mask(c, g, R)
            S = kk[k0:k0 + c + g * R, 0, 0].double().cpu() * 2.0 ** 20 * d ** -0.5
            top, at = torch.where(sees, S, -math.inf).max(-1)
            assert (r["lse"][:, q0:q0 + g * R].double().cpu() - top).abs().max() <= 2 * ref.W * top.abs().max()
            assert torch.equal(r["out"][q0:q0 + g * R].cpu(), v[k0:k0 + c + g * R].cpu()[at])
            q0, k0 = q0 + g * R, k0 + c + g * R
        kk *= sign


# ---- a step that has diverged -----------------------------------------------------------------------------------

def times(fn, n):
    fn()
    torch.cuda.synchronize()
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    a.record()
    for _ in range(n):
        fn()
    b.record()
    torch.cuda.synchronize()
    return a.elapsed_time(b) / n


@pytest.mark.parametrize("where", ["do", "v", "k", "q"])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_attention_of_a_step_that_has_diverged(ps, where, bad):
    """One tensor without a finite value: every wait ends as it does otherwise, every value that meets it says so, and the call takes
    no longer by an order of magnitude (a row that is no number is not formed again)."""
    n_ctx, n_groups, k, nh, nkv, d = [300, 0], [500, 430], 4, 8, 2, 64
    q, kk, v, do = attn_inputs(71, n_ctx, n_groups, k, nh, nkv, d, BF16)
    at = dict(n_ctx=n_ctx, n_groups=n_groups, k_masks=k)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def run():
        r = ps.group_attention(q, kk, v, status=status, **at)
        return r | ps.group_attention_backward(do, q, kk, v, r["out"], r["lse"], status=status, **at)

    fine = times(run, 5)
    {"do": do, "v": v, "k": kk, "q": q}[where].fill_(bad)
    r = run()
    for n in ("dq", "dk") + (() if where == "v" else ("dv",)) + (() if where == "do" else ("out",)):
        assert not torch.isfinite(r[n]).any(), n
    assert status.item() == 0
    if math.isnan(bad):
        diverged = times(run, 2)
        assert diverged <= 10 * fine + 1.0, (fine, diverged)


@pytest.mark.parametrize("where", ["do", "v", "k", "q"])
def test_a_diverged_sequence_leaves_its_neighbours_alone(ps, where):
    """Tiles at the end of a sequence reach into the next one's rows: what is not finite there comes to nothing, for every key and
    row of the sequence, at one warp a row over the whole device."""
    n_ctx, n_groups, k, nh, nkv, d = [130, 20, 65], [90, 70, 61], 4, 4, 2, 64
    R = k + 1
    q, kk, v, do = attn_inputs(73, n_ctx, n_groups, k, nh, nkv, d, BF16)
    val, bnd = ref.attention(q, kk, v, do, n_ctx, n_groups, k, d ** -0.5)
    q0, k0 = n_groups[0] * R, n_ctx[0] + n_groups[0] * R
    q1, k1 = q0 + n_groups[1] * R, k0 + n_ctx[1] + n_groups[1] * R
    t = {"do": do, "v": v, "k": kk, "q": q}[where]
    t[(slice(k0, k1) if where in "kv" else slice(q0, q1))] = math.nan
    at = dict(n_ctx=n_ctx, n_groups=n_groups, k_masks=k)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    r = ps.group_attention(q, kk, v, status=status, **at)
    r |= ps.group_attention_backward(do, q, kk, v, r["out"], r["lse"], status=status, **at)
    assert status.item() == 0
    for n in ("out", "dq", "dk", "dv"):
        lo, hi = (k0, k1) if n in ("dk", "dv") else (q0, q1)
        off = (r[n].double().cpu() - val[n]).abs() <= bnd[n] + 1e-30
        assert off[:lo].all() and off[hi:].all(), n
        if n == "dq" or (n == "out" and where != "do"):
            assert torch.isnan(r[n][lo:hi]).all(), n
    off = (r["lse"].double().cpu() - val["lse"]).abs() <= bnd["lse"] + 1e-30
    assert off[:, :q0].all() and off[:, q1:].all()

"""Calls of the training operators off the beaten track: values that are not finite in places that do not count, views and odd
addresses, sizes at the 32-bit edge, streams, captured graphs, repeated calls."""
import math

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


def attn_both(ps, q, k, v, do, scale=None, **at):
    r = ps.group_attention(q, k, v, scale=scale, **at)
    return r | ps.group_attention_backward(do, q, k, v, r["out"], r["lse"], scale=scale, **at)


def within(got, val, bnd):
    return ((got.detach().double().cpu() - val).abs() <= bnd + 1e-30)


# ---- values that are not finite ---------------------------------------------------------------------------

@TYPES
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("where", ["k", "v", "q", "do"])
def test_attention_keeps_what_does_not_see_a_bad_value(ps, where, bad, dtype):
    """One value that is not finite: rows and keys that do not meet it come out as if it were not there."""
    n_ctx, n_groups, k, nh, nkv, d = [70, 5], [60, 30], 4, 2, 1, 64
    R = k + 1
    q, kk, v, do = attn_inputs(11, n_ctx, n_groups, k, nh, nkv, d, dtype)
    val, bnd = ref.attention(q, kk, v, do, n_ctx, n_groups, k, d ** -0.5)
    t = {"k": kk, "v": v, "q": q, "do": do}[where]
    group, place = 40, 2                     # a [MASK] row in the middle of sequence 0 and a real one
    for row in (group * R + place, (group + 1) * R):
        t[row + (n_ctx[0] if where in "kv" else 0), 0, 3] = bad
    got = attn_both(ps, q, kk, v, do, n_ctx=n_ctx, n_groups=n_groups, k_masks=k)
    sees = ref.group_mask(n_ctx[0], n_groups[0], R)
    nq, nk = sees.shape
    hit_q = torch.zeros(q.shape[0], dtype=torch.bool)      # query rows that meet a bad value
    hit_k = torch.zeros(kk.shape[0], dtype=torch.bool)     # keys whose gradients do
    for row in (group * R + place, (group + 1) * R):
        if where in "kv":
            hit_q[:nq] |= sees[:, n_ctx[0] + row]
        else:
            hit_q[row] = True
    hit_k[:nk] = (sees & hit_q[:nq, None]).any(0)
    if where in "kv":
        # the gradient of a bad row is one of its own rows' sums, and so are those of all keys that such rows see
        hit_k[[n_ctx[0] + group * R + place, n_ctx[0] + (group + 1) * R]] = True
    if where == "do":
        assert within(got["out"], val["out"], bnd["out"]).all()
    else:
        clean_rows = ~hit_q
        assert within(got["out"], val["out"], bnd["out"])[clean_rows].all()
        if where != "v":
            assert within(got["lse"], val["lse"], bnd["lse"])[:, clean_rows].all()
    assert within(got["dq"], val["dq"], bnd["dq"])[~hit_q].all()
    for n in ("dk", "dv"):
        assert within(got[n], val[n], bnd[n])[~hit_k].all()
    if math.isnan(bad) and where in "kv":      # and who does meet it says so
        assert torch.isnan(got["out"].float().cpu())[hit_q][:, :, 3].all()


@TYPES
def test_loss_reads_nothing_of_rows_that_do_not_count(ps, dtype):
    x, w, labels, up = loss_inputs(5, 300, 64, 700, 0.4, dtype)
    val, bnd = ref.loss(x, w, labels, up)
    out = labels < 0
    x[out], up[out] = math.nan, math.inf
    labels[out] = torch.tensor([-100, -1, 700, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32).cuda().repeat(300)[:int(out.sum())]
    got = ps.lm_loss(x, w, labels)
    got["lse"][out] = math.nan
    got |= ps.lm_loss_backward(x, w, labels, got["lse"], up)
    got["lse"][out] = 0
    ref.check(got, val, bnd, ("loss", "lse", "dx", "dw"))
    assert (got["dx"][out] == 0).all()


@TYPES
def test_loss_of_logits_that_are_not_finite(ps, dtype):
    x, w, labels, up = loss_inputs(6, 40, 64, 300, 0.0, dtype)
    w[:, 0], x[:, 0] = 0, 0
    w[17, 0], x[3, 0], x[4, 0], x[5, 0] = 1.0, -math.inf, math.inf, math.nan
    good = torch.ones(40, dtype=torch.bool)
    good[3:6] = False
    # 0 times an infinity is no number: rows 3 to 5 have none
    got = ps.lm_loss(x, w, labels)
    assert torch.isnan(got["loss"].cpu()[~good]).all() and torch.isfinite(got["loss"].cpu()[good]).all()
    clean = x.clone()
    clean[3:6] = 0
    val, bnd = ref.loss(clean, w, labels, up)
    for n in ("loss", "lse"):
        assert within(got[n], val[n], bnd[n])[good].all()


@TYPES
def test_embedding_ignores_padded_rows(ps, dtype):
    ids = torch.tensor([3, -1, 5, 99, 3, -7, 12, 11, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32).cuda()
    table, masks, dout = normal(1, (10, 40), 1.0, dtype), normal(2, (3, 40), 1.0, dtype), normal(3, (10, 40), 1.0, dtype)
    val, bnd = ref.embed(ids, table, masks, 0.5, dout)
    dout[[1, 3, 5, 8, 9]] = math.nan
    got = {"out": ps.embed_rows(ids, table, masks, scale=0.5)} | ps.embed_rows_backward(ids, dout, 10, 3, scale=0.5)
    ref.check(got, val, bnd, ("out", "d_table", "d_mask"))
    only = ps.embed_rows_backward(ids, dout, 10, 3, scale=0.5, want_table=False)
    assert set(only) == {"d_mask"} and torch.equal(only["d_mask"], got["d_mask"])
    only = ps.embed_rows_backward(ids, dout, 10, 3, scale=0.5, want_mask=False)
    assert set(only) == {"d_table"} and torch.equal(only["d_table"], got["d_table"])


# ---- views, odd addresses, large strides -----------------------------------------------------------------------

@TYPES
@pytest.mark.parametrize("pad, odd", [(8, 0), (3, 1)], ids=["aligned", "odd"])
def test_attention_on_views(ps, pad, odd, dtype):
    """q, k and v as parts of one buffer, gradients into another; what lies between the rows stays."""
    n_ctx, n_groups, k, nh, nkv, d = [40, 0], [30, 27], 4, 4, 2, 64
    q, kk, v, do = attn_inputs(13, n_ctx, n_groups, k, nh, nkv, d, dtype)
    at = dict(n_ctx=n_ctx, n_groups=n_groups, k_masks=k)

    def view(t):
        rows, w = t.shape[0], t.shape[1] * t.shape[2]
        buf = torch.full((rows * (w + pad) + odd + 8,), 77.0, dtype=dtype, device="cuda")
        return buf, buf[odd:odd + rows * (w + pad)].view(rows, w + pad)[:, :w].unflatten(1, t.shape[1:])

    tensors = {n: view(t) for n, t in dict(q=q, k=kk, v=v, do=do, out=q, dq=q, dk=kk, dv=v).items()}
    for n, t in (("q", q), ("k", kk), ("v", v), ("do", do)):
        tensors[n][1].copy_(t)
    V = {n: t[1] for n, t in tensors.items()}
    r = ps.group_attention(V["q"], V["k"], V["v"], out={"out": V["out"]}, **at)
    g = ps.group_attention_backward(V["do"], V["q"], V["k"], V["v"], V["out"], r["lse"], grads={n: V[n] for n in ("dq", "dk", "dv")}, **at)
    val, bnd = ref.attention(q, kk, v, do, n_ctx, n_groups, k, d ** -0.5)
    ref.check(r | g, val, bnd, ("out", "lse", "dq", "dk", "dv"))
    for n in ("out", "dq", "dk", "dv"):
        buf, t = tensors[n]
        t.fill_(77.0)
        assert (buf == 77.0).all(), n


@TYPES
@pytest.mark.parametrize("scale", [0.0, -0.3, 1e-6, 3.0])
def test_attention_scales(ps, scale, dtype):
    n_ctx, n_groups, k = [100], [40], 2
    q, kk, v, do = attn_inputs(17, n_ctx, n_groups, k, 2, 2, 64, dtype, spread=2.0 if scale < 1 else 1.0)
    got = attn_both(ps, q, kk, v, do, scale=scale, n_ctx=n_ctx, n_groups=n_groups, k_masks=k)
    val, bnd = ref.attention(q, kk, v, do, n_ctx, n_groups, k, scale)
    ref.check(got, val, bnd, ("out", "lse", "dq", "dk", "dv"))


@TYPES
def test_attention_scores_that_grow_along_the_keys(ps, dtype):
    """Every tile's maximum is far above the one before: the running sums are taken to a new reference each time."""
    n_ctx, n_groups, k = [700], [30], 4
    q, kk, v, do = attn_inputs(19, n_ctx, n_groups, k, 2, 1, 64, dtype)
    q = q.abs()
    kk *= torch.linspace(0.05, 1.0, kk.shape[0], device="cuda").to(dtype)[:, None, None]
    kk += (torch.linspace(0.0, 6.0, kk.shape[0], device="cuda")[:, None, None]).to(dtype)
    got = attn_both(ps, q, kk, v, do, n_ctx=n_ctx, n_groups=n_groups, k_masks=k)
    val, bnd = ref.attention(q, kk, v, do, n_ctx, n_groups, k, 0.125)
    ref.check(got, val, bnd, ("out", "lse", "dq", "dk", "dv"))


@TYPES
@pytest.mark.parametrize("pad, odd", [(8, 0), (5, 3)], ids=["aligned", "odd"])
def test_loss_and_embedding_on_views(ps, pad, odd, dtype):
    rows, H, V = 200, 72, 333
    x, w, labels, up = loss_inputs(23, rows, H, V, 0.2, dtype)
    buf = torch.full((2, rows * (H + pad) + odd + 8), 55.0, dtype=dtype, device="cuda")
    vx, vdx = (b[odd:odd + rows * (H + pad)].view(rows, H + pad)[:, :H] for b in buf)
    vx.copy_(x)
    got = ps.lm_loss(vx, w, labels)
    got |= ps.lm_loss_backward(vx, w, labels, got["lse"], up, grads={"dx": vdx})
    val, bnd = ref.loss(x, w, labels, up)
    ref.check(got, val, bnd, ("loss", "lse", "dx", "dw"))
    one = ps.lm_loss_backward(vx, w, labels, got["lse"], up, want_dw=False)
    assert set(one) == {"dx"} and torch.equal(one["dx"], vdx)
    one = ps.lm_loss_backward(vx, w, labels, got["lse"], up, want_dx=False)
    assert set(one) == {"dw"} and torch.equal(one["dw"], got["dw"])
    vx.fill_(55.0), vdx.fill_(55.0)
    assert (buf == 55.0).all()
    ids = torch.randint(-1, V + 2, (rows,), dtype=torch.int32).cuda()
    table, masks, dout = normal(1, (V, H), 1.0, dtype), normal(2, (2, H), 1.0, dtype), normal(3, (rows, H), 1.0, dtype)
    val, bnd = ref.embed(ids, table, masks, 1.0, dout)
    ps.embed_rows(ids, table, masks, out=vx)
    vdx.copy_(dout)
    ref.check({"out": vx} | ps.embed_rows_backward(ids, vdx, V, 2), val, bnd, ("out", "d_table", "d_mask"))
    vx.fill_(55.0), vdx.fill_(55.0)
    assert (buf == 55.0).all()


@TYPES
def test_offsets_beyond_32_bits(ps, dtype):
    """Rows so far apart that the last ones lie more than 2^32 bytes and 2^31 elements behind the first."""
    n_ctx, n_groups, k, nh, d = [300], [10], 4, 1, 64
    q, kk, v, do = attn_inputs(29, n_ctx, n_groups, k, nh, nh, d, dtype)
    rows, ld = kk.shape[0], 2 ** 31 // 340
    ld -= ld % 8
    big = torch.empty(rows * ld, dtype=dtype, device="cuda").view(rows, ld)
    vk, vv = big[:, :d].unflatten(1, (1, d)), big[:, 64:128].unflatten(1, (1, d))
    vdk, vdv = big[:, 128:192].unflatten(1, (1, d)), big[:, 256:320].unflatten(1, (1, d))
    vk.copy_(kk), vv.copy_(v)
    assert (rows - 1) * ld > 2 ** 31
    at = dict(n_ctx=n_ctx, n_groups=n_groups, k_masks=k)
    r = ps.group_attention(q, vk, vv, **at)
    r |= ps.group_attention_backward(do, q, vk, vv, r["out"], r["lse"], grads={"dk": vdk, "dv": vdv}, **at)
    val, bnd = ref.attention(q, kk, v, do, n_ctx, n_groups, k, d ** -0.5)
    ref.check(r, val, bnd, ("out", "lse", "dq", "dk", "dv"))
    x, w, labels, up = loss_inputs(31, rows, 64, 100, 0.1, dtype)
    big[:, :64].copy_(x)
    got = ps.lm_loss(big[:, :64], w, labels)
    got |= ps.lm_loss_backward(big[:, :64], w, labels, got["lse"], up, grads={"dx": big[:, 64:128]})
    val, bnd = ref.loss(x, w, labels, up)
    ref.check(got, val, bnd, ("loss", "lse", "dx", "dw"))


# ---- streams, graphs, repeated calls --------------------------------------------------------------------------------

def step(ps, dtype, seed):
    """Inputs of all operators and a function that runs them."""
    n_ctx, n_groups, k = [50, 9], [33, 70], 4
    q, kk, v, do = attn_inputs(seed, n_ctx, n_groups, k, 2, 1, 64, dtype)
    x, w, labels, up = loss_inputs(seed, 150, 64, 700, 0.2, dtype)
    g = torch.Generator().manual_seed(seed)
    ids = torch.randint(0, 54, (500,), generator=g, dtype=torch.int32).cuda()
    table, masks, dout = normal(seed, (50, 64), 1.0, dtype), normal(seed + 1, (4, 64), 1.0, dtype), normal(seed + 2, (500, 64), 1.0, dtype)
    tensors = [q, kk, v, do, x, w, up, table, masks, dout]

    def run(stream=None):
        at = dict(n_ctx=n_ctx, n_groups=n_groups, k_masks=k, stream=stream)
        r = ps.group_attention(q, kk, v, **at)
        r |= ps.group_attention_backward(do, q, kk, v, r["out"], r["lse"], **at)
        s = ps.lm_loss(x, w, labels, stream=stream)
        s |= ps.lm_loss_backward(x, w, labels, s["lse"], up, stream=stream)
        e = {"rows": ps.embed_rows(ids, table, masks, stream=stream)}
        e |= ps.embed_rows_backward(ids, dout, 50, 4, stream=stream)
        return list(r.values()) + list(s.values()) + list(e.values())

    return run, tensors


@TYPES
def test_the_same_call_gives_the_same_bits(ps, dtype):
    run, _ = step(ps, dtype, 41)
    first = run()
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(first, run()))


@TYPES
def test_two_streams_at_once(ps, dtype):
    runs = [step(ps, dtype, s)[0] for s in (43, 44)]
    want = [r() for r in runs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in runs]
    got = [[], []]
    for _ in range(4):
        for i, (r, s) in enumerate(zip(runs, streams)):
            got[i].append(r(stream=s))
    torch.cuda.synchronize()
    for i in range(2):
        for g in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(want[i], g))


@TYPES
def test_captured_and_replayed_with_other_inputs(ps, dtype):
    runs = [step(ps, dtype, s) for s in (45, 46)]
    graphs, outs = [], []
    for run, _ in runs:
        run()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(run())
        graphs.append(g)
    other = step(ps, dtype, 47)
    for run, tensors in runs:
        for t, o in zip(tensors, other[1]):
            t.copy_(o)
    for g in graphs:
        g.replay()
    torch.cuda.synchronize()
    for (run, _), out in zip(runs, outs):
        assert all(torch.equal(a, b) for a, b in zip(run(), out))


@TYPES
def test_calls_find_what_the_stream_wrote_just_before(ps, dtype):
    """Inputs that kernels ahead in the stream still write (the operators' kernels start early and wait)."""
    run, tensors = step(ps, dtype, 48)
    want = run()
    keep = [t.clone() for t in tensors]
    torch.cuda.synchronize()
    for _ in range(3):
        for t in tensors:
            t.fill_(9.0)
        torch.cuda._sleep(200000)
        for t, o in zip(tensors, keep):
            t.copy_(o)
        assert all(torch.equal(a, b) for a, b in zip(want, run()))
        for t in tensors:
            t.fill_(5.0)         # (and none that come behind are read)
        for t, o in zip(tensors, keep):
            t.copy_(o)


@TYPES
def test_degenerate_sizes(ps, dtype):
    # no groups at all: no rows, and the context's gradients are zero
    q, kk, v, do = attn_inputs(51, [130, 3], [0, 0], 4, 2, 1, 64, dtype)
    got = attn_both(ps, q, kk, v, do, n_ctx=[130, 3], n_groups=[0, 0], k_masks=4)
    assert got["out"].numel() == 0 and (got["dk"] == 0).all() and (got["dv"] == 0).all()
    x, w, labels, up = loss_inputs(52, 5, 64, 100, 0.0, dtype)
    got = ps.lm_loss(x[:0], w, labels[:0])
    got |= ps.lm_loss_backward(x[:0], w, labels[:0], got["lse"], up[:0])
    assert got["loss"].numel() == 0 and (got["dw"] == 0).all()
    none = torch.full((5,), -100, dtype=torch.int32, device="cuda")
    got = ps.lm_loss(x, w, none)
    got |= ps.lm_loss_backward(x, w, none, got["lse"], up)
    assert all((got[n] == 0).all() for n in ("loss", "lse", "dx", "dw"))
    ids = torch.zeros(0, dtype=torch.int32, device="cuda")
    assert ps.embed_rows(ids, w).shape == (0, 64)
    got = ps.embed_rows_backward(ids, x[:0], 100, 3)
    assert (got["d_table"] == 0).all() and (got["d_mask"] == 0).all()


def test_wrong_types_and_shapes_are_refused(ps):
    q, kk, v, do = attn_inputs(53, [4], [3], 1, 2, 1, 64, BF16)
    at = dict(n_ctx=[4], n_groups=[3], k_masks=1)
    for call in (lambda: ps.group_attention(q.float(), kk, v, **at), lambda: ps.group_attention(q.half(), kk.half(), v.half(), **at),
                 lambda: ps.group_attention(q, kk, v, n_ctx=[5], n_groups=[3], k_masks=1),
                 lambda: ps.group_attention(q, kk[:, :, :32], v[:, :, :32], **at),
                 lambda: ps.group_attention(q.transpose(0, 1), kk, v, **at),
                 lambda: ps.lm_loss(q[:, 0], torch.zeros(9, 32, dtype=BF16, device="cuda"), torch.zeros(6, dtype=torch.int32, device="cuda")),
                 lambda: ps.lm_loss(q[:, 0], torch.zeros(9, 64, dtype=BF16, device="cuda"), torch.zeros(6, dtype=torch.int64, device="cuda")),
                 lambda: ps.embed_rows(torch.zeros(3, dtype=torch.int64, device="cuda"), q[:, 0].contiguous()),
                 lambda: ps.embed_rows_backward(torch.zeros(5, dtype=torch.int32, device="cuda"), q[:, 0], 10)):
        with pytest.raises(ps.PsError):
            call()

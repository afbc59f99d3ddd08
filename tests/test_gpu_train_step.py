"""The training operators together: one step of a drafter (embedding -> fc -> norm -> attention of the groups -> FFN -> head),
its losses against the framework's own forward pass of the training layout, its gradients against a plain 64-bit
form and against differences of it."""
import pytest
import torch

import synth
import train_reference as ref

pytestmark = pytest.mark.gpu


def norm(x, g, eps):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + eps) * g


def rope(x, pos, base):
    """Pairs (i, i + d/2) rotated by pos * base^(-2i/d)."""
    d = x.shape[-1]
    ang = pos.double()[:, None] * base ** (-torch.arange(0, d, 2, device=x.device, dtype=torch.float64) / d)[None, :]
    c, s = torch.cos(ang).to(x.dtype)[:, None], torch.sin(ang).to(x.dtype)[:, None]
    a, b = x[..., :d // 2], x[..., d // 2:]
    return torch.cat([a * c - b * s, b * c + a * s], -1)


class Embed(torch.autograd.Function):
    @staticmethod
    def forward(ctx, ps, ids, table, masks):
        ctx.ps, ctx.ids, ctx.V, ctx.k = ps, ids, table.shape[0], masks.shape[0]
        return ps.embed_rows(ids, table, masks)

    @staticmethod
    def backward(ctx, d):
        g = ctx.ps.embed_rows_backward(ctx.ids, d.contiguous(), ctx.V, ctx.k)
        return None, None, g["d_table"], g["d_mask"]


class Attn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, ps, q, k, v, at):
        r = ps.group_attention(q, k, v, **at)
        ctx.ps, ctx.at = ps, at
        ctx.save_for_backward(q, k, v, r["out"], r["lse"])
        return r["out"]

    @staticmethod
    def backward(ctx, d):
        q, k, v, out, lse = ctx.saved_tensors
        g = ctx.ps.group_attention_backward(d.contiguous(), q, k, v, out, lse, **ctx.at)
        return None, g["dq"], g["dk"], g["dv"], None


class Loss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, ps, x, w, labels):
        r = ps.lm_loss(x, w, labels)
        ctx.ps = ps
        ctx.save_for_backward(x, w, labels, r["lse"])
        return r["loss"]

    @staticmethod
    def backward(ctx, d):
        x, w, labels, lse = ctx.saved_tensors
        g = ctx.ps.lm_loss_backward(x, w, labels, lse, d.float().contiguous())
        return None, g["dx"], g["dw"], None


def plain_attn(q, k, v, at):
    c, g, R = at["n_ctx"][0], at["n_groups"][0], at["k_masks"] + 1
    sees = ref.group_mask(c, g, R).to(q.device)
    per = q.shape[1] // k.shape[1]
    s = torch.einsum("rhd,chd->hrc", q, k.repeat_interleave(per, 1)) * q.shape[2] ** -0.5
    p = torch.softmax(s.masked_fill(~sees, -torch.inf), -1)
    return torch.einsum("hrc,chd->rhd", p, v.repeat_interleave(per, 1))


def losses(s, W, ids, feats, real, labels, at, embed, attn, head):
    """Losses of the group rows of one sequence.  ids, feats: of the context and the group rows; real: position of each row."""
    n = at["n_ctx"][0]
    x = torch.cat([embed(ids, W["embed"], W["mask_embed"]), feats], -1) @ W["w_fc"].T
    y = norm(x, W["g_in"], s.rms_eps)
    q = rope((y[n:] @ W["w_q"].T).unflatten(-1, (s.n_heads, s.head_dim)), real[n:], s.rope_base)
    k = rope((y @ W["w_k"].T).unflatten(-1, (s.n_kv_heads, s.head_dim)), real, s.rope_base)
    v = (y @ W["w_v"].T).unflatten(-1, (s.n_kv_heads, s.head_dim))
    a = x[n:] + attn(q, k, v, at).flatten(1) @ W["w_o"].T
    z = norm(a, W["g_post"], s.rms_eps)
    f = a + (torch.nn.functional.silu(z @ W["w_gate"].T) * (z @ W["w_up"].T)) @ W["w_down"].T
    return head(norm(f, W["g_final"], s.rms_eps), W["w_lm"], labels)


def setup(name, n, groups):
    import paper_2410_05589_b200 as ps
    s = synth.CONFIGS[name].with_(batch=1)
    W = synth.weights(s)
    R = s.k_masks + 1
    drafter = ps.drafter_from_shape(s, W, max_batch=1, max_ctx=n + groups + R)
    hid, tok = synth.hidden_states(s, "seq", n + groups), synth.token_ids(s, "seq", n + groups)
    T = {k: ps.to_device(v) for k, v in W.items() if v is not None}
    hid, tok = ps.to_device(hid), ps.to_device(tok)
    drafter.kv_append([0], [n], hid[:n].contiguous(), tok[:n].contiguous())
    ids = torch.empty(n + groups * R, dtype=torch.int32, device="cuda")
    ids[:n] = tok[:n]
    rows = ids[n:].view(groups, R)
    rows[:, 0] = tok[n:]
    rows[:, 1:] = s.vocab + torch.arange(R - 1, device="cuda", dtype=torch.int32)
    feats = torch.empty((n + groups * R, s.hidden), dtype=hid.dtype, device="cuda")
    feats[:n] = hid[:n]
    f = feats[n:].view(groups, R, s.hidden)
    f[:, 0], f[:, 1:] = hid[n:], T["mask_feat"][None]
    t = torch.arange(groups, device="cuda")[:, None] + torch.arange(R, device="cuda")[None, :]
    real = torch.cat([torch.arange(n, device="cuda"), (n + t).reshape(-1)])
    # row j of group t predicts the token j places after the next one
    at = t + 1
    labels = torch.where(at < groups, tok[n:][at.clamp(max=groups - 1)], -100).int().reshape(-1)
    return ps, s, drafter, T, hid[n:].contiguous(), tok[n:].contiguous(), ids, feats, real, labels


def test_step_of_the_toy_drafter():
    n, groups = 24, 37
    ps, s, drafter, T, hid, tok, ids, feats, real, labels = setup("tiny", n, groups)
    at = dict(n_ctx=[n], n_groups=[groups], k_masks=s.k_masks)
    names = ("embed", "mask_embed", "w_fc", "g_in", "w_q", "w_k", "w_v", "w_o", "g_post", "w_gate", "w_up", "w_down", "g_final", "w_lm")

    def ours(W):
        return losses(s, W, ids, feats.float(), real, labels, at, lambda i, t, m: Embed.apply(ps, i, t, m),
                      lambda q, k, v, a: Attn.apply(ps, q, k, v, a), lambda x, w, l: Loss.apply(ps, x, w, l))

    def plain(W):
        def head(x, w, lab):
            logp = torch.log_softmax(x @ w.T, -1)
            return torch.where(lab >= 0, -logp.gather(1, lab.clamp_min(0).long()[:, None])[:, 0], 0.0)
        return losses(s, W, ids, feats.double(), real, labels, at, lambda i, t, m: torch.cat([t, m])[i.long()], plain_attn, head)

    W1 = {k: T[k].clone().requires_grad_() for k in names}
    W2 = {k: T[k].double().requires_grad_() for k in names}
    l1, l2 = ours(W1), plain(W2)
    # the framework's forward pass of the same layout (its logits are within 1e-4 of a row's size of the definition's)
    logits = drafter.group_forward(0, hid, tok)["logits"].flatten(0, 1).double()
    l3 = torch.where(labels >= 0, -torch.log_softmax(logits, -1).gather(1, labels.clamp_min(0).long()[:, None])[:, 0], 0.0)
    size = logits.abs().amax()
    assert (l1 - l3).abs().max() <= 2e-4 * size + 1e-5
    assert (l1 - l2).abs().max() <= 1e-4
    m = (labels >= 0).sum()
    (l1.sum() / m).backward()
    (l2.sum() / m).backward()
    for k in names:
        # (fp32 sums of a few thousand terms behind fp32 products of the torch part: 1e-5 of the tensor's own size)
        off, scale = (W1[k].grad.double() - W2[k].grad).norm(), W2[k].grad.norm()
        assert off <= 3e-5 * scale, (k, (off / scale).item())
    # the gradient against differences of the 64-bit form along random directions
    g = torch.Generator(device="cuda").manual_seed(7)
    for k in ("mask_embed", "w_q", "w_k", "w_v", "w_lm"):
        d = torch.randn(T[k].shape, generator=g, device="cuda", dtype=torch.float64)
        d /= d.norm()
        h = 1e-4
        with torch.no_grad():
            up, down = (plain({**W2, k: W2[k] + e * d}).sum() / m for e in (h, -h))
        slope, want = (up - down) / (2 * h), (W1[k].grad.double() * d).sum()
        assert (slope - want).abs() <= 1e-4 * W2[k].grad.norm() + 1e-7, (k, slope.item(), want.item())


def test_step_in_bf16_runs_and_gives_finite_gradients():
    n, groups = 40, 50
    ps, s, drafter, T, hid, tok, ids, feats, real, labels = setup("mini", n, groups)
    at = dict(n_ctx=[n], n_groups=[groups], k_masks=s.k_masks)
    W = {k: v.clone().requires_grad_() for k, v in T.items() if k not in ("mask_feat", "b_fc")}
    l = losses(s, W, ids, feats, real, labels, at, lambda i, t, m: Embed.apply(ps, i, t, m),
               lambda q, k, v, a: Attn.apply(ps, q.contiguous(), k.contiguous(), v.contiguous(), a), lambda x, w, lab: Loss.apply(ps, x, w, lab))
    logits = drafter.group_forward(0, hid, tok)["logits"].flatten(0, 1).double()
    want = torch.where(labels >= 0, -torch.log_softmax(logits, -1).gather(1, labels.clamp_min(0).long()[:, None])[:, 0], 0.0)
    # the torch part rounds every activation to bf16, the framework's forward pass none: a few of its half steps
    assert (l - want).abs().max() <= 16 * 2.0 ** -8 * logits.abs().amax()
    (l.sum() / (labels >= 0).sum()).backward()
    for k, w in W.items():
        assert torch.isfinite(w.grad).all() and w.grad.abs().max() > 0, k

"""The operators that a program training a ParallelSpec drafter calls, at the sizes it calls them.

Group-wise parallel training (Sec. 4.1, Fig. 3) lays a sequence out as groups of k + 1 rows, a real
position and its k [MASK] positions, behind a context of real positions that only lend their keys and
values (a prompt).  The parts of such a step that know about this layout or about the vocabulary are
the ones below; the dense products between them are ordinary matrix products.

  embed   the rows' input embeddings, scaled: a token's row of the table, or a learned [MASK] row;
          backward: the sum of the rows' gradients per token and per [MASK]
  attn    attention under the groups' mask: row j of group t sees the context, the real rows of the
          groups 0..t and the [MASK] rows 1..j of its own group; backward: dq, dk, dv
  loss    softmax cross entropy of the LM head (rows with a negative label count for nothing);
          backward: the gradients of the rows and of the head

A case is a dict of plain values:

  op            "attn" | "loss" | "embed"
  model         a key of MODELS
  train         false: forward; true: forward, then backward
  attn          batch, k, ctx_lo/hi and groups_lo/hi (sizes per sequence, ragged over the batch)
  loss          rows, ignored (share of rows with label -100), dw (the head's gradient too)
  embed         groups, k, padded (rows at the end without a token), table (the table's gradient too)
"""
from __future__ import annotations

import math

import torch

own = False

# dtype, hidden, heads, kv heads, head dim, vocab: the shapes that the repository's configurations name
MODELS = {
    "tiny": ("f32", 256, 4, 4, 64, 1000),
    "mini32": ("f32", 320, 5, 5, 64, 1500),
    "mini": ("bf16", 768, 6, 6, 128, 5000),
    "7b": ("bf16", 4096, 32, 32, 128, 32000),
    "13b": ("bf16", 5120, 40, 40, 128, 32000),
    "33b": ("bf16", 6656, 52, 52, 128, 32000),
    "llama3_8b": ("bf16", 4096, 32, 8, 128, 128256),
}
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}


def _attn(name, model, train, batch, k, ctx_lo, ctx_hi, groups_lo, groups_hi):
    return {"name": name, "op": "attn", "model": model, "train": train, "batch": batch, "k": k, "ctx_lo": ctx_lo,
            "ctx_hi": ctx_hi, "groups_lo": groups_lo, "groups_hi": groups_hi}


def _loss(name, model, train, rows, ignored, dw):
    return {"name": name, "op": "loss", "model": model, "train": train, "rows": rows, "ignored": ignored, "dw": dw}


def _embed(name, model, train, groups, k, padded, table):
    return {"name": name, "op": "embed", "model": model, "train": train, "groups": groups, "k": k, "padded": padded,
            "table": table}


def listed():
    return [
        # the toy drafter in fp32 that one debugs a training loop with: launches and latency only
        _attn("attn_tiny_f32_train", "tiny", True, 1, 4, 64, 64, 40, 40),
        # scoring one group behind a cached prompt: few rows over a long axis
        _attn("attn_7b_one_group_fwd", "7b", False, 1, 4, 2011, 2011, 1, 1),
        # a ragged batch of chats: prompts and answers of a few hundred positions
        _attn("attn_13b_ragged_train", "13b", True, 4, 4, 60, 300, 150, 420),
        # grouped queries, one long answer without a prompt
        _attn("attn_8b_long_train", "llama3_8b", True, 1, 4, 0, 0, 2047, 2047),
        # the widest drafter with eight masks, evaluation
        _attn("attn_33b_k8_fwd", "33b", False, 2, 8, 500, 900, 301, 640),
        # the toy drafter's loss, with the gradient of its head
        _loss("loss_tiny_f32_train", "tiny", True, 205, 0.1, True),
        # evaluation on a held-out answer
        _loss("loss_7b_fwd", "7b", False, 333, 0.0, False),
        # training against the target's frozen head, prompts and tails masked
        _loss("loss_13b_frozen_train", "13b", True, 2560, 0.12, False),
        # a head of its own over a large vocabulary
        _loss("loss_8b_head_train", "llama3_8b", True, 4095, 0.05, True),
        # the [MASK] rows alone are learned: a few sums over all groups
        _embed("embed_13b_masks_train", "13b", True, 512, 4, 13, False),
        # the input rows of a long batch
        _embed("embed_7b_fwd", "7b", False, 2047, 4, 0, False),
        # a table of its own over a large vocabulary
        _embed("embed_8b_table_train", "llama3_8b", True, 2048, 4, 100, True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn", "attn", "loss", "loss", "embed"])
    model = rng.choice(list(MODELS))
    small = MODELS[model][0] == "f32"
    if op == "attn":
        batch, k = rng.choice([1, 1, 2, 3, 5, 8]), rng.choice([0, 1, 2, 4, 4, 7, 8, 15])
        most = max(2, min(1500 // batch, 10000 // (batch * (k + 1)), 400 if small else 1500))
        glo = _log_int(rng, 1, most)
        ghi = min(most, glo + rng.randrange(0, 1 + glo))
        chi = rng.choice([0, _log_int(rng, 1, 3000 // batch)])
        return {k_: v for k_, v in _attn("", model, rng.random() < 0.6, batch, k, rng.randrange(0, chi + 1), chi, glo,
                                         ghi).items() if k_ != "name"}
    if op == "loss":
        train = rng.random() < 0.6
        c = _loss("", model, train, _log_int(rng, 1, 1000 if small else 4000), rng.choice([0.0, 0.05, 0.3, 0.6]),
                  train and rng.random() < 0.4)
    else:
        train = rng.random() < 0.6
        c = _embed("", model, train, _log_int(rng, 1, 2000), rng.choice([0, 1, 2, 4, 4, 7]), rng.choice([0, 0, 1, 7, 64]),
                   train and rng.random() < 0.5)
    return {k_: v for k_, v in c.items() if k_ != "name"}


# ---- sizes ---------------------------------------------------------------------------------------

def _ragged(lo, hi, n):
    """n sizes between lo and hi, spread by the golden ratio."""
    return [lo + int((hi - lo) * ((i * 0.6180339887498949 + 0.999) % 1.0) + 0.5) for i in range(n)]


def _sizes(case):
    return (_ragged(case["ctx_lo"], case["ctx_hi"], case["batch"]),
            _ragged(case["groups_lo"], case["groups_hi"], case["batch"]))


def _ignored_rows(case):
    return min(case["rows"] - 1, int(round(case["rows"] * case["ignored"])))


def work(case):
    name, H, nh, nkv, d, V = MODELS[case["model"]]
    e = BYTES[name]
    if case["op"] == "attn":
        ctx, groups = _sizes(case)
        k = case["k"]
        rows_q, rows_kv = sum(g * (k + 1) for g in groups), sum(c + g * (k + 1) for c, g in zip(ctx, groups))
        # keys that the rows of a sequence see: context and real rows, then their own group's masks
        pairs = sum((k + 1) * (g * c + g * (g + 1) // 2) + g * k * (k + 1) // 2 for c, g in zip(ctx, groups))
        q, kv = rows_q * nh * d * e, rows_kv * nkv * d * e
        by, fl = 2 * q + 2 * kv + rows_q * nh * 4, 4 * d * nh * pairs
        if case["train"]:
            by, fl = by + 2 * q + 2 * kv, fl + 10 * d * nh * pairs
        return {"bytes": by, "flops": fl}
    if case["op"] == "loss":
        n = case["rows"] - _ignored_rows(case)
        by, fl = n * H * e + V * H * e + case["rows"] * 12, 2 * n * V * H
        if case["train"]:
            by, fl = by + case["rows"] * (H * e + 4), fl + 2 * n * V * H
        if case["dw"]:
            by, fl = by + V * H * e, fl + 2 * n * V * H
        return {"bytes": by, "flops": fl}
    rows = case["groups"] * (case["k"] + 1)
    used = min(V, case["groups"]) + case["k"]
    by, fl = (used + rows) * H * e + rows * 4, rows * H
    if case["train"]:
        by, fl = by + (rows + case["k"] + (V if case["table"] else 0)) * H * e, fl + rows * H
    return {"bytes": by, "flops": fl}


# ---- inputs --------------------------------------------------------------------------------------

def _normal(gen, shape, sigma, dtype):
    return (torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * sigma).to(dtype)


def _zipf_tokens(gen, n, V):
    """Token ids whose frequency falls with their rank, the ranks scattered over the ids."""
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    rank = (torch.exp(u * math.log(V + 1.0)) - 1.0).long().clamp_(0, V - 1)
    return ((rank * 7919 + 13) % V).int()


def prepare(case, seed):
    name, H, nh, nkv, d, V = MODELS[case["model"]]
    dt = DTYPES[name]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    st = {"case": case}
    if case["op"] == "attn":
        ctx, groups = _sizes(case)
        R = case["k"] + 1
        rq, rkv = sum(groups) * R, sum(ctx) + sum(groups) * R
        # (queries and keys as they are after the rotation; keys and values side by side, as one product leaves them)
        kv = _normal(gen, (rkv, 2, nkv, d), 1.0, dt)
        st |= {"ctx": ctx, "groups": groups, "q": _normal(gen, (rq, nh, d), 1.0, dt), "k": kv[:, 0], "v": kv[:, 1]}
        if case["train"]:
            st["dout"] = _normal(gen, (rq, nh, d), 0.05, dt)
        # the layout of the plain form: which rows are real keys, and what each row sees of them
        real, mask, kseq, kpos, qseq, qpos, base, n = [], [], [], [], [], [], 0, 0
        for b, (c, g) in enumerate(zip(ctx, groups)):
            first = base + c + torch.arange(g) * R
            real += [torch.arange(base, base + c), first]
            mask += [(first[:, None] + torch.arange(1, R)[None, :]).reshape(-1)]
            kseq += [torch.full((c + g,), b)]
            kpos += [torch.arange(c + g)]
            qseq += [torch.full((g * R,), b)]
            qpos += [c + torch.arange(g).repeat_interleave(R)]
            base += c + g * R
        for key, v in (("real", real), ("mask", mask), ("kseq", kseq), ("kpos", kpos), ("qseq", qseq), ("qpos", qpos)):
            st[key] = torch.cat(v).cuda()
        return st
    if case["op"] == "loss":
        n = case["rows"]
        x = torch.randn((n, H), generator=gen, device="cuda")
        st["x"] = (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-5)).to(dt)   # as the final norm leaves them
        st["w"] = _normal(gen, (V, H), 0.02, dt)
        labels = _zipf_tokens(gen, n, V)
        labels[torch.randperm(n, generator=gen, device="cuda")[:_ignored_rows(case)]] = -100
        st["labels"] = labels
        if case["train"]:
            # the mean over the rows that count, with weights per row
            st["dloss"] = (0.5 + torch.rand(n, generator=gen, device="cuda")) / max(1, n - _ignored_rows(case))
        return st
    R, g = case["k"] + 1, case["groups"]
    ids = torch.empty((g, R), dtype=torch.int32, device="cuda")
    ids[:, 0] = _zipf_tokens(gen, g, V)
    ids[:, 1:] = V + torch.arange(case["k"], device="cuda", dtype=torch.int32)
    ids = ids.reshape(-1)
    if case["padded"]:
        ids[max(1, ids.numel() - case["padded"]):] = -1
    st |= {"ids": ids, "table": _normal(gen, (V, H), 0.02, dt), "scale": math.sqrt(H),
           "mask_rows": _normal(gen, (case["k"], H), 0.02, dt) if case["k"] else None}
    if case["train"]:
        st["dout"] = _normal(gen, (ids.numel(), H), 0.01, dt)
    return st


# ---- one pass ------------------------------------------------------------------------------------

def _attn_plain(st):
    case = st["case"]
    k, R = case["k"], case["k"] + 1
    dt = st["q"].dtype
    rows, nh, d = st["q"].shape
    nkv = st["k"].shape[1]
    per, scale = nh // nkv, 1.0 / math.sqrt(d)
    q = st["q"].float().view(rows, nkv, per, d).permute(1, 2, 0, 3).reshape(nkv, per * rows, d)
    kr, vr = st["k"][st["real"]].float().transpose(0, 1), st["v"][st["real"]].float().transpose(0, 1)
    sees = (st["qseq"][:, None] == st["kseq"][None, :]) & (st["kpos"][None, :] <= st["qpos"][:, None])
    n = sees.shape[1]
    s = torch.matmul(q, kr.transpose(1, 2)).mul_(scale).view(nkv, per, rows, n)
    s.masked_fill_(~sees, -math.inf)
    top = s.amax(-1)
    if k:
        g = rows // R   # the groups' own masks: [kv head][query head][group][row][mask]
        km = st["k"][st["mask"]].float().view(g, k, nkv, d).permute(2, 0, 1, 3)
        vm = st["v"][st["mask"]].float().view(g, k, nkv, d).permute(2, 0, 1, 3)
        q5 = q.view(nkv, per, g, R, d)
        s2 = torch.matmul(q5, km.transpose(2, 3)[:, None]).mul_(scale)
        j = torch.arange(R, device=q.device)
        s2.masked_fill_(j[None, 1:] > j[:, None], -math.inf)
        top = torch.maximum(top, s2.amax(-1).view(nkv, per, rows))
    p = s.sub_(top[..., None]).exp_()
    total = p.sum(-1)
    if k:
        p2 = s2.sub_(top.view(nkv, per, g, R, 1)).exp_()
        total = total + p2.sum(-1).view(nkv, per, rows)
    lse = top + total.log()
    p.div_(total[..., None])
    pm = p.view(nkv, per * rows, n)
    o = torch.matmul(pm, vr).view(nkv, per, rows, d)
    if k:
        p2.div_(total.view(nkv, per, g, R, 1))
        o = o + torch.matmul(p2, vm[:, None]).view(nkv, per, rows, d)

    def rows_first(x):   # [kv head][query head][row][d] -> [row][head][d]
        return x.permute(2, 0, 1, 3).reshape(rows, nh, d).to(dt)

    res = {"out": rows_first(o), "lse": lse.reshape(nh, rows)}
    if not case["train"]:
        return res
    do = st["dout"].float().view(rows, nkv, per, d).permute(1, 2, 0, 3).reshape(nkv, per * rows, d)
    delta = (do.view(nkv, per, rows, d) * o).sum(-1)
    dk, dv = torch.zeros_like(st["k"], dtype=torch.float32), torch.zeros_like(st["k"], dtype=torch.float32)
    dv[st["real"]] = torch.matmul(pm.transpose(1, 2), do).transpose(0, 1)
    ds = torch.matmul(do, vr.transpose(1, 2)).view(nkv, per, rows, n)
    ds.sub_(delta[..., None]).mul_(p).mul_(scale)
    dsm = ds.view(nkv, per * rows, n)
    dk[st["real"]] = torch.matmul(dsm.transpose(1, 2), q).transpose(0, 1)
    dq = torch.matmul(dsm, kr).view(nkv, per, rows, d)
    if k:
        do5 = do.view(nkv, per, g, R, d)
        dv[st["mask"]] = torch.matmul(p2.transpose(3, 4), do5).sum(1).permute(1, 2, 0, 3).reshape(g * k, nkv, d)
        ds2 = torch.matmul(do5, vm.transpose(2, 3)[:, None]).sub_(delta.view(nkv, per, g, R, 1)).mul_(p2).mul_(scale)
        dk[st["mask"]] = torch.matmul(ds2.transpose(3, 4), q5).sum(1).permute(1, 2, 0, 3).reshape(g * k, nkv, d)
        dq = dq + torch.matmul(ds2, km[:, None]).view(nkv, per, rows, d)
    return res | {"dq": rows_first(dq), "dk": dk.to(dt), "dv": dv.to(dt)}


def _loss_plain(st):
    case = st["case"]
    x, w = st["x"].float(), st["w"].float()
    counts = st["labels"] >= 0
    at = torch.where(counts, st["labels"], 0).long()[:, None]
    logits = torch.matmul(x, w.t())
    top = logits.amax(-1, keepdim=True)
    picked = logits.gather(1, at)
    p = logits.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = top + total.log()
    zero = torch.zeros((), device=x.device)
    res = {"loss": torch.where(counts, (lse - picked)[:, 0], zero), "lse": torch.where(counts, lse[:, 0], zero)}
    if not case["train"]:
        return res
    up = torch.where(counts, st["dloss"], zero)[:, None]
    g = p.mul_(up / total)
    g.scatter_add_(1, at, -up)
    res["dx"] = torch.matmul(g, w).to(st["x"].dtype)
    if case["dw"]:
        res["dw"] = torch.matmul(g.t(), x).to(st["w"].dtype)
    return res


def _embed_plain(st):
    case = st["case"]
    V, H = st["table"].shape
    rows, ids = st["table"], st["ids"].long()
    if case["k"]:
        rows = torch.cat([rows, st["mask_rows"]])
    there = (ids >= 0)[:, None]
    out = torch.where(there, rows[ids.clamp_min(0)].float() * st["scale"], 0.0)
    res = {"out": out.to(rows.dtype)}
    if not case["train"]:
        return res
    d = torch.where(there, st["dout"].float() * st["scale"], 0.0)
    if case["table"]:
        grads = torch.zeros((V + case["k"], H), device=d.device).index_add_(0, ids.clamp_min(0), d)
        res["d_table"] = grads[:V].to(rows.dtype)
        grads = grads[V:]
    else:
        at = torch.where((ids >= V), ids - V, case["k"])
        grads = torch.zeros((case["k"] + 1, H), device=d.device).index_add_(0, at, d)[:case["k"]]
    if case["k"]:
        res["d_mask"] = grads.to(rows.dtype)
    return res


def run(st):
    case = st["case"]
    if not own:
        return {"attn": _attn_plain, "loss": _loss_plain, "embed": _embed_plain}[case["op"]](st)
    import paper_2410_05589_b200 as ps
    if case["op"] == "attn":
        at = dict(n_ctx=st["ctx"], n_groups=st["groups"], k_masks=case["k"])
        res = ps.group_attention(st["q"], st["k"], st["v"], **at)
        if case["train"]:
            res |= ps.group_attention_backward(st["dout"], st["q"], st["k"], st["v"], res["out"], res["lse"], **at)
        return res
    if case["op"] == "loss":
        res = ps.lm_loss(st["x"], st["w"], st["labels"])
        if case["train"]:
            res |= ps.lm_loss_backward(st["x"], st["w"], st["labels"], res["lse"], st["dloss"], want_dw=case["dw"])
        return res
    res = {"out": ps.embed_rows(st["ids"], st["table"], st["mask_rows"], scale=st["scale"])}
    if case["train"]:
        res |= ps.embed_rows_backward(st["ids"], st["dout"], vocab=st["table"].shape[0], k_masks=case["k"],
                                      scale=st["scale"], want_table=case["table"])
    return res


# ---- the definitions in 64 bits --------------------------------------------------------------------

def _attn_exact(case, st):
    """Sequence by sequence and head by head, over all its rows as keys and a mask from the definition."""
    R = case["k"] + 1
    q, k, v = st["q"].double(), st["k"].double(), st["v"].double()
    rows, nh, d = q.shape
    per = nh // k.shape[1]
    out, lse = torch.zeros_like(q), torch.zeros((nh, rows), dtype=torch.float64, device=q.device)
    train = case["train"]
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    q0 = k0 = 0
    for c, g in zip(st["ctx"], st["groups"]):
        i = torch.arange(c + g * R, device=q.device)
        group = torch.where(i < c, -1, torch.div(i - c, R, rounding_mode="floor"))
        j = torch.where(i < c, 0, (i - c) % R)
        gq, jq = group[c:, None], j[c:, None]
        sees = ((j == 0) & (group <= gq)) | ((group == gq) & (j <= jq))
        qs, ks = slice(q0, q0 + g * R), slice(k0, k0 + c + g * R)
        q0, k0 = qs.stop, ks.stop
        for h in range(nh):
            s = (q[qs, h] @ k[ks, h // per].T) / math.sqrt(d)
            s = s.masked_fill(~sees, -math.inf)
            lse[h, qs] = torch.logsumexp(s, -1)
            p = torch.exp(s - lse[h, qs][:, None])
            out[qs, h] = p @ v[ks, h // per]
            if train:
                do = st["dout"][qs, h].double()
                dv[ks, h // per] += p.T @ do
                dp = do @ v[ks, h // per].T
                ds = p * (dp - (p * dp).sum(-1, keepdim=True)) / math.sqrt(d)
                dq[qs, h] = ds @ k[ks, h // per]
                dk[ks, h // per] += ds.T @ q[qs, h]
    res = {"out": out, "lse": lse}
    return res | {"dq": dq, "dk": dk, "dv": dv} if train else res


def _loss_exact(case, st):
    keep = torch.nonzero(st["labels"] >= 0)[:, 0]
    n = case["rows"]
    w, x, label = st["w"].double(), st["x"][keep].double(), st["labels"][keep].long()
    loss, lse = (torch.zeros(n, dtype=torch.float64, device=x.device) for _ in range(2))
    logits = x @ w.T
    lse[keep] = torch.logsumexp(logits, -1)
    loss[keep] = lse[keep] - logits[torch.arange(len(keep), device=x.device), label]
    res = {"loss": loss, "lse": lse}
    if case["train"]:
        g = torch.softmax(logits, -1)
        g[torch.arange(len(keep), device=x.device), label] -= 1.0
        g *= st["dloss"][keep].double()[:, None]
        res["dx"] = torch.zeros((n, x.shape[1]), dtype=torch.float64, device=x.device)
        res["dx"][keep] = g @ w
        if case["dw"]:
            res["dw"] = g.T @ x
    return res


def _embed_exact(case, st):
    V, H = st["table"].shape
    ids = st["ids"].long()
    there = torch.nonzero(ids >= 0)[:, 0]
    table = st["table"].double()
    if case["k"]:
        table = torch.cat([table, st["mask_rows"].double()])
    out = torch.zeros((len(ids), H), dtype=torch.float64, device=ids.device)
    out[there] = st["scale"] * table[ids[there]]
    res = {"out": out}
    if case["train"]:
        total = torch.zeros((V + case["k"], H), dtype=torch.float64, device=ids.device)
        total.index_add_(0, ids[there], st["dout"][there].double())
        total *= st["scale"]
        if case["table"]:
            res["d_table"] = total[:V]
        if case["k"]:
            res["d_mask"] = total[V:]
    return res


def exact(case, seed):
    st = prepare(case, seed)
    return {"attn": _attn_exact, "loss": _loss_exact, "embed": _embed_exact}[case["op"]](case, st)

"""Plain 64-bit forms of the training operators, each with a bound on what the kernels may be off.

Bounds (u: half a step of the storage type where a value is rounded to it, 2^-8 for bf16 and nothing for fp32, whose
roundings are those of the sums; w = 2^-23: one addition or product in fp32, truncated):
  a score is off by at most es = (d + 8) w scale |q|.|k| + 4 w (1 + |s|), so that a probability is off by the
  factor 1 + 2 es (itself and its sum), and by u where it is rounded for a product;
  a sum of n terms is off by n w of the sum of its terms' magnitudes.
"""
from __future__ import annotations

import math

import torch

W = 2.0 ** -23


def half_step(dtype):
    return torch.finfo(dtype).eps / 2 if dtype == torch.bfloat16 else 0.0


def group_mask(ctx, groups, R):
    """Which rows (context and group rows, in storage order) each group row of one sequence sees."""
    sees = torch.zeros((groups * R, ctx + groups * R), dtype=torch.bool)
    for t in range(groups):
        for j in range(R):
            r = t * R + j
            sees[r, :ctx] = True
            for x in range(t + 1):
                sees[r, ctx + x * R] = True
            for m in range(1, j + 1):
                sees[r, ctx + t * R + m] = True
    return sees


def attention(q, k, v, dout, n_ctx, n_groups, k_masks, scale):
    """(values, bounds) of out, lse, dq, dk, dv: dicts of float64 tensors on the CPU."""
    dt, R = q.dtype, k_masks + 1
    u = half_step(dt)
    q, k, v, do = (x.detach().double().cpu() for x in (q, k, v, dout))
    rows, nh, d = q.shape
    per = nh // k.shape[1]
    val = {"out": torch.zeros_like(q), "lse": torch.zeros((nh, rows), dtype=torch.float64), "dq": torch.zeros_like(q),
           "dk": torch.zeros_like(k), "dv": torch.zeros_like(v)}
    bnd = {n: torch.zeros_like(x) for n, x in val.items()}
    q0 = k0 = 0
    for c, g in zip(n_ctx, n_groups):
        sees = group_mask(c, g, R)
        qs, ks = slice(q0, q0 + g * R), slice(k0, k0 + c + g * R)
        q0, k0 = qs.stop, ks.stop
        n = c + g * R + 8
        if g == 0:
            continue
        for h in range(nh):
            hk = h // per
            Q, K, V, dO = q[qs, h], k[ks, hk], v[ks, hk], do[qs, h]
            # (what a row does not see is not there: it may hold anything)
            S = torch.where(sees, (Q @ K.nan_to_num(0, 0, 0).T) * scale, torch.zeros((), dtype=torch.float64))
            es = torch.where(sees, (d + 8) * W * abs(scale) * (Q.abs() @ K.nan_to_num(0, 0, 0).abs().T) + 4 * W * (1 + S.abs()), 0.0)
            S = torch.where(sees, S, -math.inf)
            lse = torch.logsumexp(S, -1)
            P = torch.exp(S - lse[:, None])
            top = es.amax(-1, keepdim=True)
            ep = 2 * top + n * W
            Vf, Kf = V.nan_to_num(0, 0, 0), K.nan_to_num(0, 0, 0)
            O = P @ Vf
            eO = (ep + u + n * W) * (P @ Vf.abs()) + u * O.abs()
            val["out"][qs, h], bnd["out"][qs, h] = O, eO
            val["lse"][h, qs], bnd["lse"][h, qs] = lse, top[:, 0] + (n + 4) * W + 4 * W * lse.abs()
            # backward: p from the stored lse
            dP = dO @ Vf.T
            D = (dO * O).sum(-1, keepdim=True)
            eD = (dO.abs() * (eO + d * W * O.abs())).sum(-1, keepdim=True)
            edP = d * W * (dO.abs() @ Vf.abs().T)
            if u:   # rows of up to 32 keys: delta from the probabilities, not from the rounded out
                few = (sees.sum(-1, keepdim=True) <= 32)
                eD = torch.where(few, (P * (edP + (2 * ep + (n + 4) * W) * dP.abs())).sum(-1, keepdim=True), eD)
            dS = P * (dP - D)
            ep2 = 2 * ep + 4 * W
            edS = P * (eD + edP + W * (dP.abs() + D.abs())) * (1 + ep2) + (ep2 + u) * dS.abs()
            m = rows + 8   # (terms of the key sums, over all query heads of the head)
            val["dv"][ks, hk] += P.T @ dO
            bnd["dv"][ks, hk] += (ep2 + u).T.max() * (P.T @ dO.abs()) + per * m * W * (P.T @ dO.abs())
            val["dq"][qs, h] = dS @ Kf * scale
            bnd["dq"][qs, h] = abs(scale) * (edS @ Kf.abs() + n * W * (dS.abs() @ Kf.abs())) + u * val["dq"][qs, h].abs()
            val["dk"][ks, hk] += dS.T @ Q * scale
            bnd["dk"][ks, hk] += abs(scale) * (edS.T @ Q.abs() + per * m * W * (dS.abs().T @ Q.abs()))
    for n in ("dk", "dv"):
        bnd[n] += u * val[n].abs()
    return val, bnd


def loss(x, w, labels, dloss):
    """(values, bounds) of loss, lse, dx, dw."""
    u = half_step(x.dtype)
    n, H = x.shape
    V = w.shape[0]
    x, w, up, labels = x.detach().double().cpu(), w.detach().double().cpu(), dloss.double().cpu(), labels.long().cpu()
    keep = torch.nonzero((labels >= 0) & (labels < V))[:, 0]
    X, lab, up = x[keep], labels[keep], up[keep][:, None]
    S = X @ w.T
    es = ((H + 8) * W * (X.abs() @ w.abs().T) + 4 * W * (1 + S.abs())).amax(-1, keepdim=True) if len(keep) else S[:, :1]
    lse = torch.logsumexp(S, -1)
    elem = torch.arange(len(keep))
    val = {k: torch.zeros(n, dtype=torch.float64) for k in ("loss", "lse")}
    bnd = {k: torch.zeros(n, dtype=torch.float64) for k in ("loss", "lse")}
    val["lse"][keep], val["loss"][keep] = lse, lse - S[elem, lab]
    bnd["lse"][keep] = es[:, 0] + (V + 8) * W + 4 * W * lse.abs()
    bnd["loss"][keep] = 2 * bnd["lse"][keep] + 4 * W * val["loss"][keep].abs()
    P = torch.exp(S - lse[:, None])
    hot = torch.zeros_like(P)
    hot[elem, lab] = 1.0
    G = up * (P - hot)
    eG = up.abs() * P * (2 * es + bnd["lse"][keep][:, None] + 4 * W) + (u + 2 * W) * G.abs()
    val["dx"], bnd["dx"] = torch.zeros_like(x), torch.zeros_like(x)
    val["dx"][keep] = G @ w
    bnd["dx"][keep] = eG @ w.abs() + (V + 8) * W * (G.abs() @ w.abs()) + u * (G @ w).abs()
    val["dw"] = G.T @ X
    bnd["dw"] = eG.T @ X.abs() + (n + 8) * W * (G.abs().T @ X.abs()) + u * val["dw"].abs()
    return val, bnd


def embed(ids, table, mask_rows, scale, dout):
    """(values, bounds) of out, d_table, d_mask."""
    u = half_step(table.dtype)
    V, H = table.shape
    ids, t, d = ids.long().cpu(), table.detach().double().cpu(), dout.double().cpu()
    k = 0
    if mask_rows is not None:
        k = mask_rows.shape[0]
        t = torch.cat([t, mask_rows.detach().double().cpu()])
    there = torch.nonzero((ids >= 0) & (ids < V + k))[:, 0]
    out = torch.zeros((len(ids), H), dtype=torch.float64)
    out[there] = scale * t[ids[there]]
    grad, mag = torch.zeros_like(t), torch.zeros_like(t)
    grad.index_add_(0, ids[there], d[there])
    mag.index_add_(0, ids[there], d[there].abs())
    grad, mag = grad * scale, mag * abs(scale)
    eg = u * grad.abs() + (len(ids) + 4) * W * mag
    return ({"out": out, "d_table": grad[:V], "d_mask": grad[V:]},
            {"out": (u + 2 * W) * out.abs(), "d_table": eg[:V], "d_mask": eg[V:]})


def check(got, val, bnd, names):
    for n in names:
        g = got[n].detach().double().cpu()
        assert g.shape == val[n].shape, n
        off = (g - val[n]).abs()
        bad = ~(off <= bnd[n] + 1e-30)
        if bad.any():
            at = tuple(int(i) for i in torch.nonzero(bad)[0])
            raise AssertionError(f"{n}: {int(bad.sum())} of {bad.numel()} values off, first at {at}: got {g[at].item()}, want "
                                 f"{val[n][at].item()}, bound {bnd[n][at].item():.3g}")

"""Plain 64-bit implementations of the layer operators beside the stage calls, with bounds for what their kernels round to bf16.

A bf16 rounding is off by at most H = 2^-8 of the value.  The attention kernels round P, dS and the results; scores, sums and statistics
are fp32, whose errors (products of up to 128 terms, exponents of up to some tens) stay below S = 2e-5 of the sums of absolute values."""
import math

import torch

H = 2.0 ** -8
S = 2.0e-5
F64 = torch.float64


def cross_attention(q, k, v, do, q_len, kv_len, scale, exact_delta):
    """q, do [b, nq, a, d]; k, v [b, nk, kh, d] (any type, read as 64 bits; rows behind the lengths are not used); lengths as lists.
    Returns {name: (value, bound)} for o, lse, dq, dk, dv; exact_delta(kv_len): whether the kernel's delta is free of o's rounding."""
    b, nq, a, d = q.shape
    nk, kh = k.shape[1], k.shape[2]
    dev = q.device
    z = lambda *s: torch.zeros(s, dtype=F64, device=dev)  # noqa: E731
    out = {"o": (z(b, nq, a, d), z(b, nq, a, d)), "lse": (z(b, a, nq) - math.inf, z(b, a, nq)), "dq": (z(b, nq, a, d), z(b, nq, a, d)),
           "dk": (z(b, nk, kh, d), z(b, nk, kh, d)), "dv": (z(b, nk, kh, d), z(b, nk, kh, d))}
    for i in range(b):
        m, n = q_len[i], kv_len[i]
        if m == 0 or n == 0:
            continue
        for h in range(a):
            g = h // (a // kh)
            qh, kx, vx, dh = [t.double() for t in (q[i, :m, h], k[i, :n, g], v[i, :n, g], do[i, :m, h])]
            s = (qh @ kx.t()) * scale
            lse = torch.logsumexp(s, 1)
            p = (s - lse[:, None]).exp()
            o = p @ vx
            slack = p @ vx.abs()
            out["o"][0][i, :m, h] = o
            o_err = H * (1 + S) * (slack + o.abs()) + S * slack
            out["o"][1][i, :m, h] = o_err
            out["lse"][0][i, h, :m] = lse
            out["lse"][1][i, h, :m] = S * (1 + s.abs().amax(1))
            dp = dh @ vx.t()
            dp_abs = dh.abs() @ vx.abs().t()
            delta = (p * dp).sum(1, keepdim=True)
            delta_err = S * (p * dp_abs).sum(1, keepdim=True)
            if not exact_delta(n):
                delta_err = delta_err + (dh.abs() * o_err).sum(1, keepdim=True)
            ds = p * (dp - delta)
            ds_err = H * ds.abs() + p * (1 + H) * (S * (dp_abs + (p * dp_abs).sum(1, keepdim=True)) + delta_err)
            dq = scale * ds @ kx
            out["dq"][0][i, :m, h] = dq
            out["dq"][1][i, :m, h] = (1 + H) * scale * (ds_err @ kx.abs()) + H * dq.abs()
            out["dk"][0][i, :n, g] += scale * ds.t() @ qh
            out["dk"][1][i, :n, g] += (1 + H) * scale * (ds_err.t() @ qh.abs())
            out["dv"][0][i, :n, g] += p.t() @ dh
            out["dv"][1][i, :n, g] += (1 + H) * (H + S) * (p.t() @ dh.abs())
    for name in ("dk", "dv"):
        out[name][1].add_(H * out[name][0].abs())
    return out


def balance(logits, idx, mask, seq, top_k, coef, z_coef, grad_scale):
    """Returns counts, tokens, loss (with autograd), gradient and the size of the terms the gradient is a difference of."""
    T, E = logits.shape
    G = T // seq
    x = logits.double().detach().clone()
    keep = mask.bool() if mask is not None else torch.ones(T, dtype=torch.bool, device=x.device)
    keep_p = keep & ~torch.isneginf(logits).all(1)
    x[~keep_p] = 0.0
    x.requires_grad_()
    counts = torch.zeros((G, E), dtype=torch.int64, device=x.device)
    tokens = keep.reshape(G, seq).sum(1)
    N = int(tokens.sum())
    bal, z = x.sum() * 0, x.sum() * 0
    f_rows = torch.zeros((T, E), dtype=F64, device=x.device)
    for g in range(G):
        rows = torch.arange(g * seq, (g + 1) * seq, device=x.device)
        rows = rows[keep[rows]]
        if not rows.numel():
            continue
        ids = idx[rows].long().reshape(-1)
        counts[g] = torch.bincount(ids[(ids >= 0) & (ids < E)], minlength=E)
        f_rows[rows] = counts[g].double() / (rows.numel() * top_k)
    p = x.softmax(1) * keep_p[:, None]
    if N:
        bal = E / N * (f_rows * p).sum()
        z = torch.where(keep_p, torch.logsumexp(x, 1), 0.0).square().sum() / N
    loss = coef * bal + z_coef * z
    grad = grad_scale * torch.autograd.grad(loss, x)[0]
    n = max(N, 1)
    terms = abs(grad_scale) * p.detach() * (abs(coef) * E / n * (f_rows + (f_rows * p.detach()).sum(1, keepdim=True)) +
                                            2 * abs(z_coef) / n * torch.logsumexp(x.detach(), 1).abs()[:, None])
    return counts, torch.cat((tokens, tokens.sum()[None])), torch.stack((loss, bal, z)).detach(), grad, terms


def frequencies(kind, base, factor, slow, fast, trained, rot):
    i = torch.arange(rot // 2, dtype=F64)
    if kind == 2:
        base = base * factor ** (rot / (rot - 2.0))
    th = base ** (-2.0 * i / rot)
    if kind == 1:
        return th / factor
    if kind == 3:
        turns = trained * th / (2 * math.pi)
        keep = ((turns - slow) / (fast - slow)).clamp(0, 1)
        return th * (keep + (1 - keep) / factor)
    return th


def rotate(x, cs, layout, rot, bwd):
    """x [T, heads, d], cs [T, rot / 2, 2]; 64 bits."""
    x = x.double().clone()
    c, s = cs[:, None, :, 0].double(), cs[:, None, :, 1].double() * (-1 if bwd else 1)
    if layout:
        u, w = x[..., 0:rot:2].clone(), x[..., 1:rot:2].clone()
        x[..., 0:rot:2], x[..., 1:rot:2] = u * c - w * s, w * c + u * s
    else:
        u, w = x[..., :rot // 2].clone(), x[..., rot // 2:rot].clone()
        x[..., :rot // 2], x[..., rot // 2:rot] = u * c - w * s, w * c + u * s
    return x

"""Plain 64-bit implementations of the operators for training on packed documents, with bounds for what their kernels round.

A bf16 rounding is off by at most H = 2^-8 of the value.  Sums, scores and statistics are fp32, whose errors (products of up to 128 terms, exponents of up to some
tens) stay below S = 2e-5 of the sums of absolute values; a capped score is off by cap 2^-21 at most (1 + e and its reciprocal, 2^-23 each, times 2 cap)."""
import math

import torch

H = 2.0 ** -8
S = 2.0e-5
F64 = torch.float64


def plan(starts, prefix, window, T, seq):
    """Lists of (span, pos, first) of every token, token by token."""
    span, pos, first = [], [], []
    for t in range(T):
        row = t // seq * seq
        doc = next((i for i in range(len(starts) - 1) if starts[i] <= t < starts[i + 1]), None)
        if doc is None:
            span.append((0, 0))
            pos.append(0)
            first.append(1)
            continue
        lo, hi, end = max(starts[doc], row), t + 1, min(starts[doc + 1], row + seq)
        if window:
            lo = max(lo, t + 1 - window)
        if prefix is not None:
            hi = max(hi, min(starts[doc] + prefix[doc], end))
        span.append((lo - row, hi - row))
        pos.append(t - starts[doc])
        first.append(int(t == starts[doc]))
    return span, pos, first


def span_attention(q, k, v, do, span, pos, slopes, cap, scale, rest=True):
    """q, do [b, nq, a, d]; k, v [b, nk, kh, d] (any type, read as 64 bits); span [b, nq, 2], pos [b, nq] integers.  Returns {name: (value, bound)} for o, lse, dq, dk,
    dv; rest: whether the backward call is given what o's rounding left over."""
    b, nq, a, d = q.shape
    nk, kh = k.shape[1], k.shape[2]
    dev = q.device
    z = lambda *s: torch.zeros(s, dtype=F64, device=dev)  # noqa: E731
    out = {"o": (z(b, nq, a, d), z(b, nq, a, d)), "lse": (z(b, a, nq) - math.inf, z(b, a, nq)), "dq": (z(b, nq, a, d), z(b, nq, a, d)),
           "dk": (z(b, nk, kh, d), z(b, nk, kh, d)), "dv": (z(b, nk, kh, d), z(b, nk, kh, d))}
    j = torch.arange(nk, device=dev)
    for i in range(b):
        seen = (j >= span[i, :, :1]) & (j < span[i, :, 1:])
        live = seen.any(1)
        if not bool(live.any()):
            continue
        seen, p_at = seen[live], pos[i][live].double()[:, None]
        for h in range(a):
            g = h // (a // kh)
            qh, dh = q[i, live, h].double(), do[i, live, h].double()
            kx, vx = k[i, :, g].double(), v[i, :, g].double()
            used = seen.any(0)[:, None]      # (what nothing sees may hold anything)
            kx, vx = torch.where(used, kx, 0.0), torch.where(used, vx, 0.0)
            s = (qh @ kx.t()) * scale
            turn = 1.0
            s_err = S * (1 + (qh.abs() @ kx.abs().t()) * scale)
            if cap:
                t = torch.tanh(s / cap)
                s, turn = cap * t, 1 - t * t
                s_err = s_err * turn + cap * 2.0 ** -21 + S * s.abs()
            if slopes is not None:
                far = float(slopes[h]) * (j.double() - p_at).abs()
                s, s_err = s - far, s_err + 2.0 ** -22 * far
            s = s.masked_fill(~seen, -math.inf)
            lse = torch.logsumexp(s, 1)
            p = (s - lse[:, None]).exp()
            s_err = torch.where(seen, s_err, 0.0)
            lse_err = (p * s_err).sum(1) + S * (1 + lse.abs())
            p_rel = torch.where(seen, s_err + lse_err[:, None] + S, 0.0) * 1.1      # (exp(e) - 1 < 1.1 e for e < 0.1)
            assert float(p_rel.max()) < 0.1
            o = p @ vx
            spread = p @ vx.abs() + o.abs()
            # weights p (1 + e) / sum p (1 + e), |e| <= H + p_rel
            o_err = (H * (1 + 3 * H)) * spread + 2 * (p * p_rel) @ vx.abs() + 2 * (p * p_rel).sum(1, keepdim=True) * o.abs() + S * spread
            out["o"][0][i, live, h] = o
            out["o"][1][i, live, h] = o_err + H * o.abs()
            out["lse"][0][i, h, live] = lse
            out["lse"][1][i, h, live] = lse_err
            dp = dh @ vx.t()
            dp_abs = dh.abs() @ vx.abs().t()
            delta = (p * dp).sum(1, keepdim=True)
            away = (p * (dp - delta).abs()).sum(1, keepdim=True)
            delta_err = (H * (1 + 3 * H)) * away + 2 * (p * p_rel * (dp - delta).abs()).sum(1, keepdim=True) + S * (p * dp_abs).sum(1, keepdim=True)
            delta_err = delta_err + (2.0 ** -16 if rest else H) * (dh.abs() * o.abs()).sum(1, keepdim=True)
            ds = p * (dp - delta)
            ds_err = p_rel * ds.abs() + p * (S * dp_abs + delta_err)
            if cap:
                ds_err = ds_err * turn + ds.abs() * 2.0 ** -19      # 4 r (1 - r), r off by 2^-22
                ds = ds * turn
            ds_err = ds_err + H * (ds.abs() + ds_err)
            dq = scale * ds @ kx
            out["dq"][0][i, live, h] = dq
            out["dq"][1][i, live, h] = (1 + H) * scale * (ds_err @ kx.abs()) + S * scale * (ds.abs() @ kx.abs()) + H * dq.abs()
            out["dk"][0][i, :, g] += scale * ds.t() @ qh
            out["dk"][1][i, :, g] += (1 + H) * scale * (ds_err.t() @ qh.abs()) + S * scale * (ds.abs().t() @ qh.abs())
            out["dv"][0][i, :, g] += p.t() @ dh
            out["dv"][1][i, :, g] += (1 + H) * ((p * (H + S + p_rel * (1 + H))).t() @ dh.abs())
    for name in ("dk", "dv"):
        out[name][1].add_(H * out[name][0].abs())
    return out


def weights(kind, g):
    """f, 1 - f, w and dw/dg of gates in 64 bits (1 - f as sigmoid(-g): near f = 1 the difference has no digits left)."""
    f, r = g.sigmoid(), (-g).sigmoid()
    if kind == 0:
        return f, r, torch.ones_like(f), torch.zeros_like(f)
    if kind == 1:
        return f, r, r, -f * r
    w = (r * (1 + f)).sqrt()
    return f, r, w, -f * f * r / w


def scan(kind, x, g, dy, first, length, h0, dlast):
    """x, g, dy [b, n, c]; first [b, n] or None; length list or None; h0, dlast [b, c] or None.  Returns {name: (value, bound)} for y, last, dx, dg, dh0."""
    b, n, c = x.shape
    x, g, dy = x.double(), g.double(), dy.double()
    f, less, w, dw = weights(kind, g)
    zero = torch.zeros((b, c), dtype=F64, device=x.device)
    h, hs = (h0.double() if h0 is not None else zero), (h0.double().abs() if h0 is not None else zero)
    length = length or [n] * b
    y, before, before_s, ys = [torch.zeros_like(x) for _ in range(4)]
    keep = torch.ones((b, n, 1), dtype=torch.bool, device=x.device) if first is None else (first == 0)[..., None]
    on = torch.stack([torch.arange(n, device=x.device) < m for m in length])[..., None]
    # hs: the sum of the absolute terms, times how many roundings each of them has been through, so the error is 2^-21 of it or less
    for t in range(n):
        before[:, t] = torch.where(keep[:, t], h, 0.0)
        before_s[:, t] = torch.where(keep[:, t], hs, 0.0)
        u = w[:, t] * x[:, t]
        new, news = f[:, t] * before[:, t] + u, f[:, t] * (before_s[:, t] + before[:, t].abs()) + u.abs()
        h, hs = torch.where(on[:, t], new, h), torch.where(on[:, t], news, hs)
        y[:, t], ys[:, t] = torch.where(on[:, t], new, 0.0), torch.where(on[:, t], news, 0.0)
    E = 2.0 ** -20      # of f, w, the products and sums of a token: four roundings of 2^-24, functions of 2^-22
    out = {"y": (y, H * y.abs() + 2 * E * ys), "last": (h, E * hs)}
    mu, mus = (dlast.double() if dlast is not None else zero), (dlast.double().abs() if dlast is not None else zero)
    dx, dg, dxe, dge = [torch.zeros_like(x) for _ in range(4)]
    for t in range(n - 1, -1, -1):
        lam, lams = dy[:, t] + mu, dy[:, t].abs() + mus + mu.abs()
        dx[:, t], dxe[:, t] = torch.where(on[:, t], w[:, t] * lam, 0.0), torch.where(on[:, t], w[:, t] * lams, 0.0)
        r = less[:, t]
        gate = before[:, t] * f[:, t] * r + x[:, t] * dw[:, t]
        gates = before_s[:, t] * f[:, t] * r + (x[:, t] * dw[:, t]).abs()
        dg[:, t], dge[:, t] = torch.where(on[:, t], lam * gate, 0.0), torch.where(on[:, t], lams * gates + lam.abs() * gates + lams * gate.abs(), 0.0)
        fk = torch.where(keep[:, t], f[:, t], 0.0)
        mu, mus = torch.where(on[:, t], fk * lam, mu), torch.where(on[:, t], fk * (lams + lam.abs()), mus)
    out.update(dx=(dx, H * dx.abs() + 2 * E * dxe), dg=(dg, H * dg.abs() + 4 * E * dge), dh0=(mu, E * mus))
    return out


def philox(counter, key):
    """Ten rounds on Python's whole numbers; counter of four words, key of two."""
    x, k = list(counter), list(key)
    for _ in range(10):
        a, b = x[0] * 0xD2511F53, x[2] * 0xCD9E8D57
        x = [(b >> 32) ^ x[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ x[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return x


def stays(T, n, p, seed, offset):
    """[T, n] truth values, and the share that stays."""
    keep = round((1.0 - float(torch.tensor(p, dtype=torch.float32))) * 65536)
    out = torch.zeros(T * n, dtype=torch.bool)
    m = (1 << 32) - 1
    offset %= 1 << 64
    for i in range(T * n // 8):
        w = philox([i & m, i >> 32, offset & m, offset >> 32], [seed & m, seed >> 32])
        for e in range(8):
            out[8 * i + e] = (w[e // 2] >> 16 * (e % 2) & 0xFFFF) < keep
    return out.reshape(T, n), keep / 65536


def embedding_gradient(dx, ids, scale, V, given=None):
    """Value and bound: fp32 sums of n terms in chunks of 32, parts of those in eighths."""
    h = dx.shape[1]
    out = given.double().clone() if given is not None else torch.zeros((V, h), dtype=F64, device=dx.device)
    size = out.abs()
    at = (ids >= 0) & (ids < V)
    rows, where = dx.double()[at] * scale, ids[at].long()
    count = torch.bincount(where, minlength=V).double()[:, None]
    for to, what in ((out, rows), (size, rows.abs())):
        if int(count.max()) > 4096:      # (many additions to one place take the GPU ten seconds)
            to.copy_(to.cpu().index_add_(0, where.cpu(), what.cpu()))
        else:
            to.index_add_(0, where, what)
    return out, size * 2.0 ** -24 * (3 + torch.minimum(count, 32 + 8 + count / 256))

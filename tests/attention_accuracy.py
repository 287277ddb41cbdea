"""How exact the gradients of cross attention are: bounds and limits counted from what the kernels round, and a model of those roundings in 64 bits that
shows what the limits tell apart.

  dq     is rounded once (H); dS goes into its product as two bf16 numbers, off by H^2;  delta is off by no more than TAU sum_k |dS_k| of its row, by
         nothing where it comes from the scores themselves (up to 256 keys, or with the key loop in slices).  With delta off by x, dS is off by P x and sums up
         to x over a row (sum P = 1), which the kernel sees and takes off again with M, the mean of the first 64 keys:  sum (dS + P x) K - x M
         = sum dS K + x sum P (K - M), so dq is off by x sum P |K - M| at most, element by element
  dk     is rounded once, its dS once; the delta it takes is always the corrected one
  fp32   a product of d terms adds up d / 32 + 32 roundings at most, E = 40 * 2^-24 of the terms' absolute values; an exponent that is off by e takes its
         exponential e off, and a row's log-sum-exp is off by what its exponents are
The roundings of a whole tensor are as good as independent: half steps of bf16 are 1.66e-3 of a tensor's 2-norm, whatever the tensor."""
import math

import torch

H = 2.0 ** -8
TAU = 2.0 ** -8
E = 40 * 2.0 ** -24
F64 = torch.float64
ONE_ROUNDING = 1.66e-3      # relative 2-norm of one rounding to bf16


def sharp_queries(k, heads, rows, gain, g):
    """rows x heads queries, each the image of one key (times gain) and noise: the larger the gain, the more of a row's weight is on that key.  k [n, kh, d]."""
    n, kh, d = k.shape
    grp = heads // kh
    q = torch.randn((rows, heads, d), generator=g)
    for h in range(heads):
        q[:, h] += gain * k[torch.randint(n, (rows,), generator=g), h // grp]
    return q


def gradients(q, k, v, do, scale, exact_delta):
    """One sequence: q, do [m, a, d]; k, v [n, kh, d], read as 64 bits.  Returns {name: (value, bound)} for dq and dk."""
    q, k, v, do = [t.to(F64) for t in (q, k, v, do)]
    a, kh = q.shape[1], k.shape[1]
    out = {"dq": (torch.zeros_like(q), torch.zeros_like(q)), "dk": (torch.zeros_like(k), torch.zeros_like(k))}
    for h in range(a):
        g = h // (a // kh)
        qh, kx, vx, dh = q[:, h], k[:, g], v[:, g], do[:, h]
        s = scale * qh @ kx.t()
        lse = torch.logsumexp(s, 1, keepdim=True)
        p = (s - lse).exp()
        dp = dh @ vx.t()
        ds = p * (dp - (p * dp).sum(1, keepdim=True))
        # exponents: the score's sum, and two roundings of it, of lse and of their difference; twice, since lse has the same
        e = (2 * (E * scale * qh.abs() @ kx.abs().t() + 2.0 ** -22 * (s.abs() + lse.abs()))).amax(1, keepdim=True)
        dp_abs = dh.abs() @ vx.abs().t()
        size = ds.abs().sum(1, keepdim=True)
        noise = e * (ds.abs() + p * size) + E * p * (dp_abs + (p * dp_abs).sum(1, keepdim=True))
        for name, rounded, other in (("dq", H * H, kx), ("dk", H, qh)):
            err = rounded * ds.abs() + noise
            if name == "dq":
                far = 0.0 if exact_delta else TAU / (1 - TAU) * size * (p @ (kx - kx[:64].mean(0)).abs())
                out[name][0][:, h] = scale * ds @ other
                out[name][1][:, h] = scale * (1 + H) * (err @ other.abs() + far)
            else:
                out[name][0][:, g] += scale * ds.t() @ other
                out[name][1][:, g] += scale * (1 + H) * (err.t() @ other.abs())
    for value, bound in out.values():
        bound.add_(H * value.abs())
    return out


def bf16(t):
    return t.to(torch.bfloat16).to(t.dtype)


def as_the_kernels_round(q, k, v, do, scale, exact_delta, parts=2, repeat=True, correct=True):
    """dq and dk as the kernels make them but for fp32: dS in `parts` bf16 parts for dq, which is corrected by what delta was off by times sum P K where that is more
    than TAU sum |dS|, else times the mean of 64 keys (repeat), and the corrected delta for dk (correct)."""
    q, k, v, do = [t.to(F64) for t in (q, k, v, do)]
    a, kh = q.shape[1], k.shape[1]
    dq, dk = torch.zeros_like(q), torch.zeros_like(k)
    for h in range(a):
        g = h // (a // kh)
        qh, kx, vx, dh = q[:, h], k[:, g], v[:, g], do[:, h]
        p = (scale * qh @ kx.t()).softmax(1)
        dp = dh @ vx.t()
        stored = (dh * bf16(bf16(p) @ vx)).sum(1, keepdim=True)
        delta = (p * dp).sum(1, keepdim=True) if exact_delta else stored
        ds = p * (dp - delta)
        off = ds.sum(1, keepdim=True)
        x = bf16(ds)
        if parts == 2:
            x = x + bf16(ds - x)
        got = x @ kx
        if repeat and not exact_delta:
            got = got - off * torch.where(off.abs() > TAU * ds.abs().sum(1, keepdim=True), p @ kx, kx[:64].mean(0))
        dq[:, h] = bf16(scale * got)
        dk[:, g] += scale * bf16(p * (dp - delta - (off if correct else 0.0))).t() @ qh
    return {"dq": dq, "dk": bf16(dk)}


def distance(x, y):
    return float((x.to(F64) - y).norm() / y.norm())


# Limits of the relative 2-norm.
# dq of ordinary rows (d^-1/2 q.k of standard deviation 1: weights with sum P^2 of about e / n, 0.03 at most; or of any where delta comes from the scores):
#   its own rounding u and, where delta comes from the stored output, that one's share.  The output carries P's rounding and its own, together
#   sqrt(2) u |o| with |o| = sqrt(sum P^2) |v|, and delta / |v| with it, so dS / (P |v|) is off by sqrt(2) u sqrt(0.03) = 0.25 u:  1.71e-3 in all.
#   One more rounding of dS makes sqrt(2) u, 2.35e-3.
DQ_ORDINARY = 2.1e-3
# dq of sharp rows: c = |off| / sum |dS| of the rows that are not taken again is spread over 0 .. TAU, TAU / sqrt(3) in the mean square; a row on one key has
#   sum |dS| = 2 |dS_top|, so its dq is off by 2 c; with the result's own rounding sqrt((2 TAU / sqrt(3))^2 + 1.66e-3^2) = 4.8e-3.
DQ_SHARP = math.sqrt((2 * TAU) ** 2 / 3 + ONE_ROUNDING ** 2)
# the same with delta from the scores: its own rounding, and the fp32 of dP - delta
DQ_SHARP_EXACT = 2.1e-3
# dk: dS and the result are rounded, sqrt(2) * 1.66e-3 = 2.35e-3, and a quarter more where a key's few terms, which have either sign, cancel
DK_SHARP = 3.0e-3

"""What the speed of the operators for training on packed documents is measured on: attention in which every query sees a span of the
keys, the gated linear recurrence, the embedding with its gradient, and dropout.

A case is one pass through one operator on inputs that are already on the GPU:

  lookup  rp_op_embed_fwd            the rows of the tokens, scaled
  embed   rp_op_embed_fwd, _bwd      the same, and the gradient of the table, written anew or added to what is there
  drop    rp_op_dropout              dropout of a branch, alone (as its gradient takes it) or onto the residual stream
  scan    rp_op_scan_fwd             h_t = f_t h_t-1 + w(f_t) x_t from a state: outputs and the last state
  recur   rp_op_scan_fwd, _bwd       the same, and the gradients of x, of the gates and of the state before
  span    rp_op_span_attn_fwd        attention: output, log-sum-exp
  attend  rp_op_span_attn_fwd, _bwd  the same, and dq, dk, dv

With `own` false the same results come from elementary torch operations in 32 bits.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
BF16, F32, F64, I32, I64 = torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.int64
PLAIN, MEAN, ENERGY = 0, 1, 2      # what the recurrence's input is weighted with: 1, 1 - f, sqrt(1 - f^2)


def listed():
    return [
        # eight sequences that each add one token
        dict(name="lookup_8x4096", kind="lookup", T=8, V=151936, h=4096, scale=1.0, pad=0, add=0),
        # a padded batch through a narrower model, on top of the gradient that the tied head has left
        dict(name="embed_4084x2880", kind="embed", T=4084, V=32000, h=2880, scale=53.665631, pad=1, add=1),
        # a long document and a large vocabulary, the table's gradient written anew
        dict(name="embed_16384x4096", kind="embed", T=16384, V=151936, h=4096, scale=1.0, pad=0, add=0),
        # the gradient of a short batch's branch
        dict(name="drop_512x2048", kind="drop", T=512, n=2048, p=0.1, res=0),
        # the branch of a wide layer, onto the residual stream
        dict(name="drop_16384x5120", kind="drop", T=16384, n=5120, p=0.05, res=1),
        # generation: one token of eight sequences, from their states
        dict(name="scan_token_8x4096", kind="scan", batch=8, seq=1, c=4096, weight=MEAN, docs=1, ragged=0, state=1),
        # training on a padded batch, sequences of an odd length
        dict(name="recur_4x1021x2880", kind="recur", batch=4, seq=1021, c=2880, weight=ENERGY, docs=1, ragged=1, state=0),
        # training on a long row of packed documents
        dict(name="recur_16384x4096", kind="recur", batch=1, seq=16384, c=4096, weight=MEAN, docs=9, ragged=0, state=1),
        # generation: one token of eight sequences, keys of different lengths, capped scores
        dict(name="span_token_8x4096", kind="span", batch=8, seq_q=1, seq_kv=4096, a=32, kh=8, d=128, docs=1, prefix=0, window=0, cap=50.0, bias=0),
        # training with prefixes and a bias by distance, narrow heads, no length a multiple of a tile
        dict(name="attend_2x1021_prefix_bias", kind="attend", batch=2, seq_q=1021, seq_kv=1021, a=64, kh=8, d=64, docs=3, prefix=1, window=0, cap=0.0, bias=1),
        # training on a window with capped scores
        dict(name="attend_4096_window_cap", kind="attend", batch=1, seq_q=4096, seq_kv=4096, a=16, kh=8, d=128, docs=1, prefix=0, window=1024, cap=30.0, bias=0),
        # training on a long row of packed documents: the largest case
        dict(name="attend_16384_docs", kind="attend", batch=1, seq_q=16384, seq_kv=16384, a=32, kh=8, d=128, docs=4, prefix=0, window=0, cap=0.0, bias=0),
    ]


HEADS = ((4, 2), (16, 8), (16, 16), (32, 8), (64, 8), (64, 4), (6, 2))


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    kind = rng.choice(("lookup", "embed", "embed", "drop", "drop", "scan", "recur", "recur", "span", "attend", "attend", "attend"))
    if kind in ("lookup", "embed"):
        h = 8 * _log(rng, 16, 640)
        V = _log(rng, 1000, 151936)
        T = _log(rng, 1, min(32768, 16384 * 4096 // h))
        return dict(kind=kind, T=T, V=V, h=h, scale=rng.choice((1.0, 1.0, h ** 0.5)), pad=rng.randint(0, 1) if T > 8 else 0, add=rng.randint(0, 1))
    if kind == "drop":
        n = 8 * _log(rng, 8, 3200)
        return dict(kind=kind, T=_log(rng, 1, 16384 * 5120 // n), n=n, p=rng.choice((0.0, 0.05, 0.1, 0.2, 0.5, 0.9)), res=rng.randint(0, 1))
    if kind in ("scan", "recur"):
        c, batch = 8 * _log(rng, 8, 1024), rng.choice((1, 1, 2, 3, 8))
        seq = _log(rng, 1, max(1, min(32768, 16384 * 4096 // (c * batch))))
        if kind == "recur":
            seq = max(2, seq)
        return dict(kind=kind, batch=batch, seq=seq, c=c, weight=rng.randint(0, 2), docs=rng.randint(1, max(1, min(12, seq // 8))), ragged=rng.randint(0, 1),
                    state=rng.randint(0, 1))
    a, kh = rng.choice(HEADS)
    d = rng.choice((64, 128, 128))
    batch = rng.choice((1, 1, 2, 4, 8))
    most = 32 * 8192 * 8192 * 128 // (a * d * batch)      # seq_q * seq_kv
    cap, bias = rng.choice((0.0, 0.0, 20.0, 50.0)), rng.choice((0, 0, 1))
    if kind == "span" and rng.random() < 0.6:             # steps of a generation, or the last piece of a long prompt
        seq_q = rng.choice((1, 1, 2, 5, 17, 300))
        seq_kv = max(seq_q, _log(rng, 1, min(32768, max(1, most // seq_q))))
        return dict(kind=kind, batch=batch, seq_q=seq_q, seq_kv=seq_kv, a=a, kh=kh, d=d, docs=1, prefix=0, window=rng.choice((0, 0, _log(rng, 8, 4096))), cap=cap,
                    bias=bias)
    seq = _log(rng, 16, int(math.sqrt(most)))             # (the gradients of a softmax over one key are zero: nothing to compare)
    return dict(kind=kind, batch=batch, seq_q=seq, seq_kv=seq, a=a, kh=kh, d=d, docs=rng.randint(1, max(1, min(12, seq // 16))), prefix=rng.randint(0, 1),
                window=rng.choice((0, 0, _log(rng, 8, 4096))), cap=cap, bias=bias)


# ---------------------------------------------------------------------------------------------------- inputs
def _starts(g, rows, seq, docs):
    """[rows, docs] first tokens of the documents that a row is packed with; the first one's is 0."""
    s = torch.randint(0, seq, (rows, docs), generator=g, device=DEV)
    s[:, 0] = 0
    return s.sort(1).values


def _lengths(g, batch, longest, least):
    """Lengths of a padded batch: the longest fills it, the others are spread."""
    n = torch.randint(least, longest + 1, (batch,), generator=g, device=DEV, dtype=I32)
    n[0] = longest
    return n


def _spans(c, g):
    """What every query sees, [batch, seq_q, 2] (first key, key behind the last), and its position among the keys."""
    b, nq, nk = c["batch"], c["seq_q"], c["seq_kv"]
    t = torch.arange(nq, device=DEV).expand(b, nq)
    if nq != nk:                     # queries behind a cache of a length of its own
        pos = t + (_lengths(g, b, nk, nq).long() - nq)[:, None]
        lo, hi = torch.zeros_like(pos), pos + 1
    else:
        starts = _starts(g, b, nq, c["docs"])
        doc = torch.searchsorted(starts, t.contiguous(), right=True) - 1
        pos, lo, hi = t, starts.gather(1, doc), t + 1
        if c["prefix"]:              # the first part of every document sees itself both ways, up to half of it
            ends = torch.cat((starts[:, 1:], torch.full((b, 1), nq, device=DEV)), 1)
            n = (torch.rand((b, c["docs"]), generator=g, device=DEV) * 0.5 * (ends - starts)).long()
            hi = torch.maximum(hi, (starts + n).gather(1, doc))
    if c["window"]:
        lo = torch.maximum(lo, pos + 1 - c["window"])
    return torch.stack((lo, hi), -1).to(I32).contiguous(), pos.to(I32).contiguous()


def prepare(case, seed):
    c, g = case, torch.Generator(device=DEV).manual_seed(seed)

    def normal(*shape, std=1.0, dtype=BF16):
        return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, std, generator=g)

    s = {"case": c, "stream": torch.cuda.current_stream().cuda_stream}
    if c["kind"] in ("lookup", "embed"):
        T, V, h = c["T"], c["V"], c["h"]
        # frequent tokens have low numbers: about as many tokens between 10 and 100 as between 1000 and 10000
        s["ids"] = torch.exp(torch.rand(T, generator=g, device=DEV) * math.log(V)).long().sub_(1).clamp_(0, V - 1).to(I32)
        if c["pad"]:                 # padding has no row
            s["ids"][torch.rand(T, generator=g, device=DEV) < 0.15] = -1
        s["table"] = normal(V, h, std=0.02)
        s["x"] = torch.empty((T, h), dtype=BF16, device=DEV)
        if c["kind"] == "embed":
            s["dx"] = normal(T, h)
            s["dtable"] = normal(V, h, dtype=F32) if c["add"] else torch.empty((V, h), dtype=F32, device=DEV)
        return s
    if c["kind"] == "drop":
        s["x"] = normal(c["T"], c["n"])
        s["res"] = normal(c["T"], c["n"], std=2.0) if c["res"] else None
        s["y"] = torch.empty_like(s["x"])
        s["seed"] = (seed * 0x9E3779B97F4A7C15 + 12345) % (1 << 64)
        s["offset"] = seed % 1000 * 7919
        return s
    if c["kind"] in ("scan", "recur"):
        b, n, ch = c["batch"], c["seq"], c["c"]
        s["x"] = normal(b * n, ch)
        # gates that keep half of the state a token and gates that keep 0.998 of it
        s["g"] = (normal(b * n, ch, dtype=F32) + 6.0 * torch.rand(ch, generator=g, device=DEV)).to(BF16)
        s["y"] = torch.empty_like(s["x"])
        s["first"] = None
        if c["docs"] > 1:                # (a row's first document may go on from the row before)
            s["first"] = torch.zeros((b, n), dtype=torch.uint8, device=DEV).scatter_(1, _starts(g, b, n, c["docs"])[:, 1:], 1)
        s["len"] = _lengths(g, b, n, 0) if c["ragged"] else None
        s["h0"] = normal(b, ch, dtype=F32) if c["state"] else None
        s["last"] = torch.empty((b, ch), dtype=F32, device=DEV)
        if c["kind"] == "recur":
            s["dy"] = normal(b * n, ch)
            s["dlast"] = normal(b, ch, dtype=F32) if c["state"] else None
            s["dx"], s["dg"] = torch.empty_like(s["x"]), torch.empty_like(s["x"])
            s["dh0"] = torch.empty((b, ch), dtype=F32, device=DEV) if c["state"] else None
        return s
    b, nq, nk, a, kh, d = [c[x] for x in ("batch", "seq_q", "seq_kv", "a", "kh", "d")]
    s["q"], s["k"], s["v"] = normal(b * nq, a, d, std=2.0), normal(b * nk, kh, d), normal(b * nk, kh, d)
    s["span"], s["pos"] = _spans(c, g)
    s["slopes"] = (2.0 ** (-8.0 * torch.arange(1, a + 1, device=DEV) / a)).float() if c["bias"] else None
    s["o"] = torch.empty_like(s["q"])
    s["lse"] = torch.empty((b, a, nq), dtype=F32, device=DEV)
    if c["kind"] == "attend":
        s["do"] = normal(b * nq, a, d)
        s["rest"] = torch.empty_like(s["q"])
        s["dq"], s["dk"], s["dv"] = [torch.empty_like(s[x]) for x in ("q", "k", "v")]
        s["delta"] = torch.empty_like(s["lse"])
    return s


# ---------------------------------------------------------------------------------------------------- one pass
def run(state):
    return _own(state) if own else _plain(state)


def _scratch(s, n):
    if "scratch" not in s:      # a program asks once and keeps it
        s["scratch"] = torch.empty(max(n(), 16), dtype=torch.uint8, device=DEV)
    return s["scratch"]


def _own(s):
    from paper_2604_27085_amd import binding as B
    c, st = s["case"], s["stream"]
    if c["kind"] in ("lookup", "embed"):
        T, V, h = c["T"], c["V"], c["h"]
        B.rp_op_embed_fwd(st, s["table"], h, s["ids"], c["scale"], s["x"], h, T, V, h)
        if c["kind"] == "lookup":
            return s["x"]
        w = _scratch(s, lambda: B.rp_op_embed_scratch(T, V, h))
        B.rp_op_embed_bwd(st, s["dx"], h, s["ids"], c["scale"], s["dtable"], h, c["add"], T, V, h, w)
        return {"x": s["x"], "dtable": s["dtable"]}
    if c["kind"] == "drop":
        n = c["n"]
        B.rp_op_dropout(st, s["x"], n, s["res"], n, s["y"], n, c["T"], n, c["p"], s["seed"], s["offset"])
        return s["y"]
    if c["kind"] in ("scan", "recur"):
        b, n, ch = c["batch"], c["seq"], c["c"]
        if "scratch" not in s:
            s["states"] = torch.empty(B.rp_op_scan_sizes(b, n, ch)[0] // 4, dtype=F32, device=DEV) if c["kind"] == "recur" else None
        w = _scratch(s, lambda: B.rp_op_scan_sizes(b, n, ch)[1])
        B.rp_op_scan_fwd(st, c["weight"], s["x"], s["g"], s["y"], ch, ch, ch, s["first"], s["len"], s["h0"], s["last"], s["states"], b, n, ch, w)
        if c["kind"] == "scan":
            return {"y": s["y"], "last": s["last"]}
        B.rp_op_scan_bwd(st, c["weight"], s["x"], s["g"], s["dy"], s["dx"], s["dg"], ch, ch, ch, ch, ch, s["first"], s["len"], s["states"], s["dlast"], s["dh0"],
                         b, n, ch, w)
        return {x: s[x] for x in ("y", "last", "dx", "dg") + (("dh0",) if c["state"] else ())}
    b, nq, nk, a, kh, d = [c[x] for x in ("batch", "seq_q", "seq_kv", "a", "kh", "d")]
    w = _scratch(s, lambda: max(B.rp_op_span_attn_scratch(b, nq, nk, a, kh, d)[:2 if c["kind"] == "attend" else 1]))
    qd, kd, scale = a * d, kh * d, d ** -0.5
    B.rp_op_span_attn_fwd(st, s["q"], s["k"], s["v"], s["o"], s.get("rest"), s["lse"], qd, kd, kd, qd, s["span"], s["pos"], s["slopes"], c["cap"], b, nq, nk, a, kh,
                          d, scale, w)
    if c["kind"] == "span":
        return {"o": s["o"], "lse": s["lse"]}
    B.rp_op_span_attn_bwd(st, s["q"], s["k"], s["v"], s["o"], s["rest"], s["do"], s["lse"], s["delta"], s["dq"], s["dk"], s["dv"], qd, kd, kd, qd, qd, qd, kd, kd,
                          s["span"], s["pos"], s["slopes"], c["cap"], b, nq, nk, a, kh, d, scale, w)
    return {x: s[x] for x in ("o", "lse", "dq", "dk", "dv")}


def _plain(s):
    c = s["case"]
    if c["kind"] in ("lookup", "embed"):
        ids = s["ids"].long()
        there = ids >= 0
        x = torch.where(there[:, None], s["table"][ids.clamp(min=0)].float() * c["scale"], 0.0).to(BF16)
        if c["kind"] == "lookup":
            return x
        if not c["add"]:
            s["dtable"].zero_()
        s["dtable"].index_add_(0, ids.clamp(min=0), torch.where(there[:, None], s["dx"].float() * c["scale"], 0.0))
        return {"x": x, "dtable": s["dtable"]}
    if c["kind"] == "drop":
        return _plain_dropout(s, c)
    if c["kind"] in ("scan", "recur"):
        return _plain_scan(s, c)
    return _plain_attention(s, c)


def _words(group, seed, offset):
    """Philox 4x32 of ten rounds: four random words [groups, 4] from the 64-bit counter of each group, an offset and a key."""
    low = 0xFFFFFFFF
    x0, x1 = group & low, group >> 32
    x2, x3 = torch.full_like(group, offset & low), torch.full_like(group, offset >> 32)
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        a, b = x0 * 0xD2511F53, x2 * 0xCD9E8D57
        x0, x1, x2, x3 = (b >> 32 & low) ^ x1 ^ k0, b & low, (a >> 32 & low) ^ x3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack((x0, x1, x2, x3), 1)


def _kept(s, c):
    """[T, n]: which elements stay, and the share of them that does on average, as the generator's 16 bits resolve it."""
    keep = round((1.0 - float(np.float32(c["p"]))) * 65536)
    w = _words(torch.arange(c["T"] * c["n"] // 8, device=DEV, dtype=I64), s["seed"], s["offset"])
    bits = torch.stack((w & 0xFFFF, w >> 16), 2)
    return (bits < keep).reshape(c["T"], c["n"]), keep / 65536


def _plain_dropout(s, c):
    stay, share = _kept(s, c)
    y = torch.where(stay, s["x"].float() * (1.0 / share), 0.0)
    return (y + s["res"].float() if c["res"] else y).to(BF16)


def _scan(f, u):
    """h_t = f_t h_t-1 + u_t over the second dimension, by doubling: after k steps an element holds what 2^k tokens add up to."""
    f, u, step = f.clone(), u.clone(), 1
    while step < f.shape[1]:
        u[:, step:] += f[:, step:] * u[:, :-step].clone()
        f[:, step:] *= f[:, :-step].clone()
        step *= 2
    return u


def _plain_scan(s, c):
    b, n, ch = c["batch"], c["seq"], c["c"]
    x, g = s["x"].float().reshape(b, n, ch), s["g"].float().reshape(b, n, ch)
    f, r = 1.0 / (1.0 + torch.exp(-g)), 1.0 / (1.0 + torch.exp(g))        # r = 1 - f
    w = {PLAIN: torch.ones_like(f), MEAN: r, ENERGY: (r * (1.0 + f)).sqrt()}[c["weight"]]
    new = s["first"].bool()[..., None] if c["docs"] > 1 else torch.zeros((b, n, 1), dtype=torch.bool, device=DEV)
    live = (torch.arange(n, device=DEV) < (s["len"][:, None] if c["ragged"] else n)).expand(b, n)[..., None]
    h0 = s["h0"] if c["state"] else torch.zeros((b, ch), device=DEV)
    carry = torch.where(new, 0.0, f)          # padding keeps the state as it is
    carry, u = torch.where(live, carry, 1.0), torch.where(live, w * x, 0.0)
    u[:, 0] += carry[:, 0] * h0
    h = _scan(carry, u)
    out = {"y": torch.where(live, h, 0.0).reshape(b * n, ch).to(BF16), "last": h[:, -1].clone()}
    if c["kind"] == "scan":
        return out
    before = torch.where(new, 0.0, torch.cat((h0[:, None], h[:, :-1]), 1))
    lam = torch.where(live, s["dy"].float().reshape(b, n, ch), 0.0)
    if c["state"]:
        lam[:, -1] += s["dlast"]
    lam = _scan(torch.cat((carry[:, 1:], torch.ones_like(carry[:, :1])), 1).flip(1), lam.flip(1)).flip(1)
    dw = {PLAIN: torch.zeros_like(f), MEAN: -f * r, ENERGY: -f * f * (r / (1.0 + f)).sqrt()}[c["weight"]]
    out["dx"] = torch.where(live, lam * w, 0.0).reshape(b * n, ch).to(BF16)
    out["dg"] = torch.where(live, lam * (before * f * r + x * dw), 0.0).reshape(b * n, ch).to(BF16)
    if c["state"]:
        out["dh0"] = carry[:, 0] * lam[:, 0]
    return out


def _plain_attention(s, c):
    b, nq, nk, a, kh, d = [c[x] for x in ("batch", "seq_q", "seq_kv", "a", "kh", "d")]
    scale, grp = d ** -0.5, a // kh

    def heads(t, n):      # [b * n, heads, d] -> [b, kh, heads / kh * n, d]
        return t.float().reshape(b, n, kh, -1, d).permute(0, 2, 3, 1, 4).reshape(b, kh, -1, d)

    def rows(t, n, h):
        return t.reshape(b, kh, h // kh, n, d).permute(0, 3, 1, 2, 4).reshape(b * n, h, d).to(BF16)

    def lines(t):         # [b, nq, nk] -> one for every head of a group, as the scores are laid out
        return t[:, None, None].expand(b, 1, grp, nq, t.shape[-1])

    q, k, v = heads(s["q"], nq), heads(s["k"], nk), heads(s["v"], nk)
    j = torch.arange(nk, device=DEV)
    unseen = (j < s["span"][..., :1]) | (j >= s["span"][..., 1:])
    p = (q @ k.transpose(2, 3)).mul_(scale)
    slope = None
    if c["cap"]:
        p.div_(c["cap"]).tanh_()
        slope = 1.0 - p * p if c["kind"] == "attend" else None
        p.mul_(c["cap"])
    p = p.reshape(b, kh, grp, nq, nk)
    if c["bias"]:
        p.sub_(s["slopes"].reshape(1, kh, grp, 1, 1) * lines((j - s["pos"][..., None]).abs().float()))
    p = p.masked_fill_(lines(unseen), -math.inf).reshape(b, kh, grp * nq, nk)
    top = p.amax(-1, keepdim=True)
    p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = top + total.log()
    p.div_(total)
    o = p @ v
    out = {"o": rows(o, nq, a), "lse": lse.reshape(b, a, nq)}
    if c["kind"] == "span":
        return out
    do = heads(s["do"], nq)
    dv = p.transpose(2, 3) @ do
    ds = (do @ v.transpose(2, 3)).sub_((do * o).sum(-1, keepdim=True)).mul_(p).mul_(scale)
    if slope is not None:
        ds.mul_(slope)
    out.update(dq=rows(ds @ k, nq, a), dk=rows(ds.transpose(2, 3) @ q, nk, kh), dv=rows(dv, nk, kh))
    return out


# ---------------------------------------------------------------------------------------------------- what a pass needs
def work(case):
    """Every input read once, every output written once.  Where documents, lengths and tokens are drawn, what they come to on average."""
    c = case
    if c["kind"] in ("lookup", "embed"):
        T, V, h = float(c["T"]), float(c["V"]), c["h"]
        # tokens are log-uniform: number v has a share of 1 / (v ln V) of them, so these many different ones are among T
        kinds = float((1.0 - np.exp(-T / (np.arange(1.0, V + 1.0) * math.log(V)))).sum())
        n = 4.0 * T + 2.0 * kinds * h + 2.0 * T * h
        if c["kind"] == "lookup":
            return {"bytes": n, "flops": T * h}
        return {"bytes": n + 4.0 * T + 2.0 * T * h + (8.0 * kinds * h if c["add"] else 4.0 * V * h), "flops": 3.0 * T * h}
    if c["kind"] == "drop":
        n = float(c["T"]) * c["n"]
        return {"bytes": (4.0 + 2.0 * c["res"]) * n, "flops": 2.0 * n}
    if c["kind"] in ("scan", "recur"):
        n = float(c["batch"] * c["seq"]) * c["c"]
        live = 0.5 + 0.5 / c["batch"] if c["ragged"] else 1.0
        state = 4.0 * c["batch"] * c["c"]
        if c["kind"] == "scan":
            return {"bytes": (4.0 * live + 2.0) * n + state * (1 + c["state"]), "flops": 8.0 * n}
        return {"bytes": (10.0 * live + 6.0) * n + state * (1 + 3 * c["state"]), "flops": 24.0 * n}
    b, nq, nk, a, kh, d = [float(c[x]) for x in ("batch", "seq_q", "seq_kv", "a", "kh", "d")]
    if nq != nk:
        keys = nk + (b - 1.0) * 0.5 * (nk + nq)
        if c["window"]:
            keys = min(keys, b * (c["window"] + nq))
        pairs = nq * max(keys - 0.5 * b * nq, 0.5 * keys)
    else:
        keys, length = b * nk, nq / c["docs"]
        seen = nq / (c["docs"] + 1.0) * (1.0 + c["prefix"] / 12.0)          # keys of a query on average
        pairs = b * nq * (min(seen, max(c["window"] * (1.0 - 0.5 * c["window"] / length), 0.5 * c["window"])) if c["window"] else seen)
    if c["kind"] == "span":
        return {"bytes": 4.0 * (b * nq * a + keys * kh) * d + 4.0 * b * nq * (a + 2), "flops": 4.0 * pairs * a * d}
    return {"bytes": 2.0 * (6.0 * b * nq * a + 6.0 * keys * kh) * d + 8.0 * b * nq * a, "flops": 14.0 * pairs * a * d}


# ---------------------------------------------------------------------------------------------------- 64-bit definition
def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] in ("lookup", "embed"):
        live = torch.nonzero(s["ids"] >= 0)[:, 0]
        ids = s["ids"][live].long()
        x = torch.zeros((c["T"], c["h"]), dtype=F64, device=DEV)
        x[live] = c["scale"] * s["table"].double()[ids]
        if c["kind"] == "lookup":
            return x
        order = ids.argsort(stable=True)
        which, count = torch.unique_consecutive(ids[order], return_counts=True)
        dt = s["dtable"].double() if c["add"] else torch.zeros((c["V"], c["h"]), dtype=F64, device=DEV)
        ends = count.cumsum(0).tolist()
        rows = s["dx"].double()[live[order]]
        for v, n, e in zip(which.tolist(), count.tolist(), ends):
            dt[v] += c["scale"] * rows[e - n:e].sum(0)
        return {"x": x, "dtable": dt}
    if c["kind"] == "drop":
        keep = round((1.0 - float(np.float32(c["p"]))) * 65536)
        groups = np.arange(c["T"] * c["n"] // 8, dtype=np.uint64)
        low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
        ctr = [groups & low, groups >> half, np.full_like(groups, s["offset"] & 0xFFFFFFFF), np.full_like(groups, s["offset"] >> 32)]
        key = [s["seed"] & 0xFFFFFFFF, s["seed"] >> 32]
        for i in range(10):
            p, q = ctr[0] * np.uint64(0xD2511F53), ctr[2] * np.uint64(0xCD9E8D57)
            k = [np.uint64((key[0] + i * 0x9E3779B9) % (1 << 32)), np.uint64((key[1] + i * 0xBB67AE85) % (1 << 32))]
            ctr = [(q >> half) ^ ctr[1] ^ k[0], q & low, (p >> half) ^ ctr[3] ^ k[1], p & low]
        stay = np.stack([v for w in ctr for v in (w & np.uint64(0xFFFF), w >> np.uint64(16))], 1) < keep
        y = s["x"].double() * torch.from_numpy(stay.reshape(c["T"], c["n"])).to(DEV) * (65536.0 / keep)
        return y + s["res"].double() if c["res"] else y
    if c["kind"] in ("scan", "recur"):
        return _exact_scan(s, c)
    b, nq, nk, a, kh, d = [c[x] for x in ("batch", "seq_q", "seq_kv", "a", "kh", "d")]
    train = c["kind"] == "attend"
    q, k, v = [s[n].double().reshape(b, -1, s[n].shape[1], d) for n in ("q", "k", "v")]
    do = s["do"].double().reshape(q.shape) if train else None
    o, lse = torch.zeros_like(q), torch.full((b, a, nq), -math.inf, dtype=F64, device=DEV)
    dq, dk, dv = [torch.zeros_like(t) for t in (q, k, v)]
    at = torch.arange(nk, device=DEV)[None]
    for i in range(b):
        lo, hi, pos = s["span"][i, :, :1].long(), s["span"][i, :, 1:].long(), s["pos"][i, :, None].long()
        for first in range(0, nq, 4096):       # queries in pieces: 64 bits of all pairs of a long row would be large
            m = slice(first, min(first + 4096, nq))
            seen = (at >= lo[m]) & (at < hi[m])
            far = (at - pos[m]).abs().double() if c["bias"] else None
            for h in range(a):
                g = h // (a // kh)
                qh, kx, vx = [t.clone().requires_grad_(train) for t in (q[i, m, h], k[i, :, g], v[i, :, g])]
                sc = qh @ kx.t() / math.sqrt(d)
                if c["cap"]:
                    sc = c["cap"] * torch.tanh(sc / c["cap"])
                if c["bias"]:
                    sc = sc - s["slopes"][h].double() * far
                sc = sc.masked_fill(~seen, -math.inf)
                oh = sc.softmax(1) @ vx
                o[i, m, h], lse[i, h, m] = oh.detach(), torch.logsumexp(sc.detach(), 1)
                if train:
                    gq, gk, gv = torch.autograd.grad(oh, (qh, kx, vx), do[i, m, h])
                    dq[i, m, h] = gq
                    dk[i, :, g] += gk
                    dv[i, :, g] += gv
    got = {"o": o.reshape(-1, a, d), "lse": lse}
    if train:
        got.update(dq=dq.reshape(-1, a, d), dk=dk.reshape(-1, kh, d), dv=dv.reshape(-1, kh, d))
    return got


def _exact_scan(s, c):
    """Token by token, and back."""
    b, n, ch = c["batch"], c["seq"], c["c"]
    x, f = s["x"].double().reshape(b, n, ch), s["g"].double().reshape(b, n, ch).sigmoid()
    r = (-s["g"].double()).sigmoid().reshape(b, n, ch)
    w = [torch.ones_like(f), r, (r * (2.0 - r)).sqrt()][c["weight"]]
    h = s["h0"].double() if c["state"] else torch.zeros((b, ch), dtype=F64, device=DEV)
    length = s["len"].tolist() if c["ragged"] else [n] * b
    new = s["first"].tolist() if c["docs"] > 1 else [[0] * n] * b
    keep = torch.tensor([[0.0 if new[i][t] else 1.0 for t in range(n)] for i in range(b)], dtype=F64, device=DEV)[..., None]
    on = torch.tensor([[1.0 if t < length[i] else 0.0 for t in range(n)] for i in range(b)], dtype=F64, device=DEV)[..., None]
    before, y = torch.empty_like(x), torch.empty_like(x)
    fk, wx = f * keep, w * x
    for t in range(n):
        before[:, t] = h * keep[:, t]
        h = torch.lerp(h, torch.addcmul(wx[:, t], fk[:, t], h), on[:, t])
        y[:, t] = h * on[:, t]
    got = {"y": y.reshape(-1, ch), "last": h}
    if c["kind"] == "scan":
        return got
    dy = s["dy"].double().reshape(b, n, ch) * on
    back = s["dlast"].double() if c["state"] else torch.zeros_like(h)
    lam = torch.empty_like(x)
    for t in range(n - 1, -1, -1):
        back = back + dy[:, t]
        lam[:, t] = back * on[:, t]
        back = torch.lerp(back, fk[:, t] * back, on[:, t])
    # w as a function of f: 1, 1 - f, sqrt(1 - f^2); df / dg = f (1 - f)
    dw_df = [torch.zeros_like(f), -torch.ones_like(f), -f / w][c["weight"]]
    got.update(dx=(lam * w).reshape(-1, ch), dg=(lam * (before + x * dw_df) * f * r).reshape(-1, ch))
    if c["state"]:
        got["dh0"] = back
    return got

"""What the speed of the single operators beside the stage calls is measured on: rotary positions in other layouts and scalings,
cross attention, and the balance loss of a mixture's router.

A case is one pass through one operator on inputs that are already on the GPU:

  table    rp_op_rope_table_scaled   the (cos, sin) table of scaled rotary positions
  rope     rp_op_rope                rotation of the query and key heads, or (bwd) of their gradients
  cross    rp_op_cross_attn_fwd      attention of every query to another sequence's keys: output, log-sum-exp
  train    rp_op_cross_attn_fwd, _bwd: the same, and dq, dk, dv
  balance  rp_op_moe_balance         loss, counts and the gradient of the router logits, alone or added to what the layer left

With `own` false the same results come from elementary torch operations in 32 bits (64 for the angles and the long sums).
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
BF16, F32, F64, I32 = torch.bfloat16, torch.float32, torch.float64, torch.int32
PLAIN, LINEAR, BASE, PARTS = 0, 1, 2, 3      # kinds of scaling


def _scaling(kind, factor=1.0, base=1.0e6, trained=4096, amplitude=1.0):
    return dict(scaling=kind, factor=factor, base=base, trained=trained, slow=1.0, fast=32.0, amplitude=amplitude)


def listed():
    return [
        # a program's own table for ordinary training lengths, and the table of a model whose context was extended 32 times
        dict(name="table_2048", kind="table", n_pos=2048, rot=64, **_scaling(LINEAR, 4.0)),
        dict(name="table_131072", kind="table", n_pos=131072, rot=128, **_scaling(PARTS, 32.0, amplitude=1.34657)),
        # eight sequences that each add one token, at positions of their own: launch and latency
        dict(name="rope_token_8", kind="rope", bwd=0, layout=1, d=128, rot=128, a=16, kh=8, batch=8, seq=1, given=1, n_pos=4096, **_scaling(PLAIN)),
        # a long document through a wide layer, extended by parts
        dict(name="rope_half_16384", kind="rope", bwd=0, layout=0, d=128, rot=128, a=64, kh=8, batch=1, seq=16384, given=0, n_pos=16384,
             **_scaling(PARTS, 4.0, amplitude=1.13863)),
        # the gradient of neighbouring pairs over half of a narrow head, sequences of an odd length
        dict(name="rope_part_bwd_4x1021", kind="rope", bwd=1, layout=1, d=64, rot=32, a=64, kh=8, batch=4, seq=1021, given=0, n_pos=1021, **_scaling(PLAIN)),
        # generation: eight sequences, one new token each, encoder states of different lengths
        dict(name="cross_token_8x1500", kind="cross", batch=8, seq_q=1, seq_kv=1500, a=16, kh=8, d=128, ragged=1),
        # generation from a long document: few rows, the keys are all there is to read
        dict(name="cross_token_2x32768", kind="cross", batch=2, seq_q=1, seq_kv=32768, a=64, kh=8, d=128, ragged=0),
        # training on a padded batch, narrow heads, no length a multiple of a tile
        dict(name="train_4x509x1500", kind="train", batch=4, seq_q=509, seq_kv=1500, a=64, kh=8, d=64, ragged=2),
        # training on a long text beside a longer source: the largest case
        dict(name="train_4096x8192", kind="train", batch=1, seq_q=4096, seq_kv=8192, a=32, kh=8, d=128, ragged=0),
        # the router of a small layer in a short batch: launches
        dict(name="balance_256x32", kind="balance", T=256, seq=256, E=32, top_k=4, masked=0, z=0.0, add=0),
        # a padded batch, balanced sequence by sequence, on top of the gradient that the layer has left
        dict(name="balance_4x1001x256", kind="balance", T=4004, seq=1001, E=256, top_k=8, masked=1, z=1.0e-3, add=1),
        # the longest step of the widest mixture
        dict(name="balance_31744x128", kind="balance", T=31744, seq=31744, E=128, top_k=8, masked=0, z=1.0e-3, add=1),
    ]


HEADS = ((4, 2), (16, 8), (16, 16), (32, 8), (64, 8), (64, 4))


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    kind = rng.choice(("table", "rope", "rope", "rope", "cross", "cross", "train", "train", "train", "balance", "balance"))
    how = rng.choice((PLAIN, LINEAR, BASE, PARTS))
    scaling = _scaling(how, 1.0 if how == PLAIN else rng.choice((2.0, 4.0, 8.0, 32.0)), rng.choice((1.0e4, 5.0e5, 1.0e6)), rng.choice((2048, 4096, 8192)),
                       rng.choice((1.0, 1.13863)) if how == PARTS else 1.0)
    if kind == "table":
        return dict(kind=kind, n_pos=_log(rng, 16, 131072), rot=2 * rng.randint(2, 64), **scaling)
    if kind == "rope":
        d = rng.choice((64, 80, 96, 128, 128, 256))
        a, kh = rng.choice(HEADS)
        batch, bwd, layout, given = rng.choice((1, 1, 2, 3, 8)), rng.randint(0, 1), rng.randint(0, 1), rng.randint(0, 1)
        seq = _log(rng, 1, max(1, int(16384 * 72 * 128 / ((a + kh) * d * batch))))
        rot = rng.choice((d, d, d // 2, d // 4, 2 * rng.randint(2, d // 2)))
        return dict(kind=kind, bwd=bwd, layout=layout, d=d, rot=rot, a=a, kh=kh, batch=batch, seq=seq, given=given,
                    n_pos=max(seq, _log(rng, 1, 32768)) if given else seq, **scaling)
    if kind in ("cross", "train"):
        a, kh = rng.choice(HEADS)
        d, ragged = rng.choice((64, 128, 128)), rng.randint(0, 2)
        most = 32 * 4096 * 8192 * 128 // (a * d)              # batch * seq_q * seq_kv
        batch = rng.choice((1, 1, 2, 4, 8))
        seq_q = _log(rng, 1, 4096)
        if kind == "cross" and rng.random() < 0.5:
            seq_q = rng.choice((1, 1, 2, 5, 17))
        seq_kv = _log(rng, 1, max(1, min(32768, most // (batch * seq_q))))
        if kind == "train":      # (the gradients of a softmax over one key are zero: nothing to compare)
            seq_kv = max(4, min(8192, seq_kv))
        return dict(kind=kind, batch=batch, seq_q=seq_q, seq_kv=seq_kv, a=a, kh=kh, d=d, ragged=ragged)
    E = rng.choice((8, 32, 60, 128, 160, 256, 1024))
    groups = rng.choice((1, 1, 1, 2, 4, 7))
    seq = _log(rng, 1, 31744 * 128 // max(E, 128) // groups)
    return dict(kind=kind, T=groups * seq, seq=seq, E=E, top_k=rng.choice((1, 2, 4) if E == 8 else (1, 2, 4, 8)), masked=rng.randint(0, 1), z=rng.choice((0.0, 1.0e-3)), add=rng.randint(0, 1))


# ---------------------------------------------------------------------------------------------------- inputs
COEF, GRAD = 1.0e-2, 0.5        # weight of the balance loss, and the scale that its gradient arrives with


def _frequencies(c):
    """[rot / 2] in 64 bits, on the GPU."""
    i = torch.arange(0, c["rot"], 2, dtype=F64, device=DEV) / c["rot"]
    if c["scaling"] == BASE:
        return (c["base"] * c["factor"] ** (c["rot"] / (c["rot"] - 2.0))) ** -i
    th = c["base"] ** -i
    if c["scaling"] == LINEAR:
        return th / c["factor"]
    if c["scaling"] == PARTS:
        keep = ((c["trained"] * th / (2.0 * math.pi) - c["slow"]) / (c["fast"] - c["slow"])).clamp(0.0, 1.0)
        return th * (keep + (1.0 - keep) / c["factor"])
    return th


def _table(c):
    ang = torch.arange(c["n_pos"], dtype=F64, device=DEV)[:, None] * _frequencies(c)
    return torch.stack((ang.cos(), ang.sin()), -1).mul_(c["amplitude"]).to(F32)


def _lengths(g, batch, longest, least):
    """Lengths of a padded batch: the longest fills it, the others are spread."""
    n = torch.randint(least, longest + 1, (batch,), generator=g, device=DEV, dtype=I32)
    n[0] = longest
    return n


def prepare(case, seed):
    c, g = case, torch.Generator(device=DEV).manual_seed(seed)

    def normal(*shape, std=1.0, dtype=BF16):
        return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, std, generator=g)

    s = {"case": c, "stream": torch.cuda.current_stream().cuda_stream}
    if c["kind"] == "table":
        # the table depends on the case alone; the base is a model's own and varies with it
        s["base"] = float(np.float32(c["base"] * (1.0 + 1.0e-3 * (seed % 997))))
        s["cs"] = torch.empty((c["n_pos"], c["rot"] // 2, 2), dtype=F32, device=DEV)
        return s
    if c["kind"] == "rope":
        T, a, kh, d = c["batch"] * c["seq"], c["a"], c["kh"], c["d"]
        s["q"], s["k"] = normal(T, a, d), normal(T, kh, d)
        s["oq"], s["ok"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
        s["cs"] = _table(c)
        s["pos"] = None
        if c["given"]:      # every sequence goes on from where its own past ends
            start = torch.randint(0, c["n_pos"] - c["seq"] + 1, (c["batch"], 1), generator=g, device=DEV, dtype=I32)
            s["pos"] = (start + torch.arange(c["seq"], dtype=I32, device=DEV)).reshape(-1)
        return s
    if c["kind"] == "balance":
        T, E, G = c["T"], c["E"], c["T"] // c["seq"]
        # a router in training: some experts are preferred by all tokens
        s["logits"] = normal(T, E, std=1.5, dtype=F32) + normal(E, std=0.7, dtype=F32)
        s["idx"] = s["logits"].topk(c["top_k"], 1).indices.to(I32)
        s["mask"] = None
        if c["masked"]:     # padding behind every sequence
            n = _lengths(g, G, c["seq"], 0)
            s["mask"] = (torch.arange(c["seq"], device=DEV)[None] < n[:, None]).reshape(-1).to(torch.uint8)
        s["given"] = normal(T, E, std=1.0e-4, dtype=F32)
        s["dlogits"] = torch.empty_like(s["logits"])
        s["counts"] = torch.empty((G, E), dtype=I32, device=DEV)
        s["tokens"] = torch.empty(G + 1, dtype=I32, device=DEV)
        s["loss"] = torch.empty(3, dtype=F32, device=DEV)
        return s
    b, nq, nk, a, kh, d = [c[x] for x in ("batch", "seq_q", "seq_kv", "a", "kh", "d")]
    s["q"], s["k"], s["v"] = normal(b * nq, a, d, std=2.0), normal(b * nk, kh, d), normal(b * nk, kh, d)
    s["kv_len"] = _lengths(g, b, nk, 0) if c["ragged"] else None
    s["q_len"] = _lengths(g, b, nq, 1) if c["ragged"] == 2 else None
    s["o"] = torch.empty_like(s["q"])
    s["lse"] = torch.empty((b, a, nq), dtype=F32, device=DEV)
    if c["kind"] == "train":
        s["do"] = normal(b * nq, a, d)
        s["dq"], s["dk"], s["dv"] = [torch.empty_like(s[n]) for n in ("q", "k", "v")]
        s["delta"] = torch.empty_like(s["lse"])
    return s


# ---------------------------------------------------------------------------------------------------- one pass
def run(state):
    return _own(state) if own else _plain(state)


def _own(s):
    from paper_2604_27085_amd import binding as B
    c, st = s["case"], s["stream"]
    if c["kind"] == "table":
        sc = B.make_rope_scaling(c["scaling"], s["base"], c["factor"], c["slow"], c["fast"], c["trained"], c["amplitude"])
        B.rp_op_rope_table_scaled(st, s["cs"], sc, c["n_pos"], c["rot"])
        return s["cs"]
    if c["kind"] == "rope":
        a, kh, d = c["a"], c["kh"], c["d"]
        B.rp_op_rope(st, c["bwd"], c["layout"], d, c["rot"], s["q"], s["k"], a * d, kh * d, s["oq"], s["ok"], a * d, kh * d, s["cs"], c["n_pos"], s["pos"],
                     c["batch"] * c["seq"], c["seq"], a, kh)
        return {"q": s["oq"], "k": s["ok"]}
    if c["kind"] == "balance":
        if "scratch" not in s:
            s["scratch"] = torch.empty(B.rp_op_moe_balance_scratch(c["T"], c["seq"], c["E"]), dtype=torch.uint8, device=DEV)
        B.rp_op_moe_balance(st, s["logits"], s["idx"], s["mask"], c["T"], c["seq"], c["E"], c["top_k"], COEF, c["z"], GRAD, s["counts"], s["tokens"], s["loss"],
                            s["given"] if c["add"] else None, s["dlogits"], s["scratch"])
        return {"loss": s["loss"], "counts": s["counts"], "tokens": s["tokens"], "dlogits": s["dlogits"]}
    b, nq, nk, a, kh, d = [c[x] for x in ("batch", "seq_q", "seq_kv", "a", "kh", "d")]
    if "scratch" not in s:      # a program asks once and keeps it
        fwd, bwd = B.rp_op_cross_attn_scratch(b, nq, nk, a, kh, d)
        s["scratch"] = torch.empty(max(fwd, bwd if c["kind"] == "train" else 0, 16), dtype=torch.uint8, device=DEV)
    qd, kd, scale = a * d, kh * d, d ** -0.5
    B.rp_op_cross_attn_fwd(st, s["q"], s["k"], s["v"], s["o"], s["lse"], qd, kd, kd, qd, s["q_len"], s["kv_len"], b, nq, nk, a, kh, d, scale, s["scratch"])
    if c["kind"] == "cross":
        return {"o": s["o"], "lse": s["lse"]}
    B.rp_op_cross_attn_bwd(st, s["q"], s["k"], s["v"], s["o"], s["do"], s["lse"], s["delta"], s["dq"], s["dk"], s["dv"], qd, kd, kd, qd, qd, qd, kd, kd,
                           s["q_len"], s["kv_len"], b, nq, nk, a, kh, d, scale, s["scratch"])
    return {n: s[n] for n in ("o", "lse", "dq", "dk", "dv")}


def _rotate(x, c, cs):
    """x [T, heads, d] and cs [T, rot / 2, 2] in 32 bits."""
    rot = c["rot"]
    co, si = cs[:, None, :, 0], cs[:, None, :, 1]
    if c["bwd"]:
        si = -si
    x = x.float()
    if c["layout"]:
        x1, x2 = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack((x1 * co - x2 * si, x2 * co + x1 * si), -1).flatten(-2)
    else:
        x1, x2 = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat((x1 * co - x2 * si, x2 * co + x1 * si), -1)
    return torch.cat((y, x[..., rot:]), -1).to(BF16)


def _plain(s):
    c = s["case"]
    if c["kind"] == "table":
        return _table(dict(c, base=s["base"]))
    if c["kind"] == "rope":
        pos = s["pos"].long() if c["given"] else torch.arange(c["seq"], device=DEV).repeat(c["batch"])
        cs = s["cs"][pos]
        return {"q": _rotate(s["q"], c, cs), "k": _rotate(s["k"], c, cs)}
    if c["kind"] == "balance":
        return _plain_balance(s, c)
    return _plain_attention(s, c)


def _plain_balance(s, c):
    T, n, E, G = c["T"], c["seq"], c["E"], c["T"] // c["seq"]
    m = s["mask"].float() if c["masked"] else torch.ones(T, device=DEV)
    lse = torch.logsumexp(s["logits"], 1)
    p = (s["logits"] - lse[:, None]).exp() * m[:, None]
    group = torch.arange(G, device=DEV).repeat_interleave(n)[:, None].expand(-1, c["top_k"])
    counts = torch.zeros((G, E), dtype=F64, device=DEV).index_put_((group, s["idx"].long()), m.double()[:, None].expand(-1, c["top_k"]), accumulate=True)
    tokens = m.double().reshape(G, n).sum(1)
    N = tokens.sum()
    per = 1.0 / N.clamp(min=1.0)
    f = counts / (tokens.clamp(min=1.0) * c["top_k"])[:, None]
    bal = E * per * (f * p.double().reshape(G, n, E).sum(1)).sum()
    z = per * (m.double() * torch.where(m > 0, lse, 0.0).double().square()).sum()
    f = f.float()[:, None]
    pg = p.reshape(G, n, E)
    grad = (COEF * E * per).float() * pg * (f - (f * p.reshape(G, n, E)).sum(-1, keepdim=True))
    if c["z"]:
        grad = grad + (2.0 * c["z"] * per).float() * lse.reshape(G, n, 1) * pg
    grad = GRAD * grad.reshape(T, E)
    if c["add"]:
        grad = s["given"] + grad
    return {"loss": torch.stack((COEF * bal + c["z"] * z, bal, z)).float(), "counts": counts.to(I32), "tokens": torch.cat((tokens, N[None])).to(I32),
            "dlogits": grad}


def _plain_attention(s, c):
    b, nq, nk, a, kh, d = [c[x] for x in ("batch", "seq_q", "seq_kv", "a", "kh", "d")]
    scale, grp = d ** -0.5, a // kh

    def heads(t, n):      # [b * n, heads, d] -> [b, kh, heads / kh * n, d]
        return t.float().reshape(b, n, kh, -1, d).permute(0, 2, 3, 1, 4).reshape(b, kh, -1, d)

    def rows(t, n, h):
        return t.reshape(b, kh, h // kh, n, d).permute(0, 3, 1, 2, 4).reshape(b * n, h, d).to(BF16)

    q, k, v = heads(s["q"], nq), heads(s["k"], nk), heads(s["v"], nk)
    p = (q @ k.transpose(2, 3)).mul_(scale)
    live = None
    if c["ragged"]:
        p.masked_fill_((torch.arange(nk, device=DEV)[None] >= s["kv_len"][:, None])[:, None, None], -math.inf)
        live = (s["kv_len"] > 0)[:, None].expand(b, nq)
        if s["q_len"] is not None:
            live = live & (torch.arange(nq, device=DEV)[None] < s["q_len"][:, None])
        live = live[:, None, None].expand(b, 1, grp, nq).reshape(b, 1, grp * nq, 1)
    top = p.amax(-1, keepdim=True)
    if live is not None:
        top = torch.where(live, top, 0.0)
    p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = top + total.log()
    if live is not None:
        total, lse = torch.where(live, total, math.inf), torch.where(live, lse, -math.inf)
    p.div_(total)
    o = p @ v
    if live is not None:
        o = torch.where(live, o, 0.0)
    out = {"o": rows(o, nq, a), "lse": lse.reshape(b, kh, grp, nq).reshape(b, a, nq)}
    if c["kind"] == "cross":
        return out
    do = heads(s["do"], nq)
    if live is not None:
        do = torch.where(live, do, 0.0)
    dv = p.transpose(2, 3) @ do
    ds = (do @ v.transpose(2, 3)).sub_((do * o).sum(-1, keepdim=True)).mul_(p).mul_(scale)
    out.update(dq=rows(ds @ k, nq, a), dk=rows(ds.transpose(2, 3) @ q, nk, kh), dv=rows(dv, nk, kh))
    return out


# ---------------------------------------------------------------------------------------------------- what a pass needs
def work(case):
    """Every input read once, every output written once.  Padded batches count what the lengths leave on average: prepare() fills the
    first sequence and spreads the others evenly."""
    c = case
    if c["kind"] == "table":
        n = c["n_pos"] * (c["rot"] // 2)
        return {"bytes": 8.0 * n, "flops": 20.0 * n}
    if c["kind"] == "rope":
        n = float(c["batch"] * c["seq"]) * (c["a"] + c["kh"])
        return {"bytes": 4.0 * n * c["d"] + 4.0 * min(c["n_pos"], c["batch"] * c["seq"]) * c["rot"], "flops": 3.0 * n * c["rot"]}
    if c["kind"] == "balance":
        n = float(c["T"]) * c["E"]
        return {"bytes": 4.0 * n * (2.0 + c["add"]) + 4.0 * c["T"] * c["top_k"], "flops": 12.0 * n}
    b, nq, nk, a, kh, d = [c[x] for x in ("batch", "seq_q", "seq_kv", "a", "kh", "d")]
    keys = nk * (1.0 + 0.5 * (b - 1)) if c["ragged"] else float(b * nk)
    pairs = nq * keys
    if c["ragged"] == 2:
        pairs = nq * nk * (1.0 + 0.25 * (b - 1))
    if c["kind"] == "cross":
        return {"bytes": 4.0 * (b * nq * a + keys * kh) * d + 4.0 * b * nq * a, "flops": 4.0 * pairs * a * d}
    return {"bytes": 2.0 * (6.0 * b * nq * a + 4.0 * keys * kh + 2.0 * b * nk * kh) * d + 8.0 * b * nq * a, "flops": 14.0 * pairs * a * d}


# ---------------------------------------------------------------------------------------------------- 64-bit definition
def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] in ("table", "rope"):
        i = np.arange(c["rot"] // 2, dtype=np.float64)
        base = s.get("base", c["base"])
        if c["scaling"] == BASE:
            base = base * np.power(c["factor"], c["rot"] / (c["rot"] - 2.0))
        turn = np.exp(-2.0 * i / c["rot"] * np.log(base))            # radians a position
        if c["scaling"] == LINEAR:
            turn = turn / c["factor"]
        if c["scaling"] == PARTS:
            turns = c["trained"] * turn / (2.0 * np.pi)              # over the trained length
            share = np.clip((turns - c["slow"]) / (c["fast"] - c["slow"]), 0.0, 1.0)
            turn = share * turn + (1.0 - share) * turn / c["factor"]
        turn = torch.from_numpy(turn).to(DEV)
    if c["kind"] == "table":
        z = torch.polar(torch.full((), c["amplitude"], dtype=F64, device=DEV), torch.outer(torch.arange(c["n_pos"], dtype=F64, device=DEV), turn))
        return torch.view_as_real(z)
    if c["kind"] == "rope":
        pos = s["pos"].double() if c["given"] else torch.arange(c["batch"] * c["seq"], dtype=F64, device=DEV).remainder_(c["seq"])
        z = torch.polar(torch.full((), c["amplitude"], dtype=F64, device=DEV), torch.outer(pos, -turn if c["bwd"] else turn))[:, None]
        got = {}
        for name in ("q", "k"):
            x = s[name].double()
            pairs = x[..., :c["rot"]].reshape(x.shape[0], x.shape[1], *((-1, 2) if c["layout"] else (2, -1)))
            pairs = pairs if c["layout"] else pairs.transpose(2, 3)
            y = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * z)
            x[..., :c["rot"]] = (y if c["layout"] else y.transpose(2, 3)).reshape(x.shape[0], x.shape[1], c["rot"])
            got[name] = x
        return got
    if c["kind"] == "balance":
        x = s["logits"].double().requires_grad_()
        keep = s["mask"].bool() if c["masked"] else torch.ones(c["T"], dtype=torch.bool, device=DEV)
        N = keep.sum().clamp(min=1)
        bal, z = x.sum() * 0.0, torch.where(keep, torch.logsumexp(x, 1), 0.0).square().sum() / N
        for g in range(c["T"] // c["seq"]):
            at = torch.arange(g * c["seq"], (g + 1) * c["seq"], device=DEV)[keep[g * c["seq"]:(g + 1) * c["seq"]]]
            if at.numel():
                share = torch.bincount(s["idx"][at].reshape(-1).long(), minlength=c["E"]).double() / (at.numel() * c["top_k"])
                bal = bal + c["E"] * (share * x[at].softmax(1).mean(0)).sum() * at.numel() / N
        loss = COEF * bal + c["z"] * z
        grad = GRAD * torch.autograd.grad(loss, x)[0]
        return {"loss": torch.stack((loss, bal, z)).detach(), "counts": None, "tokens": None, "dlogits": grad + s["given"].double() if c["add"] else grad}
    b, nq, nk, a, kh, d = [c[x] for x in ("batch", "seq_q", "seq_kv", "a", "kh", "d")]
    q, k, v = [s[n].double().reshape(b, -1, s[n].shape[1], d) for n in ("q", "k", "v")]
    do = s["do"].double().reshape(q.shape) if c["kind"] == "train" else None
    o, lse = torch.zeros_like(q), torch.full((b, a, nq), -math.inf, dtype=F64, device=DEV)
    dq, dk, dv = [torch.zeros_like(t) for t in (q, k, v)]
    q_len = s["q_len"].tolist() if s["q_len"] is not None else [nq] * b
    kv_len = s["kv_len"].tolist() if s["kv_len"] is not None else [nk] * b
    for i in range(b):
        m, n = q_len[i], kv_len[i]
        for h in range(a if n else 0):
            part = [q[i, :m, h], k[i, :n, h // (a // kh)], v[i, :n, h // (a // kh)]]
            qh, kx, vx = [t.clone().requires_grad_(do is not None) for t in part]
            sc = (qh @ kx.t()) / math.sqrt(d)
            oh = sc.softmax(1) @ vx
            o[i, :m, h], lse[i, h, :m] = oh.detach(), torch.logsumexp(sc.detach(), 1)
            if do is not None:
                gq, gk, gv = torch.autograd.grad(oh, (qh, kx, vx), do[i, :m, h])
                dq[i, :m, h] = gq
                dk[i, :n, h // (a // kh)] += gk
                dv[i, :n, h // (a // kh)] += gv
    got = {"o": o.reshape(-1, a, d), "lse": lse}
    if do is not None:
        got.update(dq=dq.reshape(-1, a, d), dk=dk.reshape(-1, kh, d), dv=dv.reshape(-1, kh, d))
    return got

"""The layer operators run together, as a decoder layer with cross attention and a mixture's router would: norm, projections, rotary positions, cross
attention, routing and balance loss, forward and backward, against the same layer in 64 bits; and captured into a graph."""
import math

import pytest

import ops_reference as R

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"
BF16, F64 = torch.bfloat16, torch.float64


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2604_27085_amd import binding
    return binding


def rel_l2(a, b):
    return float((a.double() - b).norm() / b.norm())


class Layer:
    """y = x + rmsnorm -> q -> rotate -> cross attention (keys: projected and rotated encoder states) -> output projection;  router logits = rmsnorm(y) Wr^T
    -> top-k -> balance loss.  The gradient of sum(y * dy) + the balance loss."""

    def __init__(self, b=2, nq=40, nk=72, h=256, a=8, kh=2, d=64, E=16, top_k=2, rot=32, layout=1):
        self.dims = (b, nq, nk, h, a, kh, d, E, top_k, rot, layout)
        g = torch.Generator(device=DEV).manual_seed(11)
        rnd = lambda *s, std=1.0: (std * torch.randn(s, generator=g, device=DEV)).to(BF16)  # noqa: E731
        self.x, self.enc, self.dy = rnd(b * nq, h), rnd(b * nk, h), rnd(b * nq, h, std=0.1)
        self.g1, self.g2 = [(1 + 0.1 * torch.randn(h, generator=g, device=DEV)).to(BF16) for _ in range(2)]
        self.wq, self.wk, self.wv, self.wo, self.wr = rnd(a * d, h, std=0.1), rnd(kh * d, h, std=0.1), rnd(kh * d, h, std=0.06), rnd(h, a * d, std=0.06), rnd(E, h, std=0.1)
        self.kv_len = torch.tensor([nk, nk - 29][:b], dtype=torch.int32, device=DEV)
        self.pos = (torch.arange(nq, dtype=torch.int32, device=DEV) + 5).repeat(b)
        e = lambda *s, t=BF16: torch.empty(s, dtype=t, device=DEV)  # noqa: E731
        T, S, f32 = b * nq, b * nk, torch.float32
        self.n1, self.q, self.k, self.v, self.o, self.y, self.n2 = e(T, h), e(T, a * d), e(S, kh * d), e(S, kh * d), e(T, a * d), e(T, h), e(T, h)
        self.r1, self.r2, self.lse, self.delta = e(T, t=f32), e(T, t=f32), e(b, a, nq, t=f32), e(b, a, nq, t=f32)
        self.logits, self.dlogits, self.loss = e(T, E, t=f32), e(T, E, t=f32), e(3, t=f32)
        self.dn2, self.dyt, self.do, self.dq, self.dk, self.dv, self.dn1, self.dx, self.denc = (e(T, h), e(T, h), e(T, a * d), e(T, a * d), e(S, kh * d), e(S, kh * d),
                                                                                          e(T, h), e(T, h), e(S, h))
        self.dlog16 = e(T, E)
        i32 = lambda *s: torch.empty(s, dtype=torch.int32, device=DEV)  # noqa: E731
        n = T * top_k
        self.route = dict(idx=i32(T, top_k), w=e(T, top_k, t=f32), counts=i32(E), seg=i32(E + 1), tab=i32(4 * (n // 256 + E + 1)), nt=i32(1), slot=i32(n), tok=i32(n),
                          hist=i32((n + 511) // 512 * E))
        self.counts, self.tokens = i32(b, E), i32(b + 1)
        self.cs = e(nq + nk + 8, rot // 2, 2, t=f32)
        self.ws = None

    def run(self, B):
        b, nq, nk, h, a, kh, d, E, top_k, rot, layout = self.dims
        T, S, qd, kd, st = b * nq, b * nk, a * d, kh * d, torch.cuda.current_stream().cuda_stream
        if self.ws is None:
            self.ws = torch.empty(max(*B.rp_op_cross_attn_scratch(b, nq, nk, a, kh, d), 16), dtype=torch.uint8, device=DEV)
            self.bws = torch.empty(B.rp_op_moe_balance_scratch(T, nq, E), dtype=torch.uint8, device=DEV)
        nt = lambda x, w, y, m, n, k, **kw: B.rp_op_gemm(st, 0, 0, x, w, y, m, n, k, k, k, n, **kw)  # noqa: E731
        nn = lambda x, w, y, m, n, k, **kw: B.rp_op_gemm(st, 1, 0, x, w, y, m, n, k, k, n, n, **kw)  # noqa: E731
        B.rp_op_rope_table_scaled(st, self.cs, B.make_rope_scaling(B.ROPE_BY_PARTS, 1.0e4, 4.0, 1.0, 8.0, 64, 1.1), self.cs.shape[0], rot)
        B.rp_op_rmsnorm_fwd(st, self.x, self.g1, self.n1, self.r1, T, h, 1e-6)
        nt(self.n1, self.wq, self.q, T, qd, h)
        nt(self.enc, self.wk, self.k, S, kd, h)
        nt(self.enc, self.wv, self.v, S, kd, h)
        B.rp_op_rope(st, 0, layout, d, rot, self.q, None, qd, 0, self.q, None, qd, 0, self.cs, self.cs.shape[0], self.pos, T, nq, a, 0)      # in place
        B.rp_op_rope(st, 0, layout, d, rot, None, self.k, 0, kd, None, self.k, 0, kd, self.cs, self.cs.shape[0], None, S, nk, 0, kh)
        args = (None, self.kv_len, b, nq, nk, a, kh, d, d ** -0.5, self.ws)
        B.rp_op_cross_attn_fwd(st, self.q, self.k, self.v, self.o, self.lse, qd, kd, kd, qd, *args)
        nt(self.o, self.wo, self.y, T, h, qd, R=self.x, ldr=h)
        B.rp_op_rmsnorm_fwd(st, self.y, self.g2, self.n2, self.r2, T, h, 1e-6)
        B.rp_op_gemm(st, 0, 1, self.n2, self.wr, self.logits, T, E, h, h, h, E)
        r = self.route
        B.rp_op_moe_route_plan(st, self.logits, T, E, top_k, r["idx"], r["w"], r["counts"], r["seg"], r["tab"], r["nt"], r["slot"], r["tok"], r["hist"])
        B.rp_op_moe_balance(st, self.logits, r["idx"], None, T, nq, E, top_k, 0.5, 0.05, 1.0, self.counts, self.tokens, self.loss, None, self.dlogits, self.bws)
        # backward
        self.dlog16.copy_(self.dlogits)
        nn(self.dlog16, self.wr, self.dn2, T, h, E)
        B.rp_op_rmsnorm_bwd(st, self.dn2, 0, self.y, self.g2, self.r2, self.dy, self.dyt, None, None, T, h)
        nn(self.dyt, self.wo, self.do, T, qd, h)
        B.rp_op_cross_attn_bwd(st, self.q, self.k, self.v, self.o, self.do, self.lse, self.delta, self.dq, self.dk, self.dv, qd, kd, kd, qd, qd, qd, kd, kd, *args)
        B.rp_op_rope(st, 1, layout, d, rot, self.dq, None, qd, 0, self.dq, None, qd, 0, self.cs, self.cs.shape[0], self.pos, T, nq, a, 0)
        B.rp_op_rope(st, 1, layout, d, rot, None, self.dk, 0, kd, None, self.dk, 0, kd, self.cs, self.cs.shape[0], None, S, nk, 0, kh)
        nn(self.dq, self.wq, self.dn1, T, h, qd)
        B.rp_op_rmsnorm_bwd(st, self.dn1, 0, self.x, self.g1, self.r1, self.dyt, self.dx, None, None, T, h)
        B.rp_op_gemm(st, 1, 0, self.dk, self.wk, self.denc, S, h, kd, kd, h, h, A2=self.dv, B2=self.wv, K2=kd, lda2=kd, ldb2=h)

    def results(self):
        return {n: getattr(self, n) for n in ("y", "logits", "loss", "counts", "dx", "denc", "dq", "dk", "dv", "lse")}

    def reference(self):
        b, nq, nk, h, a, kh, d, E, top_k, rot, layout = self.dims
        x, enc = [t.double().cpu().requires_grad_() for t in (self.x, self.enc)]
        w = {n: getattr(self, n).double().cpu() for n in ("wq", "wk", "wv", "wo", "wr", "g1", "g2", "dy")}
        rms = lambda t, g: t * torch.rsqrt(t.square().mean(-1, keepdim=True) + 1e-6) * g  # noqa: E731
        ang = torch.arange(self.cs.shape[0], dtype=F64)[:, None] * R.frequencies(3, 1.0e4, 4.0, 1.0, 8.0, 64, rot)
        cs = float(torch.tensor(1.1, dtype=torch.float32)) * torch.stack((ang.cos(), ang.sin()), -1)

        def turn(t, heads, pos):
            t = t.reshape(-1, heads, d)
            c, s = cs[pos][:, None, :, 0], cs[pos][:, None, :, 1]
            u, v = (t[..., 0:rot:2], t[..., 1:rot:2]) if layout else (t[..., :rot // 2], t[..., rot // 2:rot])
            p = torch.stack((u * c - v * s, v * c + u * s), -1)
            p = p.flatten(-2) if layout else p.transpose(-1, -2).flatten(-2)
            return torch.cat((p, t[..., rot:]), -1)

        q = turn(rms(x, w["g1"]) @ w["wq"].t(), a, self.pos.cpu().long()).reshape(b, nq, a, d)
        k = turn(enc @ w["wk"].t(), kh, torch.arange(nk).repeat(b)).reshape(b, nk, kh, d)
        v = (enc @ w["wv"].t()).reshape(b, nk, kh, d)
        outs = []
        for i in range(b):
            n = int(self.kv_len[i])
            outs.append(torch.stack([((q[i, :, j] @ k[i, :n, j // (a // kh)].t()) / math.sqrt(d)).softmax(1) @ v[i, :n, j // (a // kh)] for j in range(a)], 1))
        y = x + torch.cat(outs).reshape(b * nq, a * d) @ w["wo"].t()
        logits = rms(y, w["g2"]) @ w["wr"].t()
        idx = self.route["idx"].cpu().long()      # the choices that were made: a bf16 step of the logits may turn a close one
        p = logits.softmax(1)
        loss_b = 0.0
        counts = torch.zeros((b, E), dtype=torch.int64)
        for i in range(b):
            sl = slice(i * nq, (i + 1) * nq)
            counts[i] = torch.bincount(idx[sl].reshape(-1), minlength=E)
            loss_b = loss_b + E * ((counts[i].double() / (nq * top_k)) * p[sl].mean(0)).sum() / b
        loss_z = torch.logsumexp(logits, 1).square().mean()
        total = 0.5 * loss_b + 0.05 * loss_z
        dx, denc = torch.autograd.grad((y * w["dy"]).sum() + total, (x, enc))
        return {"y": y.detach(), "logits": logits.detach(), "loss": torch.stack((total, loss_b, loss_z)).detach(), "counts": counts, "dx": dx, "denc": denc}


@pytest.mark.parametrize("kw", [dict(), dict(layout=0, rot=64, nq=8, nk=200), dict(d=128, h=512, a=4, kh=4, rot=128, nq=136, nk=264, E=32, top_k=4)])
def test_a_layer_with_cross_attention_and_a_router(B, kw):
    """bf16 storage of every intermediate: 2e-2 relative, as the stage's own parity; the loss is a smooth function of logits that are off by a
    few steps of bf16, 1e-2 relative."""
    L = Layer(**kw)
    L.run(B)
    torch.cuda.synchronize()
    got, want = L.results(), L.reference()
    assert torch.equal(got["counts"].cpu().long(), want["counts"])
    for name in ("y", "logits", "dx", "denc"):
        assert rel_l2(got[name].cpu(), want[name]) < 2e-2, name
    assert bool(((got["loss"].cpu().double() - want["loss"]).abs() <= 1e-2 * want["loss"].abs()).all())


def test_captured_and_replayed(B):
    """The whole layer in a graph, replayed on changing inputs with eager runs between the replays: the same bits every time."""
    L = Layer(b=2, nq=8, nk=600, d=128, h=256, a=4, kh=2)      # few rows: keys in slices, joined
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        L.run(B)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.run(B)
    for i in range(4):
        L.x.copy_(torch.randn(L.x.shape, generator=torch.Generator(device=DEV).manual_seed(i), device=DEV).to(BF16))
        L.kv_len.copy_(torch.tensor([600 - 100 * i, 7 + i], dtype=torch.int32, device=DEV))
        L.run(B)
        torch.cuda.synchronize()
        eager = {n: t.clone() for n, t in L.results().items()}
        for t in L.results().values():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for name, t in L.results().items():
            assert torch.equal(t, eager[name]), (i, name)


def test_on_a_stream_of_its_own(B):
    L = Layer()
    L.run(B)
    torch.cuda.synchronize()
    first = {n: t.clone() for n, t in L.results().items()}
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        L.run(B)
    s.synchronize()
    for name, t in L.results().items():
        assert torch.equal(t, first[name]), name

"""The layer operators next to calls that were there before them: the normed rotation on a scaled table, the balance loss on the router gradients that a
stage's backward call has left; and calls with nothing to do, which write nothing."""
import pytest

import ops_reference as R
import synth

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DEV = "cuda:0"
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2604_27085_amd import binding
    return binding


def stream():
    return torch.cuda.current_stream().cuda_stream


@pytest.mark.parametrize("bwd", [0, 1])
@pytest.mark.parametrize("d", [64, 128])
def test_the_normed_rotation_takes_a_scaled_table(B, d, bwd):
    """rp_op_qknorm_rope, without its norm, on rp_op_rope_table's table, on the same one by rp_op_rope_table_scaled and on one scaled by parts: two products
    and a sum in fp32 (4 * 2^-24 of |x| + |y|), then half a step of bf16; the two equal tables differ by an fp32 rounding of each angle's cosine at most."""
    T, seq, a, k = 130, 65, 4, 2
    g = torch.Generator().manual_seed(d)
    q, kk = torch.randn((T, a, d), generator=g).to(BF16), torch.randn((T, k, d), generator=g).to(BF16)
    tables = [torch.empty((seq, d // 2, 2), device=DEV) for _ in range(3)]
    B.rp_op_rope_table(stream(), tables[0], seq, d, 1.0e6)
    B.rp_op_rope_table_scaled(stream(), tables[1], B.make_rope_scaling(B.ROPE_PLAIN, 1.0e6), seq, d)
    B.rp_op_rope_table_scaled(stream(), tables[2], B.make_rope_scaling(B.ROPE_BY_PARTS, 1.0e4, 4.0, 1.0, 8.0, 32, 1.2), seq, d)
    for cs in tables:
        oq, ok = torch.full((T, a, d), float("nan"), dtype=BF16, device=DEV), torch.full((T, k, d), float("nan"), dtype=BF16, device=DEV)
        B.rp_op_qknorm_rope(stream(), bwd, d, q.to(DEV), kk.to(DEV), a * d, k * d, oq, ok, a * d, k * d, None, None, None, None, None, None, 0, None, None, None,
                            cs, T, seq, a, k, 0, 1e-6)
        torch.cuda.synchronize()
        for x, y in ((q, oq), (kk, ok)):
            rows = cs.cpu()[torch.arange(T) % seq]
            want = R.rotate(x, rows, 0, d, bwd)
            size = R.rotate(x.abs(), rows.abs(), 0, d, 0).abs() + R.rotate(x.abs(), rows.abs(), 0, d, 1).abs()
            assert bool(((y.cpu().double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -21 * size + 1e-30).all())
    assert float((tables[0] - tables[1]).abs().max()) <= 2.0 ** -23


def test_nothing_to_do_writes_nothing(B):
    d = 64
    x, out = torch.ones((4, 2 * d), dtype=BF16, device=DEV), torch.full((4, 2 * d), 7.0, dtype=BF16, device=DEV)
    cs, i32 = torch.full((4, d // 2, 2), 7.0, device=DEV), torch.full((4,), 7, dtype=torch.int32, device=DEV)
    lse = torch.full((4, 2), 7.0, device=DEV)
    B.rp_op_rope_table_scaled(stream(), cs, B.make_rope_scaling(), 0, d)
    B.rp_op_rope(stream(), 0, 0, d, d, x, x, 2 * d, 2 * d, out, out, 2 * d, 2 * d, cs, 4, None, 0, 4, 2, 1)      # no tokens
    B.rp_op_rope(stream(), 0, 0, d, d, x, x, 2 * d, 2 * d, out, out, 2 * d, 2 * d, cs, 4, None, 4, 4, 0, 0)      # no heads
    B.rp_op_cross_attn_fwd(stream(), x, x, x, out, lse, 2 * d, d, d, 2 * d, None, None, 0, 4, 4, 2, 1, d, 0.1)   # no sequences
    B.rp_op_cross_attn_fwd(stream(), x, x, x, out, lse, 2 * d, d, d, 2 * d, None, None, 1, 0, 4, 2, 1, d, 0.1)   # no queries
    B.rp_op_cross_attn_bwd(stream(), x, x, x, x, x, lse, lse, out, out, out, 2 * d, d, d, 2 * d, 2 * d, 2 * d, d, d, None, None, 0, 4, 4, 2, 1, d, 0.1)
    B.rp_op_cross_attn_bwd(stream(), x, x, x, x, x, lse, lse, out, out, out, 2 * d, d, d, 2 * d, 2 * d, 2 * d, d, d, None, None, 1, 0, 0, 2, 1, d, 0.1)
    torch.cuda.synchronize()
    for t in (out, cs, i32, lse):
        assert bool((t == 7).all())


@pytest.mark.parametrize("coef,z", [(0.3, 0.0), (0.3, 0.02)])
def test_balance_loss_on_a_stages_router_gradients(B, coef, z):
    """A stage whose caller supplies the router logits (moe_router 0) leaves their gradient; the loss of every layer, balanced sequence by sequence, adds its
    own in place, on the same stream, and both go on to the caller's router together."""
    from paper_2604_27085_amd import harness
    from test_gpu_balance import check
    c = dict(n_layers=2, hidden=256, n_q_heads=4, n_kv_heads=2, head_dim=64, ffn=96, vocab=0, n_experts=8, top_k=2, lora_rank=8, lora=("q", "v"), train_base=0,
             batch=2, seq=72, x_from="normal")
    wl = synth.make_workload(c, 77, gains_random=True)
    run = harness.StageRunner(harness.cfg_from_dict(c, with_head=False), c["batch"], c["seq"])
    try:
        run.upload(run.pinned_blob(wl["layers"], None))
        T, E, k, st = run.T, c["n_experts"], c["top_k"], run.compute.cuda_stream
        router = torch.stack([torch.from_numpy(t) for t in wl["router_logits"]]).to(DEV)
        d_router = torch.full_like(router, float("nan"))
        i32 = lambda *s: torch.empty(s, dtype=torch.int32, device=DEV)  # noqa: E731
        idx, w, n = i32(2, T, k), torch.empty((T, k), device=DEV), T * k
        plan = (i32(E), i32(E + 1), i32(4 * (n // 256 + E + 1)), i32(1), i32(n), i32(n), i32((n + 511) // 512 * E))
        counts, tokens, loss = i32(2, c["batch"], E), i32(2, c["batch"] + 1), torch.empty((2, 3), device=DEV)
        ws = torch.empty(B.rp_op_moe_balance_scratch(T, c["seq"], E), dtype=torch.uint8, device=DEV)
        x, dy, both = harness.bf16_tensor(wl["x"], run.device), harness.bf16_tensor(wl["dy"], run.device), torch.empty_like(router)
        torch.cuda.synchronize()
        run.backward(x, dy, router=router, d_router=d_router)
        with torch.cuda.stream(run.compute):
            both.copy_(d_router)
            for li in range(2):
                B.rp_op_moe_route_plan(st, router[li], T, E, k, idx[li], w, *plan)
                B.rp_op_moe_balance(st, router[li], idx[li], None, T, c["seq"], E, k, coef, z, 1.0, counts[li], tokens[li], loss[li], both[li], both[li], ws)
        run.sync()
        assert bool(torch.isfinite(d_router).all()) and float(d_router.abs().max()) > 0
        for li in range(2):
            want = R.balance(router[li], idx[li], None, c["seq"], k, coef, z, 1.0)
            check((counts[li], tokens[li], loss[li], both[li]), want, d_router[li])
    finally:
        run.close()

"""Linear attention with a decay per head over packed sequences, on single tokens and backwards, against closed forms in 64 bits."""
import pytest
import torch

from paper_2506_18145_b200 import binding as rb

import linattn_testlib as T
from linattn_testlib import Problem, check_backward, check_forward
from serving_testlib import same_bits

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1, 8, 8), (4, 4, 64, 64), (4, 2, 128, 128), (3, 1, 40, 72), (2, 2, 128, 64), (2, 1, 64, 128), (6, 3, 16, 120), (2, 2, 72, 24)]
LENS = [[1], [0, 1, 2, 0], [31, 32, 33, 0], [127, 128, 129], [5, 0, 300, 1, 1, 64], [257, 640]]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,G,dk,dv", SHAPES)
@pytest.mark.parametrize("lens", LENS, ids=str)
def test_forward(lens, H, G, dk, dv, dtype):
    pr = Problem(lens, H, G, dk, dv, dtype, seed=sum(lens) + H, lead=3, tail=5)
    check_forward(pr, *pr.run())
    assert rb.rom_get_status(pr.ws) == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,G,dk,dv", SHAPES)
@pytest.mark.parametrize("lens", LENS, ids=str)
def test_backward(lens, H, G, dk, dv, dtype):
    pr = Problem(lens, H, G, dk, dv, dtype, seed=sum(lens) + H, lead=3, tail=5, backward=True)
    check_backward(pr, *pr.run_backward())
    assert rb.rom_get_status(pr.ws) == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H", [1, 3])
@pytest.mark.parametrize("lens", [[2300], [1024, 1024], [700, 900, 1, 0, 1200], [1] * 40 + [1500] + [1] * 40], ids=lambda v: str(v)[:24])
def test_sequences_over_many_cuts(lens, H, dtype):
    """One or three heads: the rows are cut into many segments, sequences begin, end and lie across them."""
    pr = Problem(lens, H, 1, 64, 64, dtype, seed=H, tail=2, resume=[1] * len(lens), backward=True)
    check_forward(pr, *pr.run())
    check_backward(pr, *pr.run_backward())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_plain_kernels_in_bf16_and_slots_in_place(dtype):
    """Updated in place, the pools give the same bits as with two buffers; states of sequences that span cuts are read before they are written."""
    lens = [900, 3, 0, 1400, 260]
    pr = Problem(lens, 2, 2, 64, 64, dtype, seed=5, resume=[1, 1, 1, 1, 0])
    o, s = pr.run()
    check_forward(pr, o, s)
    pool = pr.s_in.clone()
    o2, _ = pr.run(s_in=pool, s_out=pool)
    assert same_bits(o, o2)
    for i in range(len(lens)):
        assert same_bits(s[int(pr.p.slots[i])], pool[int(pr.p.slots[i])])
    if dtype == "bf16":
        plain = Problem(lens, 2, 2, 64, 64, dtype, seed=5, resume=[1, 1, 1, 1, 0], flags=rb.ROM_FLAG_SIMT_GEMM)
        check_forward(plain, *plain.run(), tensor=False)
        plain = Problem(lens, 4, 2, 64, 64, dtype, seed=5, resume=[1, 1, 1, 1, 0], flags=rb.ROM_FLAG_SIMT_GEMM, backward=True)
        check_backward(plain, *plain.run_backward(), tensor=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_pools_and_slots_outside_them(dtype):
    pr = Problem([130, 0, 64], 2, 1, 64, 64, dtype, seed=2, resume=[0, 0, 0])
    check_forward(pr, pr.run(s_in=None, s_out=None)[0], None)
    check_forward(pr, *pr.run(s_in=None))
    pr = Problem([130, 0, 64], 2, 1, 64, 64, dtype, seed=2, resume=[1, 1, 1], slots=[-1, 1 << 30, 1], n_slots=4, backward=True)
    check_forward(pr, *pr.run())
    check_backward(pr, *pr.run_backward())
    dq, dk, dv, _ = pr.run_backward(ds_out=None, ds_in=None)
    check_backward(pr, dq, dk, dv, None, no_state=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decays_from_none_to_all(dtype):
    """lambda = 1 (plain sums), slow, fast, and below the smallest number at once."""
    pr = Problem([300, 129, 1], 4, 4, 64, 64, dtype, seed=9, rates=[0.0, 1e-4, 3.0, 200.0], backward=True)
    check_forward(pr, *pr.run())
    check_backward(pr, *pr.run_backward())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_apart_scale_and_shared_heads(dtype):
    """Column slices of wider rows whose other columns are NaN; a scale of its own; eight value heads on one of q and k."""
    pr = Problem([77, 200], 8, 1, 48, 56, dtype, seed=3, wide=40, scale=-0.37, backward=True)
    check_forward(pr, *pr.run())
    dq, dk, dv, ds = pr.run_backward()
    check_backward(pr, dq, dk, dv, ds)
    buffer = torch.full((pr.p.rows, 8 * 56 + 24), 9.0, dtype=T.TORCH[dtype], device="cuda")
    view = buffer[:, 8:8 + 8 * 56]
    rb.rom_linattn_backward(pr.cfg, pr.p.ragged, pr.do, pr.q, pr.k, pr.v, pr.g, pr.s_in, pr.ds_out, dq, dk, view, ds, pr.ws)
    assert same_bits(view, dv) and (buffer[:, :8] == 9).all() and (buffer[:, 8 + 8 * 56:] == 9).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("which,bad", [("v", float("nan")), ("v", float("inf")), ("k", float("nan")), ("q", float("-inf"))])
def test_values_that_are_not_finite_stay_behind_their_row(which, bad, dtype):
    lens = [400, 150]
    pr = Problem(lens, 2, 2, 64, 64, dtype, seed=4, resume=[0, 0])
    o, s = pr.run()
    at = 173      # a row in the middle of a chunk; head 1, place 9
    getattr(pr, which)[at, 64 + 9] = bad
    o2, s2 = pr.run()
    x, y = o.view(-1, 2, 64), o2.view(-1, 2, 64)
    assert same_bits(x[:, 0], y[:, 0]) and same_bits(x[400:], y[400:])      # the other head, the other sequence
    assert torch.isfinite(y[:at].float()).all()
    # earlier rows of the same chunk may be summed by other instructions, but they are the same sums
    check_forward_rows = (y[:at].float() - x[:at].float()).abs().max() <= 2 ** -6 * x[:at].float().abs().max()
    assert check_forward_rows
    rows = y[at:400, 1].float()
    if which == "v":
        assert not torch.isfinite(rows[:, 9]).any()
        others = torch.arange(64, device="cuda") != 9
        assert torch.isfinite(rows[:, others]).all()
        assert not torch.isfinite(s2[int(pr.p.slots[0]), 1, :, 9]).any() and torch.isfinite(s2[int(pr.p.slots[0]), 1][:, others]).all()
    elif which == "k":
        assert not torch.isfinite(rows).any() and not torch.isfinite(s2[int(pr.p.slots[0]), 1, 9]).any()
    else:
        assert not torch.isfinite(rows[0]).any() and same_bits(x[at + 1:], y[at + 1:]) and same_bits(s, s2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_lost_state_stays_lost_over_every_cut(dtype):
    pr = Problem([3000], 1, 1, 64, 64, dtype, seed=6, rates=[1e-3])
    pr.v[100, 5] = float("nan")
    o, s = pr.run()
    assert torch.isfinite(o[:100].float()).all() and not torch.isfinite(o[100:, 5].float()).any() and torch.isfinite(o[:, 6:].float()).all()
    pr = Problem([3000], 1, 1, 64, 64, dtype, seed=6, rates=[1e-3], backward=True)
    pr.do[2900, 5] = float("nan")
    dq, dk, dv, ds = pr.run_backward()
    assert not torch.isfinite(dv[:2901, 5].float()).any() and torch.isfinite(dv[2901:].float()).all() and torch.isfinite(dv[:, 6:].float()).all()
    assert torch.isfinite(dk[2901:].float()).all() and not torch.isfinite(dk[:2901].float()).any() and torch.isfinite(dq[:2900].float()).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_same_from_run_to_run_in_a_graph_and_on_another_stream(dtype):
    pr = Problem([900, 333, 1], 4, 2, 128, 64, dtype, seed=8, backward=True)
    first = [*pr.run(), *pr.run_backward()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = [*pr.run(), *pr.run_backward()]
    side.synchronize()
    for a, b in zip(first, again):
        assert same_bits(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = [*pr.run(), *pr.run_backward()]
    for x in held:
        x.fill_(-7.0)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(first, held):
        assert same_bits(a, b)
    assert rb.rom_get_status(pr.ws) == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_workspace_for_smaller_batches(dtype):
    big, small = Problem([2000], 1, 1, 64, 64, dtype, seed=1, backward=True), Problem([300, 7], 1, 1, 64, 64, dtype, seed=2, backward=True)
    small.ws = big.ws
    check_forward(big, *big.run())
    check_forward(small, *small.run())
    check_backward(big, *big.run_backward())
    check_backward(small, *small.run_backward())


# ---------------------------------------------------------------------------------------------- single tokens
def step_problem(B, H, G, dk, dv, dtype, n_slots, seed=0, wide=0):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    rows = lambda w: rnd(B, w + wide).to(T.TORCH[dtype]).cuda()[:, :w]  # noqa: E731
    q, k, v = rows(G * dk), rows(G * dk), rows(H * dv)
    return q, k, v, (-torch.logspace(-0.3, -4, H)).cuda(), rnd(n_slots, H, dk, dv).cuda()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,H,G,dk,dv", [(1, 32, 32, 128, 128), (1, 1, 1, 8, 8), (5, 3, 1, 40, 72), (64, 4, 2, 64, 64), (3, 6, 2, 24, 128), (300, 2, 2, 16, 8)])
def test_step(B, H, G, dk, dv, dtype):
    q, k, v, g, pool = step_problem(B, H, G, dk, dv, dtype, B + 2, wide=16)
    cfg = rb.make_linattn_config(H, G, dk, dv, dtype)
    slot = torch.randperm(B + 2, generator=torch.Generator().manual_seed(1))[:B].to(torch.int32)
    if B > 2:
        slot[1], slot[B - 1] = -1, B + 2
    slot = slot.cuda()
    out, o = torch.full_like(pool, -7.0), torch.full((B, H * dv), -7.0, dtype=T.TORCH[dtype], device="cuda")
    rb.rom_linattn_step(cfg, q, k, v, g, slot, pool, out, o)
    named = set()
    for b, s in enumerate(slot.tolist()):
        if not 0 <= s < B + 2:
            assert (o[b] == -7).all()
            continue
        named.add(s)
        q1, k1, v1 = q[b].double().view(1, G, dk), k[b].double().view(1, G, dk), v[b].double().view(1, H, dv)
        ref, S = T.forward(q1, k1, v1, g.double(), pool[s].double(), float(cfg.scale))
        size, Ssize = T.forward(q1.abs(), k1.abs(), v1.abs(), g.double(), pool[s].double().abs(), float(cfg.scale))
        # a state: its decay's rounding, the product and the sum, 4 units; an output: those and a sum of dk terms
        T.near(o[b], ref[0].reshape(-1), size[0].reshape(-1), (dk + 8) * T.U32, dtype, f"o {b}")
        T.near(out[s], S, Ssize, 4 * T.U32, "f32", f"state {b}")
    for s in range(B + 2):
        if s not in named:
            assert (out[s] == -7).all()
    in_place, o2 = pool.clone(), torch.full_like(o, -7.0)
    rb.rom_linattn_step(cfg, q, k, v, g, slot, in_place, in_place, o2)
    assert same_bits(o, o2)
    for s in named:
        assert same_bits(in_place[s], out[s])
    if B <= 5:      # slot b without a table
        o3, out3 = torch.full_like(o, -7.0), torch.full_like(pool, -7.0)
        rb.rom_linattn_step(cfg, q, k, v, g, None, pool, out3, o3)
        o4, out4 = torch.full_like(o, -7.0), torch.full_like(pool, -7.0)
        rb.rom_linattn_step(cfg, q, k, v, g, torch.arange(B, dtype=torch.int32, device="cuda"), pool, out4, o4)
        assert same_bits(o3, o4) and same_bits(out3, out4)


def test_pools_beyond_32_bits_of_elements():
    """A slot whose state begins behind 2^31 floats."""
    H, d, n_slots = 32, 128, 4200
    cfg = rb.make_linattn_config(H, H, d, d, "bf16")
    q, k, v, g, one = step_problem(1, H, H, d, d, "bf16", 1, seed=2)
    pool = torch.empty((n_slots, H, d, d), device="cuda")
    pool[n_slots - 1] = one[0]
    slot = torch.tensor([n_slots - 1], dtype=torch.int32, device="cuda")
    o, o1, out1 = torch.empty((1, H * d), dtype=torch.bfloat16, device="cuda"), torch.empty((1, H * d), dtype=torch.bfloat16, device="cuda"), torch.empty_like(one)
    rb.rom_linattn_step(cfg, q, k, v, g, None, one, out1, o1)
    rb.rom_linattn_step(cfg, q, k, v, g, slot, pool, pool, o)
    assert same_bits(o, o1) and same_bits(pool[n_slots - 1], out1[0])


# ---------------------------------------------------------------------------------------------- as they are used
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_prompt_in_pieces_and_token_by_token(dtype):
    """Norm and rotation, then the recurrence: a prompt in two pieces and three tokens on its slot give what one call over all rows gives."""
    H, G, d, n, rot = 4, 2, 64, 150, 32
    gen = torch.Generator().manual_seed(11)
    proj = torch.randn((n, 2 * G * d + H * d), generator=gen).to(T.TORCH[dtype]).cuda()
    qk, cfg = rb.make_qk_config(G, G, d, rot, dtype), rb.make_linattn_config(H, G, d, d, dtype)
    w = (1 + 0.1 * torch.randn(d, generator=gen)).cuda()
    freq, g = (10000.0 ** (-torch.arange(rot // 2) / (rot // 2))).cuda(), (-torch.logspace(-1, -3, H)).cuda()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731

    def rows(a, b):
        x = proj[a:b]
        q, k = (torch.empty((b - a, G * d), dtype=proj.dtype, device="cuda") for _ in range(2))
        rb.rom_qk_norm_rope(qk, x[:, :G * d], x[:, G * d:2 * G * d], w, w, torch.arange(a, b, dtype=torch.int32, device="cuda"), freq, q, k)
        return q, k, x[:, 2 * G * d:]

    def piece(a, b, pool, resume):
        o, seqs = torch.empty((b - a, H * d), dtype=proj.dtype, device="cuda"), rb.make_ragged(b - a, 3, i32(0, b - a), i32(1), i32(resume))
        ws = torch.empty(rb.linattn_ragged_workspace_size(cfg, 1, b - a), dtype=torch.uint8, device="cuda")
        rb.rom_linattn_ragged(cfg, seqs, *rows(a, b), g, pool, pool, o, ws)
        return o

    whole, pool = torch.zeros((3, H, d, d), device="cuda"), torch.zeros((3, H, d, d), device="cuda")
    ref = piece(0, n, whole, 0)
    got = [piece(0, 70, pool, 0), piece(70, n - 3, pool, 1)]
    for t in range(n - 3, n):
        o = torch.empty((1, H * d), dtype=proj.dtype, device="cuda")
        rb.rom_linattn_step(cfg, *rows(t, t + 1), g, i32(1), pool, pool, o)
        got.append(o)
    got = torch.cat(got).float()
    # bf16: both sides round the scores or the state, and the output: 2 x 3 roundings of half a step in the 2-norm; fp32: the sums' rounding
    tol = 2 * 2.0 ** -8 if dtype == "bf16" else 2.0 ** -18
    assert (got - ref.float()).norm() <= tol * ref.float().norm()
    assert (pool[1] - whole[1]).norm() <= 2.0 ** -14 * whole[1].norm()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_training_step_of_norm_and_recurrence(dtype):
    """The gradient of the projection's rows through both backward calls, against the formulas in 64 bits through the stored q and k."""
    H, G, d, rot, lens = 4, 2, 64, 64, [100, 40, 160]
    n = sum(lens)
    gen = torch.Generator().manual_seed(12)
    proj = torch.randn((n, 2 * G * d + H * d), generator=gen).to(T.TORCH[dtype]).cuda()
    qkc, cfg = rb.make_qk_config(G, G, d, rot, dtype), rb.make_linattn_config(H, G, d, d, dtype)
    wq, wk = ((1 + 0.1 * torch.randn(d, generator=gen)).cuda() for _ in range(2))
    freq, g = (10000.0 ** (-torch.arange(rot // 2) / (rot // 2))).cuda(), (-torch.logspace(-1, -3, H)).cuda()
    pos = torch.cat([torch.arange(m) for m in lens]).to(torch.int32).cuda()
    start = torch.tensor([0, 100, 140, 300], dtype=torch.int32, device="cuda")
    seqs = rb.make_ragged(n, 3, start)
    xq, xk, v = proj[:, :G * d], proj[:, G * d:2 * G * d], proj[:, 2 * G * d:]
    new = lambda w: torch.empty((n, w), dtype=proj.dtype, device="cuda")  # noqa: E731
    q, k, o, do = new(G * d), new(G * d), new(H * d), torch.randn((n, H * d), generator=gen).to(proj.dtype).cuda()
    ws = torch.empty(max(rb.linattn_backward_workspace_size(cfg, 3, n), rb.qk_norm_rope_backward_workspace_size(qkc, n)), dtype=torch.uint8, device="cuda")
    dproj, dq, dk = torch.empty_like(proj), new(G * d), new(G * d)
    dwq, dwk = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    rb.rom_qk_norm_rope(qkc, xq, xk, wq, wk, pos, freq, q, k)
    rb.rom_linattn_ragged(cfg, seqs, q, k, v, g, None, None, o, ws)
    rb.rom_linattn_backward(cfg, seqs, do, q, k, v, g, None, None, dq, dk, dproj[:, 2 * G * d:], None, ws)
    rb.rom_qk_norm_rope_backward(qkc, dq, dk, xq, xk, wq, wk, pos, freq, dproj[:, :G * d], dproj[:, G * d:2 * G * d], dwq, dwk, ws)
    want = torch.empty(proj.shape, dtype=torch.float64, device="cuda")
    gq, gk = torch.empty((n, G, d), dtype=torch.float64, device="cuda"), torch.empty((n, G, d), dtype=torch.float64, device="cuda")
    zero = torch.zeros((H, d, d), dtype=torch.float64, device="cuda")
    cut = lambda x, m: x.double().reshape(n, m, d)  # noqa: E731
    for a, b in zip(start.tolist()[:-1], start.tolist()[1:]):
        x = [cut(t, m)[a:b] for t, m in ((do, H), (q, G), (k, G), (v, H))]
        gq[a:b], gk[a:b], dv, _ = T.backward(*x, g.double(), zero, zero, d ** -0.5)
        want[a:b, 2 * G * d:] = dv.reshape(b - a, -1)
    for i, (x, w, gy) in enumerate(((xq, wq, gq), (xk, wk, gk))):
        dx, dw, _ = T.norm_rope_backward(gy, cut(x, G), w.double(), pos, freq, rot, False, 1e-6)
        want[:, i * G * d:(i + 1) * G * d] = dx.reshape(n, -1)
        # dw of stored gradients that each lost half a step: independent, so the norm's share of it, twice
        assert (((dwq, dwk)[i].double() - dw).norm() <= (2 * 2.0 ** -8 if dtype == "bf16" else 2.0 ** -18) * dw.norm())
    # roundings in bf16: scores, stored dq or dk, stored dx, each half a step at most: 2^-8 of the norm as in `near`
    assert (dproj.double() - want).norm() <= (2.0 ** -8 if dtype == "bf16" else 2.0 ** -19) * want.norm()


@pytest.mark.parametrize("what", ["shape", "dtype", "host", "pitch"])
def test_binding_refuses(what):
    cfg = rb.make_linattn_config(2, 1, 64, 64, "bf16")
    x = lambda w, rows=10, dtype=torch.bfloat16: torch.zeros((rows, w), dtype=dtype, device="cuda")  # noqa: E731
    seqs = rb.make_ragged(10, 1, torch.tensor([0, 10], dtype=torch.int32, device="cuda"))
    a = dict(q=x(64), k=x(64), v=x(128), g=torch.zeros(2, device="cuda"), s_in=None, s_out=None, o=x(128), ws=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
    bad = {"shape": [("q", x(32)), ("v", x(128, 9)), ("o", x(128, 9)), ("g", torch.zeros(1, device="cuda")), ("s_out", torch.zeros(64 * 64, device="cuda"))],
           "dtype": [("k", x(64, 10, torch.float32)), ("o", x(128, 10, torch.float32)), ("g", torch.zeros(2, dtype=torch.float64, device="cuda"))],
           "host": [("q", x(64).cpu()), ("ws", a["ws"].cpu())], "pitch": [("k", x(128)[:, ::2]), ("o", x(256)[:, :128])]}[what]
    for name, t in bad:
        with pytest.raises(ValueError):
            rb.rom_linattn_ragged(cfg, seqs, *{**a, name: t}.values())
    rb.rom_linattn_ragged(cfg, seqs, *a.values())


@pytest.mark.parametrize("H,G,dk,dv,lens", [(2, 2, 128, 128, [700]), (4, 2, 64, 64, [100, 300]), (1, 1, 64, 128, [2000])])
def test_stalled_call_is_reported(H, G, dk, dv, lens):
    """The timeout path: more bytes are expected than are copied, every wait gives up, the call returns and says so, the workspace stays usable."""
    from test_gpu_parity import _status_detail
    pr = Problem(lens, H, G, dk, dv, "bf16", seed=1, backward=True)
    ref = pr.run()
    good, stalled = pr.cfg, rb.make_linattn_config(H, G, dk, dv, "bf16", flags=rb.ROM_FLAG_TEST_STALL)
    for call in (pr.run, pr.run_backward):
        pr.cfg = stalled
        call()
        torch.cuda.synchronize()
        assert 51 <= _status_detail(pr.ws)[1] <= 57
        assert rb.rom_get_status(pr.ws) == -6
        pr.cfg = good
        again = pr.run()
        assert same_bits(ref[0], again[0]) and same_bits(ref[1], again[1]) and rb.rom_get_status(pr.ws) == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_empty_sequences_alone(dtype):
    """No rows at all: a resumed sequence keeps its state, another leaves zeros; backwards the gradient passes through."""
    pr = Problem([0, 0, 0], 2, 1, 64, 64, dtype, seed=3, resume=[1, 0, 1], tail=4, backward=True)
    o, s = pr.run()
    dq, dk, dv, ds = pr.run_backward()
    for i in range(3):
        slot = int(pr.p.slots[i])
        assert same_bits(s[slot], pr.s_in[slot]) if pr.p.resumes(i) else (s[slot] == 0).all()
        assert same_bits(ds[slot], pr.ds_out[slot]) if pr.p.resumes(i) else (ds[slot] == 0).all()
    for x in (o, dq, dk, dv):
        assert (x == -7).all()
    seqs = rb.make_ragged(0, pr.p.n_slots, torch.zeros(4, dtype=torch.int32, device="cuda"), *pr.p.dev[1:])
    none, out = pr.q[:0], torch.full_like(pr.s_in, -7.0)
    rb.rom_linattn_ragged(pr.cfg, seqs, none, none, pr.v[:0], pr.g, pr.s_in, out, pr.do[:0], pr.ws)
    assert same_bits(out, s)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [40, 300])
def test_many_short_sequences(n, dtype):
    """Runs of many sequences: one, two and a few rows each, empty ones between, some longer; of more than 256 rows a sequence none."""
    g = torch.Generator().manual_seed(n)
    lens = [int(x) for x in torch.randint(0, 4, (n,), generator=g)]
    lens[n // 3], lens[n // 2] = 200, 131
    pr = Problem(lens, 3, 1, 72, 40, dtype, seed=n, backward=True)
    check_forward(pr, *pr.run())
    check_backward(pr, *pr.run_backward())
    pool = pr.s_in.clone()
    o, s = pr.run()
    o2, _ = pr.run(s_in=pool, s_out=pool)
    assert same_bits(o, o2) and all(same_bits(s[int(k)], pool[int(k)]) for k in pr.p.slots)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,lens", [(160, [300]), (150, [64, 900]), (40, [1000, 3, 2000]), (17, [4000])], ids=str)
def test_head_counts_beside_the_blocks(H, lens, dtype):
    """Whole heads on more blocks than the GPU holds, and runs that begin in one head and end in the next."""
    pr = Problem(lens, H, H, 16, 16, dtype, seed=H, rates=[0.3 * 0.97 ** h for h in range(H)], backward=True)
    check_forward(pr, *pr.run())
    check_backward(pr, *pr.run_backward())


def test_offsets_that_are_out_of_order_stay_in_bounds():
    """What they yield is unspecified; rows of the buffers and slots behind the named ones are not touched, and nothing faults."""
    H, d, rows = 2, 64, 700
    cfg = rb.make_linattn_config(H, H, d, d, "bf16")
    q, k, v = (torch.randn((rows, H * d), device="cuda").bfloat16() for _ in range(3))
    g, pool = torch.full((H,), -0.01, device="cuda"), torch.zeros((4, H, d, d), device="cuda")
    guarded = torch.full((rows + 64, H * d), -7.0, dtype=torch.bfloat16, device="cuda")
    for start in ([0, 600, 200, 5000], [-40, 300, 300, 650], [699, 0, 10, 20]):
        seqs = rb.make_ragged(rows, 3, torch.tensor(start, dtype=torch.int32, device="cuda"), torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda"))
        ws = torch.zeros(rb.linattn_ragged_workspace_size(cfg, 3, rows), dtype=torch.uint8, device="cuda")
        rb.rom_linattn_ragged(cfg, seqs, q, k, v, g, pool, pool, guarded[:rows], ws)
        torch.cuda.synchronize()
        assert (guarded[rows:] == -7).all() and (pool[3] == 0).all() and rb.rom_get_status(ws) == 0

"""How exact the serving calls are: bounds that only what a call promises satisfies (the bounds of serving_testlib.py allow the hidden rows of the FFN and the
inputs of the scan more than that), and values that are not finite."""
import numpy as np
import pytest
import torch

from oracle import rom_oracle as O
from paper_2506_18145_b200 import binding as rb

from rom_testlib import np64
from serving_testlib import TORCH, U32, Packed, check, randn, same_bits, silu_bound

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------------------------- FFN-MoE of a few tokens
HALVES = 2.0 ** -16      # a value held as the sum of two bf16 numbers: half a step (2^-8) of what half a step (2^-8) leaves


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,Dm,F,E,K", [(1, 64, 128, 1, 1), (5, 128, 256, 4, 3), (8, 64, 128, 1, 1), (9, 192, 128, 1, 1), (17, 320, 384, 3, 2), (33, 64, 256, 1, 1), (64, 128, 128, 8, 2),
                                        (64, 64, 128, 1, 1), (48, 128, 256, 2, 1)])
def test_ffn_step_hidden_rows(B, Dm, F, E, K, dtype):
    """The hidden rows are held in more bits than the storage type's: an output near zero, where half a step of it is small, shows it."""
    x, W_gu, W_down = randn(251, (B, Dm), dtype=TORCH[dtype]), randn(252, (E, 2 * F, Dm), Dm ** -0.5, TORCH[dtype]), randn(253, (E, Dm, F), F ** -0.5, TORCH[dtype])
    g = np.random.default_rng(254)
    idx = np.stack([g.permutation(E)[:K] for _ in range(B)]).astype(np.int32)
    gates = g.random((B, K)).astype(np.float32)
    cfg = rb.make_config(B, 1, Dm, 64, 16, 4, 16, E, K, dtype)
    ws = torch.full((rb.ffn_moe_step_workspace_size(cfg, F),), 255, dtype=torch.uint8, device="cuda")
    out = torch.full((B, Dm), float("nan"), dtype=TORCH[dtype], device="cuda")
    rb.rom_ffn_moe_step(cfg, F, W_gu.cuda(), W_down.cuda(), x.cuda(), torch.from_numpy(idx).cuda(), torch.from_numpy(gates).cuda(), out, ws)
    torch.cuda.synchronize()
    assert rb.rom_get_status(ws) == 0
    # a sum of n products in fp32 is at most 2 n U of its |terms| off; SiLU as in silu_bound; two products on the way to a hidden value
    X, Wg, Wd = np64(x), np64(W_gu), np64(W_down)
    held = HALVES if dtype == "bf16" else U32
    ref, bound = np.zeros((B, Dm)), np.zeros((B, Dm))
    for t in range(B):
        for k in range(K):
            e = idx[t, k]
            gu, size = Wg[e] @ X[t], np.abs(Wg[e]) @ np.abs(X[t])
            a, b = gu[:F], gu[F:]
            ea, eb = 2 * Dm * U32 * size[:F], 2 * Dm * U32 * size[F:]
            h = O.silu(a) * b * gates[t, k]
            eh = gates[t, k] * (silu_bound(a, ea) * (np.abs(b) + eb) + np.abs(O.silu(a)) * eb) + (held + 4 * U32) * np.abs(h)
            n = 2 * F if dtype == "bf16" else F
            ref[t] += Wd[e] @ h
            bound[t] += np.abs(Wd[e]) @ eh + 2 * n * U32 * (np.abs(Wd[e]) @ np.abs(h)) + 2 * K * U32 * np.abs(Wd[e] @ h)
    check(out, ref, bound, dtype, "out")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ffn_step_hidden_value_that_overflows(dtype):
    """A hidden value past the largest fp32 number makes the outputs infinite, those of its token alone."""
    B, Dm, F = 3, 64, 128
    x, W_gu, W_down = torch.zeros(B, Dm), torch.zeros(1, 2 * F, Dm), torch.ones(1, Dm, F)
    x[:, 0] = torch.tensor([1.0, 2.0 ** 70, 2.0])
    W_gu[0, 5, 0], W_gu[0, F + 5, 0] = 1.0, 1.0
    cfg = rb.make_config(B, 1, Dm, 64, 16, 4, 16, 1, 1, dtype)
    ws = torch.empty(rb.ffn_moe_step_workspace_size(cfg, F), dtype=torch.uint8, device="cuda")
    out = torch.empty((B, Dm), dtype=TORCH[dtype], device="cuda")
    rb.rom_ffn_moe_step(cfg, F, *(v.to(TORCH[dtype]).cuda() for v in (W_gu, W_down, x)), torch.zeros((B, 1), dtype=torch.int32, device="cuda"), torch.ones((B, 1), device="cuda"), out, ws)
    assert torch.all(torch.isposinf(out[1])) and torch.all(torch.isfinite(out[[0, 2]]))


# ---------------------------------------------------------------------------------------------- scan over packed sequences
SMALL = 2.0 ** -12      # |Delta A| from which on the bf16 form takes a step's input from 1 - exp(Delta A)


def scan_exact(u, delta, A, Bm, Cm, D, z, h0, disc_mode, dtype):
    """(y, bound of its error, h_last, bound of its error) of one sequence.

    A step's decay is at most 5 units of 1 off (units U of fp32; x = Delta A: its rounding and that of its exponent change exp(x) by 3 |x| exp(x) < 1.2 of them,
    the exponential is 4 off and below 1), its input (expm1(x) / A) B u at most 17 units of itself (expm1 13: the series' few, or where |x| > 0.35 those of
    exp(x) over |expm1(x)|; a quotient and three products), and the sum rounds once: within 24 units of |h_{t-1}| and |input|, which decay with the state.
    bf16 takes expm1(x) as exp(x) - 1 where |x| >= 2^-12: within 16 units of |B u / A| there."""
    n, De = u.shape
    h, G = np.array(h0), np.zeros_like(h0)
    y, bound = np.zeros((n, De)), np.zeros((n, De))
    gate = O.silu(z)
    for t in range(n):
        x = delta[t][:, None] * A
        a = np.exp(x)
        bu = Bm[t][None, :] * u[t][:, None]
        inp = np.expm1(x) / A * bu if disc_mode == 0 else delta[t][:, None] * bu
        off = 24.0 * np.abs(inp)
        if disc_mode == 0 and dtype == "bf16":
            off = np.where(np.abs(x) >= SMALL, 16.0 * np.abs(bu / A), off)
        G = a * G + U32 * (24.0 * np.abs(h) + off)
        h = a * h + inp
        v = h @ Cm[t] + D * u[t]
        e = G @ np.abs(Cm[t]) + 20.0 * U32 * (np.abs(h) @ np.abs(Cm[t]) + np.abs(D * u[t]))
        y[t] = v * gate[t]
        bound[t] = e * np.abs(gate[t]) + np.abs(v) * silu_bound(z[t], 0.0)
    return y, bound, h, G


def scan_run(p, De, dtype, disc_mode, s, h0):
    """y and the pool after a call in place."""
    cfg = rb.make_config(1, 1, 64, De, 16, 4, 16, 1, 1, dtype, disc_mode=disc_mode)
    d = {n: v.cuda() for n, v in s.items()}
    ws = torch.full((rb.scan_ragged_workspace_size(cfg, p.n, p.rows),), 255, dtype=torch.uint8, device="cuda")
    y, h = torch.zeros_like(d["u"]), h0.cuda()
    rb.rom_scan_ragged(cfg, p.ragged, d["u"], d["delta"], d["A"], d["Bm"], d["Cm"], d["D"], d["z"], h, h, y, ws)
    torch.cuda.synchronize()
    return y, h


def one_sign(rows, De, dtype, dt, seed=0):
    """Inputs of one sign, so that errors of a step add up, and Delta log-uniform in dt."""
    g = torch.Generator()
    g.manual_seed(300 + seed)
    lo, hi = np.log(dt[0]), np.log(dt[1])
    return dict(u=randn(301 + seed, (rows, De)).abs().add(0.1).to(TORCH[dtype]), delta=torch.exp(torch.rand((rows, De), generator=g) * (hi - lo) + lo),
                A=-(torch.arange(1, 17).float()[None] * (0.5 + torch.rand((De, 16), generator=g))).contiguous(), Bm=randn(302 + seed, (rows, 16)).abs().add(0.1),
                Cm=randn(303 + seed, (rows, 16)), D=1.0 + randn(304 + seed, (De,), 0.1), z=randn(305 + seed, (rows, De), dtype=TORCH[dtype]))


def check_scan(p, De, dtype, disc_mode, s, h0):
    y, h = scan_run(p, De, dtype, disc_mode, s, h0)
    f = {n: np64(v) for n, v in s.items()}
    for i in range(p.n):
        a, e = p.start[i], p.start[i + 1]
        before = np64(h0[p.slots[i]]) if p.resumes(i) else np.zeros((De, 16))
        ref, bound, last, G = scan_exact(f["u"][a:e], f["delta"][a:e], f["A"], f["Bm"][a:e], f["Cm"][a:e], f["D"], f["z"][a:e], before, disc_mode, dtype)
        check(h[p.slots[i]], last, G, "f32", f"state of sequence {i}")
        check(y[a:e], ref, bound, dtype, f"sequence {i}")


@pytest.mark.parametrize("dt", [(1e-6, 1e-5), (3e-8, 1e-6), (1e-5, 1e-1)])
@pytest.mark.parametrize("disc_mode", [0, 1])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scan_ragged_slow_decays_add_up_their_inputs(dtype, disc_mode, dt):
    """What a state gains in thousands of steps that each decay it by next to nothing."""
    p = Packed([4000, 37, 0, 1, 15, 600], lead=3, tail=2, seed=31, resume=[0, 1, 1, 0, 1, 1])
    check_scan(p, 64, dtype, disc_mode, one_sign(p.rows, 64, dtype, dt), randn(32, (p.n_slots, 64, 16), 0.3))


@pytest.mark.parametrize("disc_mode", [0, 1])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scan_ragged_steps_of_no_length_change_nothing(dtype, disc_mode):
    p = Packed([900, 3, 40], seed=33, resume=[1, 1, 1])
    s = one_sign(p.rows, 64, dtype, (0.1, 1.0), seed=1)
    s["delta"] = torch.zeros_like(s["delta"])
    h0 = randn(34, (p.n_slots, 64, 16), 0.3)
    assert same_bits(scan_run(p, 64, dtype, disc_mode, s, h0)[1], h0.cuda())


@pytest.mark.parametrize("disc_mode", [0, 1])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scan_ragged_input_that_is_infinite(dtype, disc_mode):
    """B infinite for one state at one row, of a sequence inside one chunk and of one over many: that state is infinite from there on, and the others are not touched.  (Its
    decay does not reach zero before the sequence's end.)"""
    De, at, n = 64, 5, 3
    p = Packed([500, 12], seed=35, resume=[0, 0])
    s = one_sign(p.rows, De, dtype, (1e-3, 1e-2), seed=2)
    for a in p.start[:-1]:
        s["Bm"][a + at, n] = float("inf")
    h0 = torch.zeros((p.n_slots, De, 16))
    y, h = scan_run(p, De, dtype, disc_mode, s, h0)
    s["Bm"][:, n] = 0.0
    y0, h_rest = scan_run(p, De, dtype, disc_mode, s, h0)
    others = [i for i in range(16) if i != n]
    for i, (a, e) in enumerate(zip(p.start, p.start[1:])):
        q = int(p.slots[i])
        assert torch.all(torch.isposinf(h[q, :, n])) and torch.all(torch.isfinite(h[q][:, others]))
        torch.testing.assert_close(h[q][:, others], h_rest[q][:, others], rtol=1e-4, atol=0.0)      # (the row with the infinite B is run another way)
        sign = torch.sign(s["Cm"][a + at:e, n])[:, None] * torch.sign(s["z"][a + at:e].float())
        want = (sign * float("inf")).cuda()
        assert torch.equal(y[a + at:e].float(), want) and torch.all(torch.isfinite(y[a:a + at]))


@pytest.mark.parametrize("lens", [[1500], [700, 0, 3, 900, 40], [9, 30, 1100]])
@pytest.mark.parametrize("disc_mode", [0, 1])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scan_ragged_infinite_state_stays_infinite(dtype, disc_mode, lens):
    """An initial state of infinity, of one channel and state: no step's decay is zero, the product of ten of them is.  However the rows are cut into chunks,
    that state is infinite at the end of its sequence, and nothing else differs from a call with a zero in its place."""
    De, c, n = 64, 37, 11
    p = Packed(lens, seed=41, resume=[1] * len(lens))
    s = one_sign(p.rows, De, dtype, (1.0, 2.0), seed=3)
    s["A"] = -(3.0 + torch.rand((De, 16), generator=torch.Generator().manual_seed(42)) * 8.0)
    h0 = randn(43, (p.n_slots, De, 16), 0.3)
    h0[:, c, n] = 0.0
    y0, rest = scan_run(p, De, dtype, disc_mode, s, h0)
    h0[:, c, n] = -float("inf")
    y, h = scan_run(p, De, dtype, disc_mode, s, h0)
    others = torch.ones(De, dtype=torch.bool)
    others[c] = False
    for i, (a, e) in enumerate(zip(p.start, p.start[1:])):
        q = int(p.slots[i])
        assert torch.isneginf(h[q, c, n]) and same_bits(h[q][others], rest[q][others]) and same_bits(h[q, c, :n], rest[q, c, :n]) and same_bits(h[q, c, n + 1:], rest[q, c, n + 1:])
        want = -torch.sign(s["Cm"][a:e, n]) * torch.sign(s["z"][a:e, c].float()) * float("inf")
        assert torch.equal(y[a:e, c].float(), want.cuda()) and same_bits(y[a:e][:, others], y0[a:e][:, others])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scan_ragged_state_of_zero_that_grows(dtype):
    """Steps backwards: no input before the last row, and decays whose product over ten rows is past the largest number.  A state of zero stays zero."""
    De = 64
    p = Packed([900], seed=44, resume=[0])
    s = one_sign(p.rows, De, dtype, (0.2, 0.5), seed=4)
    s["delta"] = -s["delta"]
    s["A"] = -(20.0 + 20.0 * torch.rand((De, 16), generator=torch.Generator().manual_seed(45)))
    s["u"][:-1] = 0.0
    y, h = scan_run(p, De, dtype, 1, s, torch.zeros((p.n_slots, De, 16)))
    want = (s["delta"][-1] * s["u"][-1].float())[:, None] * s["Bm"][-1][None]
    torch.testing.assert_close(h[int(p.slots[0])].cpu(), want, rtol=1e-6, atol=0.0)
    assert torch.all(y[:-1] == 0)


@pytest.mark.parametrize("B", [1, 5, 13, 30, 64])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ffn_step_infinite_weight(dtype, B):
    """An infinite weight of the down projection makes its output infinite, of the sign of weight and hidden value, and no other output differs."""
    Dm, F, d, f = 64, 256, 37, 201
    x, W_gu, W_down = randn(261, (B, Dm), dtype=TORCH[dtype]), randn(262, (1, 2 * F, Dm), Dm ** -0.5, TORCH[dtype]), randn(263, (1, Dm, F), F ** -0.5, TORCH[dtype])
    cfg = rb.make_config(B, 1, Dm, 64, 16, 4, 16, 1, 1, dtype)
    idx, gates = torch.zeros((B, 1), dtype=torch.int32, device="cuda"), torch.ones((B, 1), device="cuda")
    outs = []
    for w in (0.0, -float("inf")):
        W_down[0, d, f] = w
        ws = torch.empty(rb.ffn_moe_step_workspace_size(cfg, F), dtype=torch.uint8, device="cuda")
        outs.append(torch.empty((B, Dm), dtype=TORCH[dtype], device="cuda"))
        rb.rom_ffn_moe_step(cfg, F, W_gu.cuda(), W_down.cuda(), x.cuda(), idx, gates, outs[-1], ws)
    gu = np64(W_gu)[0] @ np64(x).T
    h = (O.silu(gu[:F]) * gu[F:])[f]
    assert torch.equal(outs[1][:, d].cpu().float(), torch.from_numpy(-np.sign(h) * np.inf).float())
    others = torch.arange(Dm) != d
    assert same_bits(outs[0][:, others], outs[1][:, others])

"""The serving calls on the GPU against the CPU oracle, sequence by sequence: packed prompts, single tokens on slots, the FFN-MoE of a few tokens, and
a run of them together with the layer's own calls.  Bounds follow the arithmetic (serving_testlib.py)."""
import numpy as np
import pytest
import torch

from oracle import rom_oracle as O
from paper_2506_18145_b200 import binding as rb
from paper_2506_18145_b200 import synth

from rom_testlib import TOL, assert_close, np64
from serving_testlib import (HALF_STEP, TORCH, U32, Packed, check, conv_reference, pool_with_junk, randn, same_bits, scan_reference, silu_bound, wide)

pytestmark = pytest.mark.gpu

SENTINEL = -77.0


def config(d_inner, dtype, d_conv=4, disc_mode=0, B=1, L=1):
    return rb.make_config(B, L, 64, d_inner, 16, d_conv, 16, 1, 1, dtype, disc_mode=disc_mode)


def pools(seed, p, shape, std, in_place):
    """(pool to read, pool to write, the written one's bits before)."""
    src = pool_with_junk(seed, p, shape, std).cuda()
    dst = src if in_place else torch.full_like(src, SENTINEL)
    return src, dst, dst.clone()


# ---------------------------------------------------------------------------------------------- conv over packed sequences
def run_conv(p, De, dtype, d_conv=4, bias=True, in_place=True, with_pools=True, left=64, right=8):
    x = randn(1, (p.rows, De), dtype=TORCH[dtype])
    x[~torch.from_numpy(p.mine())] = float("nan")
    w, b = randn(2, (d_conv, De), 0.5, TORCH[dtype]), randn(3, (De,), 0.1) if bias else None
    src, dst, before = pools(4, p, (d_conv - 1, De), 1.0, in_place)
    y = torch.full((p.rows, De), SENTINEL, dtype=TORCH[dtype], device="cuda")
    old = src.cpu().double().numpy()
    rb.rom_conv_ragged(config(De, dtype, d_conv), p.ragged, wide(x, left, right), w.cuda(), None if b is None else b.cuda(), src if with_pools else None,
                       dst if with_pools else None, y)
    torch.cuda.synchronize()
    touched = set()
    for i in range(p.n):
        a, e = p.start[i], p.start[i + 1]
        past = old[p.slots[i]] if with_pools and p.resumes(i) else np.zeros((d_conv - 1, De))
        pre, size, win = conv_reference(np64(x[a:e]), np64(w), np64(b), past)
        check(y[a:e], O.silu(pre), silu_bound(pre, (d_conv + 1) * U32 * size), dtype, f"sequence {i}")
        if p.kept(i) and with_pools:
            touched.add(int(p.slots[i]))
            np.testing.assert_array_equal(np64(dst[p.slots[i]]), win, err_msg=f"window of sequence {i}")
    outside = torch.from_numpy(~p.mine()).cuda()
    assert torch.all(y[outside] == SENTINEL)
    for s in range(p.n_slots):
        if s not in touched:
            assert same_bits(dst[s], before[s]), f"slot {s} was written"


LENGTHS = {"one": [1], "tokens": [1] * 33, "short": [0, 2, 3, 0, 1, 5, 0], "prompts": [37, 16, 1, 0, 130, 15, 17, 2, 64], "all empty": [0, 0, 0],
           "borders": [16, 16, 13, 3, 14, 2, 15, 1, 16, 0, 31, 1, 4], "long": [700, 1, 333]}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", LENGTHS)
def test_conv_ragged_lengths(lens, dtype):
    run_conv(Packed(LENGTHS[lens], lead=0, tail=0, seed=5), 192, dtype)


@pytest.mark.parametrize("dtype,d_conv,De,bias,in_place,lead,tail", [
    ("bf16", 2, 64, False, True, 3, 21), ("bf16", 3, 320, True, False, 0, 1), ("f32", 2, 128, True, False, 17, 0), ("f32", 3, 64, False, True, 1, 40), ("bf16", 4, 2112, True, True, 5, 5)])
def test_conv_ragged_shapes(dtype, d_conv, De, bias, in_place, lead, tail):
    run_conv(Packed(LENGTHS["borders"], lead=lead, tail=tail, seed=6), De, dtype, d_conv, bias, in_place)


def test_conv_ragged_slots_outside_the_pool_and_without_pools():
    lens = [5, 20, 3, 40]
    run_conv(Packed(lens, seed=7, n_slots=4, slots=[-1, 2, 4, 1 << 30], resume=[1, 1, 1, 1]), 64, "bf16")
    run_conv(Packed(lens, seed=7, resume=[1, 1, 1, 1]), 64, "f32", with_pools=False)


def test_conv_ragged_many_sequences():
    g = np.random.default_rng(11)
    run_conv(Packed(g.integers(0, 4, 1500), seed=8), 64, "bf16")


# ---------------------------------------------------------------------------------------------- scan over packed sequences
def scan_inputs(rows, De, dtype, seed=0, dt=(1e-3, 1e-1)):
    g = torch.Generator()
    g.manual_seed(900 + seed)
    lo, hi = np.log(dt[0]), np.log(dt[1])
    return dict(u=randn(21 + seed, (rows, De), dtype=TORCH[dtype]), delta=torch.exp(torch.rand((rows, De), generator=g) * (hi - lo) + lo),
                A=-(torch.arange(1, 17).float()[None] * (0.5 + torch.rand((De, 16), generator=g))).contiguous(), Bm=randn(22 + seed, (rows, 16)),
                Cm=randn(23 + seed, (rows, 16)), D=1.0 + randn(24 + seed, (De,), 0.1), z=randn(25 + seed, (rows, De), dtype=TORCH[dtype]))


def run_scan(p, De, dtype, disc_mode=0, skip=True, gate=True, in_place=True, with_pools=True, dt=(1e-3, 1e-1), seed=0):
    s = scan_inputs(p.rows, De, dtype, seed, dt)
    outside = torch.from_numpy(~p.mine())
    for n in ("u", "delta", "Bm", "Cm", "z"):
        s[n][outside] = float("nan")
    s["D"] = s["D"] if skip else None
    s["z"] = s["z"] if gate else None
    src, dst, before = pools(26, p, (De, 16), 0.3, in_place)
    old = src.cpu().double().numpy()
    y = torch.full((p.rows, De), SENTINEL, dtype=TORCH[dtype], device="cuda")
    cfg = config(De, dtype, disc_mode=disc_mode)
    ws = torch.full((rb.scan_ragged_workspace_size(cfg, p.n, p.rows),), 255, dtype=torch.uint8, device="cuda")
    d = {n: None if v is None else v.cuda() for n, v in s.items()}
    k = 8 if seed % 2 == 0 else 5                       # columns before B and C: on a 16-byte boundary or off it
    bc = torch.cat([torch.full((p.rows, k), float("nan")), s["Bm"], s["Cm"]], 1).cuda()
    rb.rom_scan_ragged(cfg, p.ragged, d["u"], d["delta"], d["A"], bc[:, k:k + 16], bc[:, k + 16:], d["D"], wide(s["z"], De, 8) if gate else None,
                       src if with_pools else None, dst if with_pools else None, y, ws)
    torch.cuda.synchronize()
    touched = set()
    for i in range(p.n):
        a, e = p.start[i], p.start[i + 1]
        h0 = old[p.slots[i]] if with_pools and p.resumes(i) else np.zeros((De, 16))
        ref, bound, h, G = scan_reference(np64(s["u"][a:e]), np64(s["delta"][a:e]), np64(s["A"]), np64(s["Bm"][a:e]), np64(s["Cm"][a:e]), np64(s["D"]),
                                          None if not gate else np64(s["z"][a:e]), h0, disc_mode)
        check(y[a:e], ref, bound, dtype, f"sequence {i}")
        if p.kept(i) and with_pools:
            touched.add(int(p.slots[i]))
            check(dst[p.slots[i]], h, G, "f32", f"state of sequence {i}")
    assert torch.all(y[outside.cuda()] == SENTINEL)
    for q in range(p.n_slots):
        if q not in touched:
            assert same_bits(dst[q], before[q]), f"slot {q} was written"
    return y, dst


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", LENGTHS)
def test_scan_ragged_lengths(lens, dtype):
    run_scan(Packed(LENGTHS[lens], seed=5), 192, dtype)


@pytest.mark.parametrize("dtype,disc_mode,De,skip,gate,in_place,lead,tail", [
    ("bf16", 1, 64, False, True, True, 3, 21), ("bf16", 0, 320, True, False, False, 0, 1), ("f32", 1, 128, True, False, False, 17, 0),
    ("f32", 0, 64, False, True, True, 1, 40), ("bf16", 0, 1088, True, True, True, 5, 5)])
def test_scan_ragged_shapes(dtype, disc_mode, De, skip, gate, in_place, lead, tail):
    run_scan(Packed(LENGTHS["borders"], lead=lead, tail=tail, seed=6), De, dtype, disc_mode, skip, gate, in_place)
    run_scan(Packed(LENGTHS["prompts"], lead=lead, tail=tail, seed=6), De, dtype, disc_mode, skip, gate, in_place, seed=1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("in_place", [True, False])
def test_scan_ragged_long_sequences_cross_many_chunks(dtype, in_place):
    run_scan(Packed([2500, 0, 1, 640, 3, 1711], lead=2, tail=9, seed=9, resume=[1, 1, 0, 1, 1, 0]), 64, dtype, in_place=in_place)


@pytest.mark.parametrize("dt", [(1e-6, 1e-5), (0.5, 60.0)])
@pytest.mark.parametrize("disc_mode", [0, 1])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scan_ragged_small_and_large_steps(dtype, disc_mode, dt):
    run_scan(Packed([300, 41], seed=10, resume=[1, 1]), 64, dtype, disc_mode, dt=dt)


def test_scan_ragged_slots_outside_the_pool_and_without_pools():
    lens = [5, 200, 3, 40]
    run_scan(Packed(lens, seed=7, n_slots=4, slots=[-1, 2, 4, 1 << 30], resume=[1, 1, 1, 1]), 64, "bf16")
    run_scan(Packed(lens, seed=7, resume=[1, 1, 1, 1]), 64, "f32", with_pools=False)


def test_scan_ragged_many_sequences():
    g = np.random.default_rng(12)
    run_scan(Packed(g.integers(0, 4, 1500), seed=8), 64, "bf16")


def test_scan_ragged_is_the_same_run_to_run():
    p = Packed([900, 31, 0, 1400, 77], seed=13, resume=[1] * 5)
    a = [run_scan(p, 128, "bf16", in_place=False) for _ in range(2)]
    assert same_bits(a[0][0], a[1][0]) and same_bits(a[0][1], a[1][1])


# ---------------------------------------------------------------------------------------------- single tokens
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,De,d_conv,padded,in_place", [(1, 64, 4, False, True), (3, 2112, 2, True, False), (37, 192, 3, True, True), (130, 256, 4, False, False)])
def test_conv_step(B, De, d_conv, padded, in_place, dtype):
    p = Packed([1] * B, seed=B, resume=[1] * B)
    if padded:
        p.slots[::4] = -1
        p.slots[1] = p.n_slots
    x, w, b = randn(31, (B, De), dtype=TORCH[dtype]), randn(32, (d_conv, De), 0.5, TORCH[dtype]), randn(33, (De,), 0.1) if B != 3 else None
    src, dst, before = pools(34, p, (d_conv - 1, De), 1.0, in_place)
    old = np64(src)
    y = torch.full((B, De), SENTINEL, dtype=TORCH[dtype], device="cuda")
    rb.rom_conv_step(config(De, dtype, d_conv, B=B), wide(x, 8, 64), w.cuda(), None if b is None else b.cuda(), torch.from_numpy(p.slots).cuda(), src, dst, y)
    torch.cuda.synchronize()
    for i in range(B):
        if not p.kept(i):
            assert torch.all(y[i] == SENTINEL)
            continue
        pre, size, win = conv_reference(np64(x[i:i + 1]), np64(w), np64(b), old[p.slots[i]])
        check(y[i:i + 1], O.silu(pre), silu_bound(pre, (d_conv + 1) * U32 * size), dtype, f"token {i}")
        np.testing.assert_array_equal(np64(dst[p.slots[i]]), win)
    for s in set(range(p.n_slots)) - {int(q) for q in p.slots}:
        assert same_bits(dst[s], before[s])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,De,disc_mode,skip,gate,padded,in_place", [(1, 64, 0, True, True, False, True), (3, 1088, 1, False, True, True, False), (37, 192, 0, True, False, True, True),
                                                                     (130, 256, 1, True, True, False, False)])
def test_scan_step(B, De, disc_mode, skip, gate, padded, in_place, dtype):
    p = Packed([1] * B, seed=B, resume=[1] * B)
    if padded:
        p.slots[::4] = -1
        p.slots[1] = p.n_slots
    s = scan_inputs(B, De, dtype)
    s["D"] = s["D"] if skip else None
    s["z"] = s["z"] if gate else None
    src, dst, before = pools(35, p, (De, 16), 0.3, in_place)
    old = np64(src)
    y = torch.full((B, De), SENTINEL, dtype=TORCH[dtype], device="cuda")
    d = {n: None if v is None else v.cuda() for n, v in s.items()}
    k = B % 4                                           # columns before B and C: on a 16-byte boundary or off it
    bc = torch.cat([torch.full((B, k), float("nan")), s["Bm"], s["Cm"]], 1).cuda()
    rb.rom_scan_step(config(De, dtype, disc_mode=disc_mode, B=B), d["u"], d["delta"], d["A"], bc[:, k:k + 16], bc[:, k + 16:], d["D"], wide(s["z"], 8, 0) if gate else None,
                     torch.from_numpy(p.slots).cuda(), src, dst, y)
    torch.cuda.synchronize()
    for i in range(B):
        if not p.kept(i):
            assert torch.all(y[i] == SENTINEL)
            continue
        ref, bound, h, G = scan_reference(np64(s["u"][i:i + 1]), np64(s["delta"][i:i + 1]), np64(s["A"]), np64(s["Bm"][i:i + 1]), np64(s["Cm"][i:i + 1]), np64(s["D"]),
                                          np64(s["z"][i:i + 1]) if gate else None, old[p.slots[i]], disc_mode)
        check(y[i:i + 1], ref, bound, dtype, f"token {i}")
        check(dst[p.slots[i]], h, G, "f32", f"state {i}")
    for q in set(range(p.n_slots)) - {int(v) for v in p.slots}:
        assert same_bits(dst[q], before[q])


@pytest.mark.parametrize("disc_mode", [0, 1])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scans_of_a_state_that_grows(dtype, disc_mode):
    """Negative steps: the state grows, by up to e here, which makes every error of a step up to e times the one that the bound counts."""
    B, De = 6, 64
    p = Packed([1] * B, seed=51, resume=[1] * B)
    s = scan_inputs(B, De, dtype, seed=51)
    g = torch.Generator()
    g.manual_seed(52)
    s["delta"] = -torch.rand((B, De), generator=g)
    s["A"] = -(0.5 + 0.5 * torch.rand((De, 16), generator=g))
    cfg = config(De, dtype, disc_mode=disc_mode, B=B)
    h0 = randn(53, (p.n_slots, De, 16), 0.3)
    d = {n: v.cuda() for n, v in s.items()}
    outs = []
    for step in (True, False):
        h, y = h0.cuda(), torch.empty(B, De, dtype=TORCH[dtype], device="cuda")
        if step:
            rb.rom_scan_step(cfg, d["u"], d["delta"], d["A"], d["Bm"], d["Cm"], d["D"], d["z"], p.dev[1], h, h, y)
        else:
            ws = torch.empty(rb.scan_ragged_workspace_size(cfg, B, B), dtype=torch.uint8, device="cuda")
            rb.rom_scan_ragged(cfg, p.ragged, d["u"], d["delta"], d["A"], d["Bm"], d["Cm"], d["D"], d["z"], h, h, y, ws)
        outs.append((y, h))
    torch.cuda.synchronize()
    for y, h in outs:
        for i in range(B):
            ref, bound, last, G = scan_reference(np64(s["u"][i:i + 1]), np64(s["delta"][i:i + 1]), np64(s["A"]), np64(s["Bm"][i:i + 1]), np64(s["Cm"][i:i + 1]),
                                                 np64(s["D"]), np64(s["z"][i:i + 1]), np64(h0[p.slots[i]]), disc_mode)
            check(y[i:i + 1], ref, np.e * bound, dtype, f"token {i}")
            check(h[p.slots[i]], last, np.e * G, "f32", f"state {i}")


def test_steps_in_slot_order_without_a_table():
    B, De = 5, 64
    cfg = config(De, "f32", B=B)
    x, w = randn(41, (B, De)), randn(42, (4, De), 0.5)
    win = randn(43, (B, 3, De)).cuda()
    got = [torch.empty(B, De, device="cuda") for _ in range(2)]
    outs = [torch.empty_like(win) for _ in range(2)]
    for y, o, slot in zip(got, outs, (None, torch.arange(B, dtype=torch.int32, device="cuda"))):
        rb.rom_conv_step(cfg, x.cuda(), w.cuda(), None, slot, win, o, y)
    assert torch.equal(*got) and torch.equal(*outs)


# ---------------------------------------------------------------------------------------------- FFN-MoE of a few tokens
def run_ffn(B, Dm, F, E, K, dtype, idx=None, seed=0, L=1):
    T = B * L
    x, W_gu, W_down = randn(51 + seed, (T, Dm), dtype=TORCH[dtype]), randn(52, (E, 2 * F, Dm), Dm ** -0.5, TORCH[dtype]), randn(53, (E, Dm, F), F ** -0.5, TORCH[dtype])
    g = np.random.default_rng(seed)
    if idx is None:
        idx = np.stack([g.permutation(E)[:K] for _ in range(T)])
    idx = np.asarray(idx, dtype=np.int32).reshape(T, K)
    gates = g.random((T, K)).astype(np.float32)
    cfg = rb.make_config(B, L, Dm, 64, 16, 4, 16, E, K, dtype)
    ws = torch.full((rb.ffn_moe_step_workspace_size(cfg, F),), 255, dtype=torch.uint8, device="cuda")
    out = torch.full((T, Dm), float("nan"), dtype=TORCH[dtype], device="cuda")
    rb.rom_ffn_moe_step(cfg, F, W_gu.cuda(), W_down.cuda(), x.cuda(), torch.from_numpy(idx).cuda(), torch.from_numpy(gates).cuda(), out, ws)
    torch.cuda.synchronize()
    assert rb.rom_get_status(ws) == (-1 if (idx >= E).any() else 0)
    # reference and bound: a sum of n products in fp32 is at most 2 n U of its |terms| off (tensor cores may cut instead of rounding), the
    # hidden row is stored in half a step, the output too
    X, Wg, Wd = np64(x), np64(W_gu), np64(W_down)
    ref, bound = np.zeros((T, Dm)), np.zeros((T, Dm))
    for t in range(T):
        for k in range(K):
            e = idx[t, k]
            if not 0 <= e < E:
                continue
            gu, size = Wg[e] @ X[t], np.abs(Wg[e]) @ np.abs(X[t])
            a, b = gu[:F], gu[F:]
            ea, eb = 2 * Dm * U32 * size[:F], 2 * Dm * U32 * size[F:]
            h = O.silu(a) * b * gates[t, k]
            eh = gates[t, k] * (silu_bound(a, ea) * (np.abs(b) + eb) + np.abs(O.silu(a)) * eb) + 4 * U32 * np.abs(h)
            eh = eh + HALF_STEP[dtype] * (np.abs(h) + eh)
            ref[t] += Wd[e] @ h
            bound[t] += np.abs(Wd[e]) @ eh + 2 * F * U32 * (np.abs(Wd[e]) @ np.abs(h)) + 2 * K * U32 * np.abs(Wd[e] @ h)
    check(out, ref, bound, dtype, "out")
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,Dm,F,E,K", [
    (1, 64, 128, 1, 1), (1, 256, 512, 8, 1), (2, 192, 384, 4, 2), (5, 128, 256, 4, 3), (16, 128, 128, 2, 1), (17, 320, 640, 3, 2), (33, 64, 256, 1, 1),
    (64, 128, 256, 8, 2), (64, 64, 128, 64, 8), (9, 64, 128, 40, 8), (3, 1088, 896, 5, 2)])
def test_ffn_step(B, Dm, F, E, K, dtype):
    run_ffn(B, Dm, F, E, K, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ffn_step_padding_repeated_and_bad_experts(dtype):
    run_ffn(4, 64, 128, 4, 2, dtype, idx=[[1, 3], [-1, -1], [2, -1], [0, 0]])
    run_ffn(3, 64, 128, 4, 2, dtype, idx=[[-1, -1], [-1, -1], [-7, -1]])
    run_ffn(3, 64, 128, 4, 2, dtype, idx=[[4, 1], [0, 1 << 30], [2, 3]])
    run_ffn(64, 64, 128, 2, 2, dtype, idx=np.ones((64, 2)))      # one expert has 128 assignments


def test_ffn_step_agrees_with_the_forward():
    """Both round the hidden row to bf16 (the step with its gate in it) and the output; an error of one rounding each way."""
    B, Dm, F, E, K = 24, 256, 512, 8, 2
    out = run_ffn(B, Dm, F, E, K, "bf16", L=1)
    x, W_gu, W_down = randn(51, (B, Dm), dtype=torch.bfloat16), randn(52, (E, 2 * F, Dm), Dm ** -0.5, torch.bfloat16), randn(53, (E, Dm, F), F ** -0.5, torch.bfloat16)
    g = np.random.default_rng(0)
    idx = np.stack([g.permutation(E)[:K] for _ in range(B)]).astype(np.int32)
    gates = g.random((B, K)).astype(np.float32)
    cfg = rb.make_config(B, 1, Dm, 64, 16, 4, 16, E, K, "bf16")
    ws = torch.empty(rb.ffn_moe_workspace_size(cfg, F), dtype=torch.uint8, device="cuda")
    ref = torch.empty_like(out)
    rb.rom_ffn_moe_forward(cfg, F, W_gu.cuda(), W_down.cuda(), x.cuda(), torch.from_numpy(idx).cuda(), torch.from_numpy(gates).cuda(), ref, ws)
    torch.cuda.synchronize()
    assert_close(np64(out), np64(ref), TOL["bf16"], "step against forward")


# ---------------------------------------------------------------------------------------------- uses that the calls above do not make
def test_offsets_past_the_buffers_are_cut():
    """seq_start beyond `rows`: the sequences end with the buffers."""
    De, rows = 64, 50
    p = Packed([20, 30], seed=14, resume=[1, 1])
    long = Packed([20, 30], seed=14, resume=[1, 1])
    long.dev[0][2] = 1 << 30
    s = scan_inputs(rows, De, "bf16")
    d = {n: v.cuda() for n, v in s.items()}
    cfg = config(De, "bf16")
    ws = torch.empty(rb.scan_ragged_workspace_size(cfg, 2, rows), dtype=torch.uint8, device="cuda")
    got = []
    for q in (p, long):
        h, win = pool_with_junk(15, q, (De, 16), 0.3).cuda(), pool_with_junk(16, q, (3, De), 1.0).cuda()
        y, v = torch.zeros_like(d["u"]), torch.zeros_like(d["u"])
        rb.rom_scan_ragged(cfg, q.ragged, d["u"], d["delta"], d["A"], d["Bm"], d["Cm"], d["D"], d["z"], h, h, y, ws)
        rb.rom_conv_ragged(cfg, q.ragged, d["u"], d["z"][:4].contiguous(), d["D"], win, win, v)
        got.append((y, h, v, win))
    for a, b in zip(*got):
        assert same_bits(a, b)


def test_no_sequences_launch_nothing():
    cfg = config(64, "f32")
    none = rb.make_ragged(10, 4, torch.zeros(1, dtype=torch.int32, device="cuda"))
    y = torch.full((10, 64), SENTINEL, device="cuda")
    rb.rom_conv_ragged(cfg, none, torch.zeros(10, 64, device="cuda"), torch.zeros(4, 64, device="cuda"), None, None, None, y)
    assert torch.all(y == SENTINEL)


def test_without_rows_fresh_states_are_zeroed_and_others_kept():
    """A batch of empty sequences with buffers of no rows at all."""
    De = 128
    p = Packed([0, 0, 0], seed=17, resume=[1, 0, 1])
    cfg = config(De, "bf16")
    e = lambda *shape, t=torch.bfloat16: torch.empty(shape, dtype=t, device="cuda")
    for in_place in (True, False):
        h, ho, _ = pools(18, p, (De, 16), 0.3, in_place)
        win, wo, _ = pools(19, p, (3, De), 1.0, in_place)
        hb, wb = h.clone(), win.clone()
        ws = torch.empty(rb.scan_ragged_workspace_size(cfg, 3, 0), dtype=torch.uint8, device="cuda")
        rb.rom_scan_ragged(cfg, p.ragged, e(0, De), e(0, De, t=torch.float32), -torch.ones(De, 16, device="cuda"), e(0, 16, t=torch.float32), e(0, 16, t=torch.float32), None, None,
                           h, ho, e(0, De), ws)
        rb.rom_conv_ragged(cfg, p.ragged, e(0, De), torch.ones(4, De, dtype=torch.bfloat16, device="cuda"), None, win, wo, e(0, De))
        torch.cuda.synchronize()
        for i in range(3):
            q = int(p.slots[i])
            for now, before in ((ho, hb), (wo, wb)):
                assert same_bits(now[q], before[q] if p.resume[i] else torch.zeros_like(before[q]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_that_are_not_finite_stay_in_their_sequence(dtype):
    De = 64
    p = Packed([30, 4, 1, 200, 9, 55], seed=20, resume=[1] * 6)
    cfg = config(De, dtype)
    s = scan_inputs(p.rows, De, dtype)
    clean = {n: v.cuda() for n, v in s.items()}
    dirty = {n: v.clone() for n, v in clean.items()}
    bad = (1, 3)
    for i in bad:
        dirty["u"][p.start[i]:p.start[i + 1]] = float("nan") if i == 1 else float("inf")
        dirty["Bm"][p.start[i]] = float("inf")
    ws = torch.empty(rb.scan_ragged_workspace_size(cfg, p.n, p.rows), dtype=torch.uint8, device="cuda")
    got = []
    for d in (clean, dirty):
        h, win = pool_with_junk(21, p, (De, 16), 0.3).cuda(), pool_with_junk(22, p, (3, De), 1.0).cuda()
        y, v = torch.zeros_like(d["u"]), torch.zeros_like(d["u"])
        rb.rom_scan_ragged(cfg, p.ragged, d["u"], d["delta"], d["A"], d["Bm"], d["Cm"], d["D"], d["z"], h, h, y, ws)
        rb.rom_conv_ragged(cfg, p.ragged, d["u"], clean["z"][:4].contiguous(), None, win, win, v)
        got.append((y, v, h, win))
    for i in range(p.n):
        rows, slot = slice(p.start[i], p.start[i + 1]), int(p.slots[i])
        for k, (a, b) in enumerate(zip(*got)):
            at = rows if k < 2 else slot
            assert same_bits(a[at], b[at]) == (i not in bad)


def test_ffn_step_values_that_are_not_finite_stay_in_their_token():
    B, Dm, F, E, K = 20, 128, 256, 4, 2
    x, W_gu, W_down = randn(71, (B, Dm), dtype=torch.bfloat16).cuda(), randn(72, (E, 2 * F, Dm), Dm ** -0.5, torch.bfloat16).cuda(), randn(73, (E, Dm, F), F ** -0.5, torch.bfloat16).cuda()
    g = np.random.default_rng(3)
    idx = torch.from_numpy(np.stack([g.permutation(E)[:K] for _ in range(B)]).astype(np.int32)).cuda()
    gates = torch.full((B, K), 0.5, device="cuda")
    cfg = rb.make_config(B, 1, Dm, 64, 16, 4, 16, E, K, "bf16")
    ws = torch.empty(rb.ffn_moe_step_workspace_size(cfg, F), dtype=torch.uint8, device="cuda")
    outs = []
    for bad in (False, True):
        if bad:
            x[7] = float("nan")
        outs.append(torch.empty_like(x))
        rb.rom_ffn_moe_step(cfg, F, W_gu, W_down, x, idx, gates, outs[-1], ws)
    keep = torch.arange(B, device="cuda") != 7
    assert same_bits(outs[0][keep], outs[1][keep]) and torch.all(torch.isnan(outs[1][7]))


def test_captured_calls_replay_on_new_inputs():
    """All serving calls in one graph on a stream of their own, replayed after the inputs, lengths and slots have changed in place."""
    De, dtype, B, Dm, F, E, K = 128, "bf16", 6, 128, 256, 4, 2
    cfg, step, ffn = config(De, dtype), config(De, dtype, B=B), rb.make_config(B, 1, Dm, 64, 16, 4, 16, E, K, dtype)
    p = Packed([40, 7, 0, 90], tail=30, seed=23, resume=[1, 0, 1, 1], n_slots=8)
    s = {n: v.cuda() for n, v in scan_inputs(p.rows, De, dtype).items()}
    t = {n: v.cuda() for n, v in scan_inputs(B, De, dtype, seed=2).items()}
    w = randn(81, (4, De), 0.5, TORCH[dtype]).cuda()
    slot = torch.tensor([3, 0, -1, 7, 5, 1], dtype=torch.int32, device="cuda")
    x, W_gu, W_down = randn(82, (B, Dm), dtype=TORCH[dtype]).cuda(), randn(83, (E, 2 * F, Dm), Dm ** -0.5, TORCH[dtype]).cuda(), randn(84, (E, Dm, F), F ** -0.5, TORCH[dtype]).cuda()
    idx, gates = torch.tensor([[0, 1], [2, 3], [-1, -1], [1, 3], [0, 2], [3, 0]], dtype=torch.int32, device="cuda"), torch.full((B, K), 0.5, device="cuda")
    h0, win0 = randn(85, (8, De, 16), 0.3).cuda(), randn(86, (8, 3, De)).cuda()
    h, win = h0.clone(), win0.clone()
    ws, ffn_ws = (torch.empty(n, dtype=torch.uint8, device="cuda") for n in (rb.scan_ragged_workspace_size(cfg, p.n, p.rows), rb.ffn_moe_step_workspace_size(ffn, F)))
    outs = [torch.zeros_like(s["u"]) for _ in range(2)] + [torch.zeros_like(t["u"]) for _ in range(2)] + [torch.zeros_like(x)]

    def calls():
        rb.rom_conv_ragged(cfg, p.ragged, s["u"], w, None, win, win, outs[0])
        rb.rom_scan_ragged(cfg, p.ragged, outs[0], s["delta"], s["A"], s["Bm"], s["Cm"], s["D"], s["z"], h, h, outs[1], ws)
        rb.rom_conv_step(step, t["u"], w, None, slot, win, win, outs[2])
        rb.rom_scan_step(step, outs[2], t["delta"], s["A"], t["Bm"], t["Cm"], s["D"], t["z"], slot, h, h, outs[3])
        rb.rom_ffn_moe_step(ffn, F, W_gu, W_down, x, idx, gates, outs[4], ffn_ws)

    def reset():
        h.copy_(h0)
        win.copy_(win0)
        for o in outs:
            o.zero_()

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        calls()
    stream.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        calls()
    for change in range(2):
        if change:
            p.dev[0].copy_(torch.tensor([0, 3, 3, 60, 160], dtype=torch.int32))
            p.dev[1].copy_(torch.tensor([6, 2, 4, 0], dtype=torch.int32))
            slot.copy_(torch.tensor([1, -1, 6, 2, 4, 0], dtype=torch.int32))
            idx.copy_(idx.flip(0))
            for v in (s["u"], t["u"], x):
                v.mul_(-0.5)
        reset()
        calls()
        torch.cuda.synchronize()
        want = [v.clone() for v in outs + [h, win]]
        reset()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs + [h, win], want):
            assert same_bits(a, b)


def test_calls_on_two_streams_at_once():
    """Each with its own workspace and outputs: as one after the other."""
    De, F, Dm, E, K, B = 512, 1024, 512, 8, 2, 32
    p = Packed([600, 1, 0, 333], seed=24, resume=[0] * 4)
    cfg, ffn = config(De, "bf16"), rb.make_config(B, 1, Dm, 64, 16, 4, 16, E, K, "bf16")
    s = {n: v.cuda() for n, v in scan_inputs(p.rows, De, "bf16").items()}
    x, W_gu, W_down = randn(91, (B, Dm), dtype=torch.bfloat16).cuda(), randn(92, (E, 2 * F, Dm), Dm ** -0.5, torch.bfloat16).cuda(), randn(93, (E, Dm, F), F ** -0.5, torch.bfloat16).cuda()
    g = np.random.default_rng(5)
    idx, gates = torch.from_numpy(np.stack([g.permutation(E)[:K] for _ in range(B)]).astype(np.int32)).cuda(), torch.full((B, K), 0.25, device="cuda")
    sets = []
    for i in range(2):
        sets.append(dict(stream=torch.cuda.Stream(), ws=torch.empty(rb.scan_ragged_workspace_size(cfg, p.n, p.rows), dtype=torch.uint8, device="cuda"),
                         fws=torch.empty(rb.ffn_moe_step_workspace_size(ffn, F), dtype=torch.uint8, device="cuda"), y=torch.zeros_like(s["u"]), h=torch.zeros(p.n_slots, De, 16, device="cuda"),
                         out=torch.zeros_like(x)))
    torch.cuda.synchronize()
    for _ in range(5):
        for q in sets:
            rb.rom_scan_ragged(cfg, p.ragged, s["u"], s["delta"], s["A"], s["Bm"], s["Cm"], s["D"], s["z"], None, q["h"], q["y"], q["ws"], stream=q["stream"])
            rb.rom_ffn_moe_step(ffn, F, W_gu, W_down, x, idx, gates, q["out"], q["fws"], stream=q["stream"])
    torch.cuda.synchronize()
    for n in ("y", "h", "out"):
        assert same_bits(sets[0][n], sets[1][n])
    assert rb.rom_get_status(sets[0]["fws"]) == 0 and rb.rom_get_status(sets[1]["fws"]) == 0


def test_offsets_past_32_bits():
    """Pools and packed buffers of more than 2^31 elements: the last slot and the last rows."""
    De, n_slots = 4096, (1 << 31) // (4096 * 16) + 2
    cfg = config(De, "bf16", B=1)
    s = scan_inputs(1, De, "bf16")
    d = {n: v.cuda() for n, v in s.items()}
    pool = torch.empty((n_slots, De, 16), device="cuda")
    pool[-1] = randn(95, (De, 16), 0.3).cuda()
    h0 = np64(pool[-1])
    slot = torch.tensor([n_slots - 1], dtype=torch.int32, device="cuda")
    y = torch.empty_like(d["u"])
    rb.rom_scan_step(cfg, d["u"], d["delta"], d["A"], d["Bm"], d["Cm"], d["D"], d["z"], slot, pool, pool, y)
    ref, bound, h, G = scan_reference(*(np64(s[n]) for n in ("u", "delta", "A", "Bm", "Cm", "D", "z")), h0, 0)
    check(y, ref, bound, "bf16", "token")
    check(pool[-1], h, G, "f32", "state")
    del pool
    rows = (1 << 31) // De + 70
    p = Packed([rows - 19, 19], seed=25, resume=[0, 0])
    x = torch.zeros((rows, De), dtype=torch.bfloat16, device="cuda")
    last = randn(96, (40, De), dtype=torch.bfloat16)
    x[-40:] = last.cuda()
    w = randn(97, (4, De), 0.5, torch.bfloat16)
    v, win = torch.empty_like(x), torch.empty((p.n_slots, 3, De), device="cuda")
    rb.rom_conv_ragged(cfg, p.ragged, x, w.cuda(), None, None, win, v)
    pre, size, want = conv_reference(np64(last[-19:]), np64(w), None, np.zeros((3, De)))
    check(v[-19:], O.silu(pre), silu_bound(pre, 5 * U32 * size), "bf16", "last rows")
    np.testing.assert_array_equal(np64(win[int(p.slots[1])]), want)
    np.testing.assert_array_equal(np64(win[int(p.slots[0])]), np64(last[18:21]))


def test_tensors_of_another_device_are_refused(monkeypatch):
    cfg = config(64, "f32", B=1)
    t = torch.zeros(1, 64, device="cuda")
    win = torch.zeros(1, 3, 64, device="cuda")
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(ValueError, match="device"):
        rb.rom_conv_step(cfg, t, torch.zeros(4, 64, device="cuda"), None, None, win, win, torch.zeros_like(t))


# ---------------------------------------------------------------------------------------------- all of them as a server uses them
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prompts_then_tokens_then_ffn(dtype):
    """Prompts of several lengths packed through conv and scan, their states handed to rom_layer_step in slots, tokens generated by it and, beside it, by
    rom_conv_step and rom_scan_step; the FFN-MoE on the step's routing.  The oracle runs every whole sequence at once."""
    s = synth.RomShape("serve", 4, 23, 128, 256, 16, 4, 16, 2, 1, dtype, 4242)
    p = synth.make_inputs(s, recipe="unit")
    W = {k: None if v is None else v.cuda() for k, v in p.items()}
    f = lambda k: None if p[k] is None else np64(p[k])
    prompt, new = [20, 3, 11, 1], 2
    ref, im = O.rom_layer_forward(f("x"), f("W_r"), f("b_r"), f("W_inz"), f("w_conv"), f("b_conv"), f("W_x"), f("W_dt"), f("b_dt"), f("A"), f("D"), f("W_out"), K=1,
                                  dt_rank=s.dt_rank, return_intermediates=True)
    idx_all = im["idx"].reshape(s.B, s.L)
    De, R, td = s.d_inner, s.dt_rank, TORCH[dtype]
    # prompts: rows packed, every projection in torch (the layer's own are not split into calls)
    rows = [(b, t) for b in range(s.B) for t in range(prompt[b])]
    x = torch.stack([W["x"][b, t] for b, t in rows])
    experts = torch.tensor([int(idx_all[b, t]) for b, t in rows], device="cuda")
    XZ = torch.einsum("rd,rfd->rf", x.double(), W["W_inz"][experts].double()).to(td)

    def small(U):
        dbl = U.double() @ W["W_x"].double().t()
        delta = torch.nn.functional.softplus(dbl[:, :R].to(td).double() @ W["W_dt"].double().t() + W["b_dt"].double()).float()
        return delta, dbl[:, R:R + 16].float().contiguous(), dbl[:, R + 16:].float().contiguous()

    pk = Packed(prompt, n_slots=s.B, slots=np.arange(s.B), resume=[0] * s.B, tail=2)
    pad = lambda v: torch.cat([v, torch.full((2, v.shape[1]), float("nan"), dtype=v.dtype, device="cuda")])
    cfg = rb.config_from_shape(s.replace(L=1))
    win, h = torch.full((s.B, 3, De), float("nan"), device="cuda"), torch.full((s.B, De, 16), float("nan"), device="cuda")
    XZp = pad(XZ)
    U, Yg = torch.zeros((pk.rows, De), dtype=td, device="cuda"), torch.zeros((pk.rows, De), dtype=td, device="cuda")
    rb.rom_conv_ragged(cfg, pk.ragged, XZp[:, :De], W["w_conv"], W["b_conv"], None, win, U)
    delta, Bm, Cm = small(U[:-2])
    ws = torch.empty(rb.scan_ragged_workspace_size(cfg, pk.n, pk.rows), dtype=torch.uint8, device="cuda")
    rb.rom_scan_ragged(cfg, pk.ragged, U, pad(delta), W["A"], pad(Bm), pad(Cm), W["D"], XZp[:, De:], None, h, Yg, ws)
    gates = torch.from_numpy(im["gate"].reshape(s.B, s.L)).float().cuda()
    O_p = torch.einsum("rc,rdc->rd", Yg[:-2].double(), W["W_out"][experts].double())
    for i, (b, t) in enumerate(rows):
        O_p[i] *= gates[b, t]
    want = np.stack([ref.reshape(s.B, s.L, -1)[b, t] for b, t in rows])
    assert_close(np64(O_p), want, TOL[dtype], "prompts")
    # tokens: the layer's step on the pools, and the slot calls beside it on copies of them
    layer_ws = rb.alloc_workspace(cfg)
    win2, h2 = win.clone(), h.clone()
    out, yt, ut = torch.empty((s.B, s.d_model), dtype=td, device="cuda"), torch.empty((s.B, De), dtype=td, device="cuda"), torch.empty((s.B, De), dtype=td, device="cuda")
    idx, gate = torch.empty((s.B, 1), dtype=torch.int32, device="cuda"), torch.empty((s.B, 1), device="cuda")
    slot = torch.arange(s.B, dtype=torch.int32, device="cuda")
    F = 256
    W_gu, W_down = randn(61, (s.E, 2 * F, s.d_model), s.d_model ** -0.5, td).cuda(), randn(62, (s.E, s.d_model, F), F ** -0.5, td).cuda()
    ffn_ws, ffn_out = torch.empty(rb.ffn_moe_step_workspace_size(cfg, F), dtype=torch.uint8, device="cuda"), torch.empty_like(out)
    for k in range(new):
        xt = torch.stack([W["x"][b, prompt[b] + k] for b in range(s.B)]).contiguous()
        rb.rom_layer_step(cfg, rb.make_weights(W), xt, win, h, out, idx, gate, layer_ws)
        want = np.stack([ref.reshape(s.B, s.L, -1)[b, prompt[b] + k] for b in range(s.B)])
        assert_close(np64(out), want, TOL[dtype], f"token {k}")
        e = idx[:, 0].long()
        XZt = torch.einsum("rd,rfd->rf", xt.double(), W["W_inz"][e].double()).to(td)
        rb.rom_conv_step(cfg, XZt[:, :De], W["w_conv"], W["b_conv"], slot, win2, win2, ut)
        delta, Bm, Cm = small(ut)
        rb.rom_scan_step(cfg, ut, delta, W["A"], Bm, Cm, W["D"], XZt[:, De:], slot, h2, h2, yt)
        O_t = torch.einsum("rc,rdc->rd", yt.double(), W["W_out"][e].double()) * gate.double()
        assert_close(np64(O_t), want, TOL[dtype], f"token {k} by the slot calls")
        rb.rom_ffn_moe_step(cfg, F, W_gu, W_down, out, idx, gate, ffn_out, ffn_ws)
        ffn = O.ffn_moe_shared_routing(np64(out), np64(W_gu), np64(W_down), idx.cpu().numpy(), np64(gate))
        assert_close(np64(ffn_out), ffn.reshape(s.B, -1), TOL[dtype], f"FFN-MoE of token {k}")
    assert_close(np64(h), np64(h2), TOL[dtype], "states")
    assert rb.rom_get_status(layer_ws) == 0 and rb.rom_get_status(ffn_ws) == 0

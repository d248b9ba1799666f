"""The serving calls at sizes where their launch rules take the other side: tiles of many rows, two tokens a warp, long chunks, blocks that walk many tiles of
weights.  Each test states by which rule its size gets there, so that a change of the rule shows."""
import math
import os

import numpy as np
import pytest
import torch

from paper_2506_18145_b200 import binding as rb
from paper_2506_18145_b200 import build as rbuild

from rom_testlib import np64
from serving_testlib import TORCH, U32, Packed, check, randn, same_bits, scan_reference
from test_gpu_serving import SENTINEL, config, run_conv, scan_inputs

pytestmark = pytest.mark.gpu


def source_says(file, *texts):
    with open(os.path.join(rbuild.CSRC, file)) as f:
        s = f.read()
    for t in texts:
        assert t in s, f"{file} has another rule now: the sizes of this test are for {t!r}"


# ---------------------------------------------------------------------------------------------- conv over packed sequences
def mixed_lengths(seed, rows, tile):
    """Lengths of `rows` rows in all: many of 0 to 5, some around the tile's, some of several tiles."""
    g = np.random.default_rng(seed)
    lens = []
    while sum(lens) < rows:
        kind = g.integers(0, 8)
        lens.append(int(g.integers(0, 6)) if kind < 4 else int(g.integers(max(tile - 2, 0), tile + 3)) if kind < 6 else int(g.integers(tile, 4 * tile + 20)))
    lens[-1] -= sum(lens) - rows
    return lens


@pytest.mark.parametrize("dtype,De,rows,tile,lead,tail,in_place", [
    ("bf16", 4160, 260, 2, 0, 0, True), ("bf16", 4160, 960, 7, 3, 1, False), ("bf16", 2112, 4160, 16, 0, 17, True), ("bf16", 4160, 4700, 32, 33, 40, True),
    ("f32", 4160, 120, 2, 1, 1, False), ("f32", 2112, 940, 7, 0, 3, True), ("f32", 4160, 1130, 16, 5, 0, True), ("f32", 4160, 2400, 32, 0, 30, False)])
def test_conv_ragged_tiles_of_many_rows(dtype, De, rows, tile, lead, tail, in_place):
    source_says("rom_conv_ragged.cu", "kConvWarps = 148 * 16", "(cb * s.rows + kConvWarps - 1) / kConvWarps", "fit > 32 ? 32", "CR_ROWS = 4")
    p = Packed(mixed_lengths(rows, rows, tile), lead=lead, tail=tail, seed=61)
    groups = -(-De // (256 if dtype == "bf16" else 128))
    assert min(-(-groups * p.rows // (148 * 16)), 32) == tile
    run_conv(p, De, dtype, in_place=in_place)


@pytest.mark.parametrize("d_conv", [2, 3])
def test_conv_ragged_tiles_of_many_rows_of_narrow_windows(d_conv):
    run_conv(Packed(mixed_lengths(7, 4700, 32), lead=2, tail=11, seed=62), 4096, "bf16", d_conv)


# ---------------------------------------------------------------------------------------------- scan of single tokens
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,De,disc_mode,padded,in_place", [(75, 4096, 0, True, True), (73, 4096, 1, False, False), (131, 2304, 0, True, False), (146, 2112, 1, True, True)])
def test_scan_step_two_tokens_a_warp(B, De, disc_mode, padded, in_place, dtype):
    source_says("rom_serve_step.cu", "kSlotBlocks = 148 * 32", "(long long)(c.d_inner / 32) * ((c.B + SS_WARPS - 1) / SS_WARPS) >= kSlotBlocks", "SS_WARPS = 2")
    assert De // 32 * -(-B // 2) >= 148 * 32
    g = np.random.default_rng(B)
    n_slots = B + 5
    slots = g.permutation(n_slots)[:B].astype(np.int32)
    if padded:
        slots[::5] = -1
        slots[1] = n_slots
    s = scan_inputs(B, De, dtype, seed=2)
    h0 = randn(63, (n_slots, De, 16), 0.3)
    used = set(int(v) for v in slots)
    for q in range(n_slots):
        if q not in used:
            h0[q] = float("nan")
    src = h0.cuda()
    dst = src if in_place else torch.full_like(src, SENTINEL)
    before = dst.clone()
    d = {n: v.cuda() for n, v in s.items()}
    y = torch.full((B, De), SENTINEL, dtype=TORCH[dtype], device="cuda")
    rb.rom_scan_step(config(De, dtype, disc_mode=disc_mode, B=B), d["u"], d["delta"], d["A"], d["Bm"], d["Cm"], d["D"], d["z"], torch.from_numpy(slots).cuda(), src, dst, y)
    torch.cuda.synchronize()
    f = {n: np64(v) for n, v in s.items()}
    for i in range(B):
        if not 0 <= slots[i] < n_slots:
            assert torch.all(y[i] == SENTINEL)
            continue
        row = slice(i, i + 1)
        ref, bound, h, G = scan_reference(f["u"][row], f["delta"][row], f["A"], f["Bm"][row], f["Cm"][row], f["D"], f["z"][row], np64(h0[slots[i]]), disc_mode)
        check(y[row], ref, bound, dtype, f"token {i}")
        check(dst[slots[i]], h, G, "f32", f"state {i}")
    for q in set(range(n_slots)) - used:
        assert same_bits(dst[q], before[q])


# ---------------------------------------------------------------------------------------------- scan over packed sequences
@pytest.mark.parametrize("lens,De,dtype,disc_mode,in_place", [
    # chunks of 48 rows and more (83 of them at most): sequences over many chunks, over one end, inside one
    ([5000, 40, 0, 1, 2200, 900], 4096, "bf16", 0, True), ([1] * 60 + [7000, 333, 2, 2], 4096, "bf16", 1, False), ([3500, 33, 0, 1400], 4096, "f32", 0, True),
    # 1792 warps a chunk: the first launch's blocks do not all run at once, and the second waits for all of them to be gone
    ([12, 1, 30, 0, 9, 14, 3, 25] * 16, 57344, "bf16", 0, True), ([12, 1, 30, 0, 9, 14, 3, 25] * 16, 57344, "f32", 1, False)])
def test_scan_ragged_long_chunks_and_many_blocks(lens, De, dtype, disc_mode, in_place):
    """All channels are computed, some of each block compared with the reference (no channel depends on another)."""
    source_says("rom_scan_ragged.cu", "148 * 12 * 6 / (De / 32)", "(long long)l.nch * (De / 32) <= 148ll * RWARPS * (c.dtype == ROM_F32 ? 2 : 3)", "RWARPS = 4")
    p = Packed(lens, lead=3, tail=21, seed=64)
    assert De // 32 > 148 * 12 or p.rows / min(148 * 12 * 6 // (De // 32), 512) >= 48
    g = torch.Generator(device="cuda")
    g.manual_seed(65)
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda")
    uniform = lambda *shape: torch.rand(shape, generator=g, device="cuda")
    mine = torch.from_numpy(p.mine()).cuda()[:, None]
    nan = torch.tensor(float("nan"), device="cuda")
    own = lambda v, t=torch.float32: torch.where(mine, v, nan).to(t)
    u, z = own(normal(p.rows, De), TORCH[dtype]), own(normal(p.rows, De), TORCH[dtype])
    delta = own(torch.exp(uniform(p.rows, De) * math.log(100.0) + math.log(1e-3)))
    Bm, Cm = own(normal(p.rows, 16)), own(normal(p.rows, 16))
    A = -(torch.arange(1, 17, device="cuda").float()[None] * (0.5 + uniform(De, 16)))
    D = 1.0 + 0.1 * normal(De)
    src = 0.3 * normal(p.n_slots, De, 16)
    h0 = src.clone()
    dst = src if in_place else torch.full_like(src, SENTINEL)
    before = dst.clone()
    y = torch.full((p.rows, De), SENTINEL, dtype=TORCH[dtype], device="cuda")
    cfg = config(De, dtype, disc_mode=disc_mode)
    ws = torch.full((rb.scan_ragged_workspace_size(cfg, p.n, p.rows),), 255, dtype=torch.uint8, device="cuda")
    rb.rom_scan_ragged(cfg, p.ragged, u, delta, A, Bm, Cm, D, z, src, dst, y, ws)
    torch.cuda.synchronize()
    assert rb.lib().rom_last_launch_count() == 2      # (chunks, that is)
    at = torch.cat([torch.arange(32), torch.arange(De - 32, De), torch.randint(0, De, (32,), generator=torch.Generator().manual_seed(66))]).cuda()
    f = {n: np64(v[:, at]) for n, v in dict(u=u, z=z, delta=delta).items()}
    Bn, Cn, An, Dn = np64(Bm), np64(Cm), np64(A[at]), np64(D[at])
    for i in range(p.n):
        r = slice(p.start[i], p.start[i + 1])
        first = np64(h0[p.slots[i]][at]) if p.resumes(i) else np.zeros((len(at), 16))
        ref, bound, h, G = scan_reference(f["u"][r], f["delta"][r], An, Bn[r], Cn[r], Dn, f["z"][r], first, disc_mode)
        check(y[r][:, at], ref, bound, dtype, f"sequence {i}")
        check(dst[p.slots[i]][at], h, G, "f32", f"state of sequence {i}")
    assert torch.all(torch.isfinite(y.float())) and torch.all(y[~mine[:, 0]] == SENTINEL)
    for q in set(range(p.n_slots)) - {int(v) for v in p.slots}:
        assert same_bits(dst[q], before[q])


# ---------------------------------------------------------------------------------------------- FFN-MoE of a few tokens
@pytest.mark.parametrize("B,Dm,F,E,K,choice", [
    (64, 2048, 8192, 16, 2, "any"),        # sixteen columns an expert, some of 32; every block walks many tiles of several experts
    (1, 2048, 8192, 8, 1, "any"),          # one token: the contracted index in parts
    (24, 1088, 8320, 4, 2, "any"),         # odd numbers of 64-element blocks and of tiles
    (64, 2048, 8192, 2, 1, "any"),         # 32 tokens an expert: 64 columns, two passes of the down projection
    (64, 2048, 16384, 4, 2, "same"),        # one expert has 128 assignments: two passes of 64, four of 32
    (40, 512, 8192, 40, 8, "any"),         # many experts of a few tokens
])
def test_ffn_step_blocks_walk_many_tiles(B, Dm, F, E, K, choice):
    """Against 64 bits on the GPU.  A tile has 64 hidden columns or 128 output rows at most and takes stages of 128 contracted elements, a ring has twelve stages at
    most: the blocks refill their rings several times (with one token the second launch's less)."""
    source_says("rom_ffn_step.cu", "FT_KB = 2, FT_K = FT_KB * BLOCK_K", "FT_MAX_STAGES = 12", "for (int h = up ? 64 : 128;", "want > 32 && up ? 64")
    g = torch.Generator(device="cuda")
    g.manual_seed(B + F)
    normal = lambda shape, std: (torch.randn(shape, generator=g, device="cuda") * std).bfloat16()
    x, W_gu, W_down = normal((B, Dm), 1.0), normal((E, 2 * F, Dm), Dm ** -0.5), normal((E, Dm, F), F ** -0.5)
    order = torch.rand((B, E), generator=g, device="cuda")
    idx = (torch.topk(order, K, dim=1).indices if choice == "any" else torch.ones((B, K), device="cuda")).to(torch.int32).contiguous()
    gates = torch.rand((B, K), generator=g, device="cuda")
    chosen = len(torch.unique(idx))
    rings = 2 if B > 1 else 1
    assert chosen * -(-F // 64) * -(-Dm // 128) >= 148 * 12 * rings and chosen * -(-Dm // 128) * -(-F // 128) >= 148 * 6 * rings
    cfg = rb.make_config(B, 1, Dm, 64, 16, 4, 16, E, K, "bf16")
    ws = torch.full((rb.ffn_moe_step_workspace_size(cfg, F),), 255, dtype=torch.uint8, device="cuda")
    outs = []
    for _ in range(3):                     # (the second finds the first's numbers in the workspace)
        out = torch.full((B, Dm), float("nan"), dtype=torch.bfloat16, device="cuda")
        rb.rom_ffn_moe_step(cfg, F, W_gu, W_down, x, idx, gates, out, ws)
        outs.append(out)
    torch.cuda.synchronize()
    assert rb.rom_get_status(ws) == 0 and same_bits(outs[0], outs[1]) and same_bits(outs[0], outs[2])
    # the bound of test_ffn_step_hidden_rows (a hidden row is held within 2^-16)
    ref, bound = torch.zeros((B, Dm), dtype=torch.float64, device="cuda"), torch.zeros((B, Dm), dtype=torch.float64, device="cuda")
    for e in range(E):
        for k in range(K):
            t = torch.nonzero(idx[:, k] == e)[:, 0]
            if not len(t):
                continue
            X, Wg, Wd, gate = x[t].double(), W_gu[e].double(), W_down[e].double(), gates[t, k].double()[:, None]
            gu, size = X @ Wg.t(), X.abs() @ Wg.abs().t()
            a, b, ea, eb = gu[:, :F], gu[:, F:], 2 * Dm * U32 * size[:, :F], 2 * Dm * U32 * size[:, F:]
            s = a * torch.sigmoid(a)
            es = 1.1 * ea + (8.0 + 2.0 * a.abs()) * U32 * s.abs()
            h = s * b * gate
            eh = gate * (es * (b.abs() + eb) + s.abs() * eb) + (2.0 ** -16 + 4 * U32) * h.abs()
            ref[t] += h @ Wd.t()
            bound[t] += eh @ Wd.abs().t() + 4 * F * U32 * (h.abs() @ Wd.abs().t()) + 2 * K * U32 * (h @ Wd.t()).abs()
    check(outs[0], np64(ref), np64(bound), "bf16", "out")
    # the sums' bound grows with their length, their error with its root: all outputs together are hardly further off than their own rounding
    assert (outs[0].double() - ref).norm() <= 1.1 * (ref.bfloat16().double() - ref).norm()

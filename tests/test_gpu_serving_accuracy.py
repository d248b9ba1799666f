"""How exact the serving calls are: bounds that only what a call promises satisfies (the bounds of serving_testlib.py allow the hidden rows of the FFN and the
inputs of the scan more than that), and values that are not finite."""
import numpy as np
import pytest
import torch

from oracle import rom_oracle as O
from paper_2506_18145_b200 import binding as rb

from rom_testlib import np64
from serving_testlib import TORCH, U32, check, randn, silu_bound

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

"""What the binding's serving calls and the workspace sizes refuse or promise: no GPU needed, the library is a stand-in that notes the calls which reach it."""
import types

import pytest
import torch

from paper_2506_18145_b200 import binding as rb

B, ROWS, SLOTS, DE, DM, F, E, K = 3, 10, 4, 64, 64, 128, 4, 2
BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


@pytest.fixture
def calls(monkeypatch):
    """Names of the library's functions that were called; tensors of the host count as those of the current device."""
    seen = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: seen.append(name) or 0

    monkeypatch.setattr(rb, "lib", Library)
    monkeypatch.setattr(rb.torch, "cuda", types.SimpleNamespace(current_device=lambda: -1))
    monkeypatch.setattr(rb, "_stream", lambda stream, device=None: 0)
    return seen


def tensors(dtype):
    """Arguments of every call, all of the sizes that it needs and no larger."""
    z = lambda *shape, t=dtype: torch.zeros(shape, dtype=t)
    seqs = rb.RomRagged(2, ROWS, SLOTS, 0, 0, 0)
    cfg = rb.make_config(B, 1, DM, DE, 16, 4, 16, E, K, dtype)
    scan = dict(u=z(ROWS, DE), delta=z(ROWS, DE, t=F32), A=z(DE, 16, t=F32), Bm=z(ROWS, 16, t=F32), Cm=z(ROWS, 16, t=F32), D=z(DE, t=F32), z=z(ROWS, DE))
    return {
        "rom_conv_ragged": (cfg, dict(seqs=seqs), dict(x=z(ROWS, DE), w_conv=z(4, DE), b_conv=z(DE, t=F32), win_in=z(SLOTS, 3, DE, t=F32), win_out=z(SLOTS, 3, DE, t=F32), y=z(ROWS, DE))),
        "rom_scan_ragged": (cfg, dict(seqs=seqs, ws=torch.zeros(64, dtype=torch.uint8)),
                            dict(scan, h_in=z(SLOTS, DE, 16, t=F32), h_out=z(SLOTS, DE, 16, t=F32), y=z(ROWS, DE))),
        "rom_conv_step": (cfg, {}, dict(x=z(B, DE), w_conv=z(4, DE), b_conv=z(DE, t=F32), slot=z(B, t=I32), win_in=z(SLOTS, 3, DE, t=F32), win_out=z(SLOTS, 3, DE, t=F32), y=z(B, DE))),
        "rom_scan_step": (cfg, {}, dict({n: v if n in ("A", "D") else v[:B].contiguous() for n, v in scan.items()}, slot=z(B, t=I32), h_in=z(SLOTS, DE, 16, t=F32),
                                        h_out=z(SLOTS, DE, 16, t=F32), y=z(B, DE))),
        "rom_ffn_moe_step": (cfg, dict(d_ff=F, ws=torch.zeros(64, dtype=torch.uint8)),
                             dict(W_gu=z(E, 2 * F, DM), W_down=z(E, DM, F), x=z(B, DM), topk_idx=z(B, K, t=I32), gates=z(B, K, t=F32), out=z(B, DM))),
    }


NAMES = list(tensors(BF))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("name", NAMES)
def test_tensors_of_the_sizes_that_a_call_needs(calls, name, dtype):
    cfg, fixed, t = tensors(dtype)[name]
    getattr(rb, name)(cfg, **fixed, **t)
    larger = {n: torch.cat([v, v[:1]]) for n, v in t.items()}      # (a longer buffer will do)
    getattr(rb, name)(cfg, **fixed, **larger)
    assert calls == [name] * 2


@pytest.mark.parametrize("name,tensor", [(n, t) for n in NAMES for t in tensors(BF)[n][2]])
def test_a_tensor_that_is_too_small_or_of_another_type(calls, name, tensor):
    cfg, fixed, t = tensors(BF)[name]
    short = t[tensor][:-1].contiguous()
    other = t[tensor].to(torch.float16 if t[tensor].dtype is not I32 else torch.int64)
    swapped = t[tensor].to(F32 if t[tensor].dtype is BF else BF)
    if t[tensor].dim() == 2:
        narrow = t[tensor][:, :-1].contiguous()
    else:
        narrow = short
    for bad in (short, narrow, other, swapped):
        with pytest.raises(ValueError):
            getattr(rb, name)(cfg, **fixed, **{**t, tensor: bad})
    assert calls == []


@pytest.mark.parametrize("name", ["rom_conv_ragged", "rom_scan_ragged"])
def test_sequences_that_name_more_than_there_is(calls, name):
    cfg, fixed, t = tensors(BF)[name]
    for seqs in (rb.RomRagged(2, ROWS + 1, SLOTS, 0, 0, 0), rb.RomRagged(2, ROWS, SLOTS + 1, 0, 0, 0)):
        with pytest.raises(ValueError):
            getattr(rb, name)(cfg, **{**fixed, "seqs": seqs}, **t)
    assert calls == []


def test_packed_conv_in_place_is_refused(calls):
    """Rows of one block are the taps of the next one's."""
    cfg, fixed, t = tensors(BF)["rom_conv_ragged"]
    with pytest.raises(ValueError, match="y is x"):
        rb.rom_conv_ragged(cfg, **fixed, **{**t, "y": t["x"]})
    assert calls == []


# ---------------------------------------------------------------------------------------------- workspaces
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d_inner", [64, 256, 1024, 2048, 4096, 8192])
def test_scan_workspace_of_the_largest_batch_does_for_all_smaller_ones(d_inner, dtype):
    cfg = rb.make_config(1, 1, 64, d_inner, 16, 4, 16, 1, 1, dtype)
    size = lambda n, r: rb.scan_ragged_workspace_size(cfg, n, r)
    rows = [0, 1, 7, 8, 15, 16, 17, 100, 500, 777, 1024, 2000, 4096, 8000, 8192, 16384, 30000, 1 << 20]
    seqs = [0, 1, 2, 5, 8, 23, 64, 500, 5000]
    for i, r in enumerate(rows):
        for j, n in enumerate(seqs):
            assert all(size(n, r) >= size(m, q) for q in rows[:i + 1] for m in seqs[:j + 1][-2:]), (n, r)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d_model,d_ff,experts,K", [(2048, 8192, 16, 2), (1280, 5120, 8, 1), (256, 1024, 4, 2), (4096, 4096, 64, 8), (64, 128, 1, 1), (512, 2048, 16, 2)])
def test_ffn_step_workspace_of_the_largest_batch_does_for_all_smaller_ones(d_model, d_ff, experts, K, dtype):
    sizes = [rb.ffn_moe_step_workspace_size(rb.make_config(n, 1, d_model, 64, 16, 4, 16, experts, K, dtype), d_ff) for n in range(1, 65)]
    assert sizes == sorted(sizes)

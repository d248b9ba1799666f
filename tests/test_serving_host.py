"""Host-side checks of the serving calls (packed sequences, single tokens on slots, FFN-MoE of a few tokens): no GPU needed, nothing is launched."""
import ctypes

import pytest
import torch

from paper_2506_18145_b200 import binding as rb
from paper_2506_18145_b200 import build as rbuild

P = 1 << 20      # a made-up address: never dereferenced, every call here ends before a launch
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, -1, -2, -3


@pytest.fixture(scope="module")
def L():
    rbuild.build()
    return rb.lib()


def cfg_of(**kw):
    base = dict(B=4, L=1, d_model=128, d_inner=256, d_state=16, d_conv=4, dt_rank=16, E=4, K=2, dtype="bf16")
    base.update(kw)
    return rb.make_config(**base)


def ragged(**kw):
    base = dict(n_seq=3, rows=100, n_slots=8, seq_start=P, slot=P, resume=P)
    base.update(kw)
    return rb.RomRagged(*base.values())


def conv_ragged(L, cfg=None, r=None, **kw):
    a = dict(x=P, ldx=256, w=P, b=P, win_in=P, win_out=P, y=P)
    a.update(kw)
    return L.rom_conv_ragged(ctypes.byref(cfg or cfg_of()), ctypes.byref(r or ragged()), *a.values(), None)


def scan_ragged(L, cfg=None, r=None, **kw):
    a = dict(u=P, delta=P, A=P, Bm=P, Cm=P, ld_bc=16, D=P, z=P, ldz=256, h_in=P, h_out=P, y=P, ws=P, ws_bytes=1 << 40)
    a.update(kw)
    return L.rom_scan_ragged(ctypes.byref(cfg or cfg_of()), ctypes.byref(r or ragged()), *a.values(), None)


def conv_step(L, cfg=None, **kw):
    a = dict(x=P, ldx=256, w=P, b=P, slot=P, n_slots=8, win_in=P, win_out=P, y=P)
    a.update(kw)
    return L.rom_conv_step(ctypes.byref(cfg or cfg_of()), *a.values(), None)


def scan_step(L, cfg=None, **kw):
    a = dict(u=P, delta=P, A=P, Bm=P, Cm=P, ld_bc=16, D=P, z=P, ldz=256, slot=P, n_slots=8, h_in=P, h_out=P, y=P)
    a.update(kw)
    return L.rom_scan_step(ctypes.byref(cfg or cfg_of()), *a.values(), None)


def ffn_step(L, cfg=None, **kw):
    a = dict(d_ff=256, W_gu=P, W_down=P, x=P, idx=P, gates=P, out=P, ws=P, ws_bytes=1 << 40)
    a.update(kw)
    return L.rom_ffn_moe_step(ctypes.byref(cfg or cfg_of()), *a.values(), None)


CALLS = {"conv_ragged": conv_ragged, "scan_ragged": scan_ragged, "conv_step": conv_step, "scan_step": scan_step, "ffn_step": ffn_step}


@pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses must not get past the checks on a machine with a device")
@pytest.mark.parametrize("name", CALLS)
def test_without_a_device_a_good_call_fails_for_the_device_alone(L, name):
    assert CALLS[name](L) in (-4, -5)


@pytest.mark.parametrize("name,bad", [
    ("conv_ragged", ["x", "w", "y"]), ("scan_ragged", ["u", "delta", "A", "Bm", "Cm", "y", "ws"]), ("conv_step", ["x", "w", "win_in", "win_out", "y"]),
    ("scan_step", ["u", "delta", "A", "Bm", "Cm", "h_in", "h_out", "y"]), ("ffn_step", ["W_gu", "W_down", "x", "idx", "gates", "out", "ws"])])
def test_missing_pointers(L, name, bad):
    for a in bad:
        assert CALLS[name](L, **{a: None}) == INVALID, a


@pytest.mark.parametrize("name,by16,by4", [
    ("conv_ragged", ["x", "w", "win_in", "win_out", "y"], ["b"]), ("scan_ragged", ["u", "delta", "A", "z", "h_in", "h_out", "y", "ws"], ["D", "Bm", "Cm"]),
    ("conv_step", ["x", "w", "win_in", "win_out", "y"], ["b", "slot"]), ("scan_step", ["u", "delta", "A", "z", "h_in", "h_out", "y"], ["D", "slot", "Bm", "Cm"]),
    ("ffn_step", ["W_gu", "W_down", "x", "out", "ws"], ["idx", "gates"])])
def test_misaligned_pointers(L, name, by16, by4):
    for a in by16:
        assert CALLS[name](L, **{a: P + 8}) == INVALID, a
    for a in by4:
        assert CALLS[name](L, **{a: P + 2}) == INVALID, a


@pytest.mark.parametrize("name", ["conv_ragged", "scan_ragged", "conv_step", "scan_step"])
def test_configs_that_the_slot_calls_refuse(L, name):
    call = CALLS[name]
    for kw, code in [(dict(d_inner=100), INVALID), (dict(d_inner=0), INVALID), (dict(d_state=8), UNSUPPORTED), (dict(B=0), INVALID), (dict(flags=16), INVALID),
                     (dict(disc_mode=2), INVALID)]:
        assert call(L, cfg_of(**kw)) == code, kw
    if name.startswith("conv"):
        assert call(L, cfg_of(d_conv=5)) == UNSUPPORTED and call(L, cfg_of(d_conv=1)) == UNSUPPORTED and call(L, cfg_of(d_conv=0)) == INVALID
        assert call(L, ldx=252) == INVALID and call(L, ldx=260) == INVALID and call(L, ldx=-256) == INVALID
        assert call(L, cfg_of(dtype="f32"), ldx=258) == INVALID
    else:
        assert call(L, ldz=128) == INVALID and call(L, ldz=258) == INVALID
        assert call(L, ld_bc=12) == INVALID and call(L, ld_bc=-16) == INVALID
    if name.endswith("step"):
        assert call(L, cfg_of(L=2)) == INVALID and call(L, n_slots=-1) == INVALID


@pytest.mark.parametrize("name", ["conv_ragged", "scan_ragged"])
def test_packed_sequences_that_are_refused(L, name):
    call = CALLS[name]
    for kw, code in [(dict(n_seq=-1), INVALID), (dict(rows=-1), INVALID), (dict(n_slots=-1), INVALID), (dict(seq_start=None), INVALID), (dict(seq_start=P + 2), INVALID),
                     (dict(slot=P + 1), INVALID), (dict(resume=P + 1), INVALID), (dict(n_seq=(1 << 20) + 1), UNSUPPORTED), (dict(rows=1 << 30), UNSUPPORTED)]:
        assert call(L, None, ragged(**kw)) == code, kw
    assert call(L, None, ragged(n_seq=0, seq_start=None)) == OK      # nothing to do


@pytest.mark.parametrize("name,a,b", [("conv_ragged", "win_in", "win_out"), ("scan_ragged", "h_in", "h_out"), ("conv_step", "win_in", "win_out"), ("scan_step", "h_in", "h_out")])
def test_pools_are_one_buffer_or_two_that_do_not_overlap(L, name, a, b):
    n = 8 * 256 * (3 if name.startswith("conv") else 16) * 4
    assert CALLS[name](L, **{a: P, b: P + n - 16}) == INVALID
    assert CALLS[name](L, **{a: P + 16, b: P}) == INVALID


def test_ffn_step_configs(L):
    for kw, code in [(dict(B=65), UNSUPPORTED), (dict(B=9, L=8), UNSUPPORTED), (dict(K=5), INVALID), (dict(K=0), INVALID), (dict(E=65, K=1), UNSUPPORTED),
                     (dict(E=16, K=9), UNSUPPORTED), (dict(d_model=96), INVALID), (dict(flags=1), INVALID), (dict(B=0), INVALID)]:
        assert ffn_step(L, cfg_of(**kw)) == code, kw
    assert ffn_step(L, d_ff=0) == INVALID and ffn_step(L, d_ff=192) == UNSUPPORTED


def test_workspaces(L):
    cfg = cfg_of()
    need = rb.ffn_moe_step_workspace_size(cfg, 256)
    assert ffn_step(L, cfg, ws_bytes=need - 1) == WORKSPACE
    need = rb.scan_ragged_workspace_size(cfg, 3, 100)
    assert scan_ragged(L, cfg, ws_bytes=need - 1) == WORKSPACE
    assert L.rom_scan_ragged_workspace_size(ctypes.byref(cfg), 3, 100, None) == INVALID
    n = ctypes.c_size_t(0)
    for args, code in [((-1, 100), INVALID), ((3, -1), INVALID), ((3, 1 << 30), UNSUPPORTED), (((1 << 20) + 1, 100), UNSUPPORTED), ((0, 0), OK)]:
        assert L.rom_scan_ragged_workspace_size(ctypes.byref(cfg), *args, ctypes.byref(n)) == code
    for c, d_ff in [(cfg_of(B=65), 256), (cfg, 100)]:
        with pytest.raises(rb.RomError):
            rb.ffn_moe_step_workspace_size(c, d_ff)


def test_binding_refuses_what_it_cannot_describe():
    rows = torch.zeros(4, 64)
    with pytest.raises(ValueError, match="device"):
        rb._rows_at(rows, 0)                                                  # not on a GPU
    with pytest.raises(ValueError, match="device"):
        rb._at(rows, 0)
    with pytest.raises(ValueError, match="contiguous"):
        rb._at(rows.t(), -1)
    with pytest.raises(ValueError, match="contiguous"):
        rb._rows_at(rows.t(), -1)
    assert rb._rows_at(torch.zeros(4, 96)[:, 32:], -1)[1] == 96 and rb._rows_at(torch.zeros(1, 96)[:, 32:], -1)[1] == 64
    i32 = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        rb.make_ragged(10, 4, i32.long())
    with pytest.raises(ValueError):
        rb.make_ragged(10, 4, i32, slot=i32)                                  # three sequences, four slots
    with pytest.raises(ValueError):
        rb._slots(torch.zeros(3, 2), torch.zeros(4, 2))
    assert rb._slots(None, torch.zeros(4, 2)) == 0
    elsewhere = ragged()
    elsewhere.device = 1
    with pytest.raises(ValueError, match="cuda:1"):
        rb._sequences(elsewhere, 0)

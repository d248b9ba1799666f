"""Linear attention and the norm and rotation of its queries and keys: the formulas' gradients against differences, and what the calls refuse on the host.  No GPU."""
import ctypes

import pytest
import torch

from paper_2506_18145_b200 import binding as rb
from paper_2506_18145_b200 import build as rbuild

import linattn_testlib as T

P = 1 << 20      # a made-up address: never dereferenced, every call here ends before a launch
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, -1, -2, -3


@pytest.fixture(scope="module")
def L():
    rbuild.build()
    return rb.lib()


def randn(g, *shape):
    return torch.randn(shape, generator=g, dtype=torch.float64)


# ---------------------------------------------------------------------------------------------- the formulas
@pytest.mark.parametrize("n,H,G,dk,dv", [(1, 2, 1, 8, 8), (7, 4, 2, 8, 16), (12, 3, 3, 16, 8)])
def test_closed_form_is_the_recurrence(n, H, G, dk, dv):
    g = torch.Generator().manual_seed(n)
    q, k, v, S0, rate = randn(g, n, G, dk), randn(g, n, G, dk), randn(g, n, H, dv), randn(g, H, dk, dv), -torch.rand(H, generator=g, dtype=torch.float64)
    o, S = T.forward(q, k, v, rate, S0, 0.3)
    for h in range(H):
        state = S0[h].clone()
        for t in range(n):
            state = torch.exp(rate[h]) * state + torch.outer(k[t, h * G // H], v[t, h])
            assert torch.allclose(o[t, h], 0.3 * q[t, h * G // H] @ state)
        assert torch.allclose(S[h], state)


@pytest.mark.parametrize("n,H,G,dk,dv", [(1, 1, 1, 8, 8), (9, 4, 2, 8, 16), (6, 3, 1, 16, 8)])
def test_gradient_formula_against_differences(n, H, G, dk, dv):
    g = torch.Generator().manual_seed(n + 40)
    x = [randn(g, n, G, dk), randn(g, n, G, dk), randn(g, n, H, dv), randn(g, H, dk, dv)]
    rate, do, dS = -torch.rand(H, generator=g, dtype=torch.float64), randn(g, n, H, dv), randn(g, H, dk, dv)

    def loss(x):
        o, S = T.forward(x[0], x[1], x[2], rate, x[3], 0.7)
        return (o * do).sum() + (S * dS).sum()

    dq, dk_, dv_, dS0 = T.backward(do, x[0], x[1], x[2], rate, x[3], dS, 0.7)
    for i, grad in enumerate((dq, dk_, dv_, dS0)):
        way = randn(g, *x[i].shape)
        step = 1e-5
        ends = [loss([y + s * step * way if j == i else y for j, y in enumerate(x)]) for s in (1.0, -1.0)]
        want = float((ends[0] - ends[1]) / (2 * step))
        # the loss is at most quadratic in each input: the central difference is exact up to rounding, 2^-53 of the terms' sum over the step
        assert abs(want - float((grad * way).sum())) <= 1e-8 * max(1.0, float((grad * way).abs().sum()))


@pytest.mark.parametrize("rot,interleaved", [(0, False), (16, False), (16, True), (32, False), (32, True)])
def test_norm_and_rotation_gradient_against_differences(rot, interleaved):
    g = torch.Generator().manual_seed(rot + interleaved)
    x, w, dy = randn(g, 3, 2, 32), randn(g, 32), randn(g, 3, 2, 32)
    pos, freq = torch.tensor([0, 5, 70000]), torch.rand(rot // 2, generator=g, dtype=torch.float64)
    loss = lambda x, w: (T.norm_rope(x, w, pos, freq, rot, interleaved, 1e-3) * dy).sum()  # noqa: E731
    dx, dw, _ = T.norm_rope_backward(dy, x, w, pos, freq, rot, interleaved, 1e-3)
    step = 1e-6
    for grad, at in ((dx, 0), (dw, 1)):
        way = randn(g, *grad.shape)
        ends = [loss(x + s * step * way, w) if at == 0 else loss(x, w + s * step * way) for s in (1.0, -1.0)]
        assert abs(float((ends[0] - ends[1]) / (2 * step)) - float((grad * way).sum())) <= 1e-7 * float((grad * way).abs().sum())


# ---------------------------------------------------------------------------------------------- refusals
def lin_cfg(**kw):
    base = dict(n_heads=4, n_qk_heads=2, d_k=64, d_v=32, dtype=rb.ROM_BF16, flags=0, scale=0.125)
    base.update(kw)
    return rb.RomLinattnConfig(*base.values())


def ragged(**kw):
    base = dict(n_seq=3, rows=100, n_slots=8, seq_start=P, slot=P, resume=P)
    base.update(kw)
    return rb.RomRagged(*base.values())


POOL = 8 * 4 * 64 * 32 * 4


def lin_ragged(L, cfg=None, r=None, **kw):
    a = dict(q=2 * P, ldq=128, k=3 * P, ldk=128, v=4 * P, ldv=128, g=P, s_in=P, s_out=P, o=5 * P, ws=P, ws_bytes=1 << 40)
    a.update(kw)
    return L.rom_linattn_ragged(ctypes.byref(cfg or lin_cfg()), ctypes.byref(r or ragged()), *a.values(), None)


def lin_step(L, cfg=None, r=None, **kw):
    a = dict(B=4, q=2 * P, ldq=128, k=3 * P, ldk=128, v=4 * P, ldv=128, g=P, slot=P, n_slots=8, s_in=P, s_out=P, o=5 * P)
    a.update(kw)
    return L.rom_linattn_step(ctypes.byref(cfg or lin_cfg()), *a.values(), None)


def lin_backward(L, cfg=None, r=None, **kw):
    a = dict(do=6 * P, q=2 * P, ldq=128, k=3 * P, ldk=128, v=4 * P, ldv=128, g=P, s_in=40 * P, ds_out=41 * P, dq=7 * P, dk=8 * P, dv=9 * P, lddv=128, ds_in=50 * P, ws=P,
             ws_bytes=1 << 40)
    a.update(kw)
    return L.rom_linattn_backward(ctypes.byref(cfg or lin_cfg()), ctypes.byref(r or ragged()), *a.values(), None)


def qk_cfg(**kw):
    base = dict(n_q_heads=4, n_k_heads=2, d_head=64, rot_dim=32, interleaved=0, dtype=rb.ROM_BF16, eps=1e-6)
    base.update(kw)
    return rb.RomQkConfig(*base.values())


def norm(L, cfg=None, r=None, **kw):
    a = dict(rows=5, q=2 * P, ldq=256, k=3 * P, ldk=128, w_q=P, w_k=P, pos=P, freq=P, q_out=4 * P, ldq_out=256, k_out=5 * P, ldk_out=128)
    a.update(kw)
    return L.rom_qk_norm_rope(ctypes.byref(cfg or qk_cfg()), *a.values(), None)


def norm_backward(L, cfg=None, r=None, **kw):
    a = dict(rows=5, gq=6 * P, gk=7 * P, q=2 * P, ldq=256, k=3 * P, ldk=128, w_q=P, w_k=P, pos=P, freq=P, dq=4 * P, lddq=256, dk=5 * P, lddk=128, dw_q=P, dw_k=P, ws=P, ws_bytes=1 << 40)
    a.update(kw)
    return L.rom_qk_norm_rope_backward(ctypes.byref(cfg or qk_cfg()), *a.values(), None)


CALLS = {"ragged": lin_ragged, "step": lin_step, "backward": lin_backward, "norm": norm, "norm_backward": norm_backward}


@pytest.mark.skipif(torch.cuda.is_available(), reason="made-up addresses must not get past the checks on a machine with a device")
@pytest.mark.parametrize("name", CALLS)
def test_without_a_device_a_good_call_fails_for_the_device_alone(L, name):
    assert CALLS[name](L) in (-4, -5)
    optional = {"ragged": [dict(s_in=None), dict(s_out=None), dict(s_in=None, s_out=None)], "step": [dict(slot=None)],
                "backward": [dict(s_in=None), dict(ds_out=None), dict(ds_in=None)], "norm": [dict(w_q=None), dict(w_k=None), dict(q_out=2 * P), dict(q_out=2 * P, k_out=3 * P)],
                "norm_backward": [dict(w_q=None, dw_q=None), dict(w_k=None, dw_k=None)]}
    for kw in optional[name]:
        assert CALLS[name](L, **kw) in (-4, -5), kw
    if "norm" in name:
        assert CALLS[name](L, qk_cfg(rot_dim=0), pos=None, freq=None) in (-4, -5)


@pytest.mark.parametrize("name,required,by16,by4", [
    ("ragged", ["q", "k", "v", "g", "o", "ws"], ["q", "k", "v", "s_in", "s_out", "o", "ws"], ["g"]),
    ("step", ["q", "k", "v", "g", "s_in", "s_out", "o"], ["q", "k", "v", "s_in", "s_out", "o"], ["g", "slot"]),
    ("backward", ["do", "q", "k", "v", "g", "dq", "dk", "dv", "ws"], ["do", "q", "k", "v", "s_in", "ds_out", "dq", "dk", "dv", "ds_in", "ws"], ["g"]),
    ("norm", ["q", "k", "pos", "freq", "q_out", "k_out"], ["q", "k", "q_out", "k_out"], ["w_q", "w_k", "pos", "freq"]),
    ("norm_backward", ["gq", "gk", "q", "k", "pos", "freq", "dq", "dk", "ws"], ["gq", "gk", "q", "k", "dq", "dk", "ws"], ["w_q", "w_k", "pos", "freq", "dw_q", "dw_k"])])
def test_pointers_that_are_refused(L, name, required, by16, by4):
    for a in required:
        assert CALLS[name](L, **{a: None}) == INVALID, a
    for a in by16:
        assert CALLS[name](L, **{a: 60 * P + 8}) == INVALID, a
    for a in by4:
        assert CALLS[name](L, **{a: 60 * P + 2}) == INVALID, a


@pytest.mark.parametrize("name", ["ragged", "step", "backward"])
def test_linear_attention_configs_that_are_refused(L, name):
    call = CALLS[name]
    for kw, code in [(dict(n_heads=0), INVALID), (dict(n_qk_heads=0), INVALID), (dict(n_qk_heads=3), INVALID), (dict(n_qk_heads=8), INVALID), (dict(d_k=0), INVALID),
                     (dict(d_v=-8), INVALID), (dict(d_k=20), UNSUPPORTED), (dict(d_v=4), UNSUPPORTED), (dict(d_k=136), UNSUPPORTED), (dict(d_v=256), UNSUPPORTED),
                     (dict(n_heads=1026), UNSUPPORTED), (dict(dtype=2), INVALID), (dict(flags=2), INVALID), (dict(flags=16), INVALID), (dict(scale=float("nan")), INVALID),
                     (dict(scale=float("inf")), INVALID)]:
        assert call(L, lin_cfg(**kw)) == code, kw
    for ld in ("ldq", "ldk", "ldv") + (("lddv",) if name == "backward" else ()):
        for bad in (120, 132, -128):
            assert call(L, **{ld: bad}) == INVALID, ld
    if name == "step":
        assert call(L, B=-1) == INVALID and call(L, n_slots=-1) == INVALID and call(L, B=0) == OK and call(L, lin_cfg(flags=4)) == INVALID
        assert call(L, lin_cfg(n_heads=1024), B=1 << 22, ldv=1024 * 32) == UNSUPPORTED
        return
    for kw, code in [(dict(n_seq=-1), INVALID), (dict(rows=-1), INVALID), (dict(n_slots=-1), INVALID), (dict(seq_start=None), INVALID), (dict(seq_start=P + 2), INVALID),
                     (dict(slot=P + 1), INVALID), (dict(resume=P + 1), INVALID), (dict(n_seq=(1 << 20) + 1), UNSUPPORTED), (dict(rows=1 << 30), UNSUPPORTED)]:
        assert call(L, None, ragged(**kw)) == code, kw
    assert call(L, None, ragged(n_seq=0, seq_start=None)) == OK


def test_buffers_that_must_not_meet(L):
    for name in ("ragged", "step"):
        for a in ("q", "k", "v"):
            assert CALLS[name](L, **{a: 5 * P}) == INVALID      # o is none of the inputs
        assert CALLS[name](L, s_in=P, s_out=P + POOL - 16) == INVALID and CALLS[name](L, s_in=P + 16, s_out=P) == INVALID
    for a in ("do", "q", "k", "v"):
        for b in ("dq", "dk", "dv"):
            assert lin_backward(L, **{a: 60 * P, b: 60 * P}) == INVALID
    for a, b in (("dq", "dk"), ("dq", "dv"), ("dk", "dv")):
        assert lin_backward(L, **{a: 60 * P, b: 60 * P}) == INVALID
    assert lin_backward(L, ds_in=41 * P) == INVALID and lin_backward(L, ds_in=40 * P) == INVALID and lin_backward(L, ds_in=41 * P + POOL - 16) == INVALID
    assert norm(L, q_out=2 * P, ldq_out=264) == INVALID      # in place means the same pitch
    assert norm(L, q_out=3 * P) == INVALID and norm(L, k_out=2 * P) == INVALID and norm(L, q_out=5 * P) == INVALID
    for a in ("gq", "gk", "q", "k"):
        for b in ("dq", "dk"):
            assert norm_backward(L, **{a: 60 * P, b: 60 * P}) == INVALID
    assert norm_backward(L, dq=5 * P) == INVALID


@pytest.mark.parametrize("name", ["norm", "norm_backward"])
def test_norm_configs_that_are_refused(L, name):
    call = CALLS[name]
    for kw, code in [(dict(n_q_heads=0), INVALID), (dict(n_k_heads=0), INVALID), (dict(n_q_heads=1025), UNSUPPORTED), (dict(d_head=0), INVALID), (dict(d_head=60), UNSUPPORTED),
                     (dict(d_head=264), UNSUPPORTED), (dict(rot_dim=24), UNSUPPORTED), (dict(rot_dim=80), INVALID), (dict(rot_dim=-16), INVALID), (dict(interleaved=2), INVALID),
                     (dict(dtype=-1), INVALID), (dict(eps=0.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID)]:
        assert call(L, qk_cfg(**kw)) == code, kw
    assert call(L, rows=-1) == INVALID and call(L, rows=1 << 30) == UNSUPPORTED
    for ld in ("ldq", "ldk") + (("ldq_out", "ldk_out") if name == "norm" else ("lddq", "lddk")):
        for bad in (120, 260, -256):
            assert call(L, **{ld: bad}) == INVALID, ld
    if name == "norm":
        assert call(L, rows=0) == OK
    else:
        assert call(L, dw_q=None) == INVALID and call(L, w_k=None) == INVALID


def test_workspaces(L):
    cfg, n = lin_cfg(), ctypes.c_size_t(0)
    for f, call in ((L.rom_linattn_ragged_workspace_size, lin_ragged), (L.rom_linattn_backward_workspace_size, lin_backward)):
        assert f(ctypes.byref(cfg), 3, 100, ctypes.byref(n)) == OK
        assert call(L, ws_bytes=n.value - 1) == WORKSPACE
        assert f(ctypes.byref(cfg), 3, 100, None) == INVALID and f(None, 3, 100, ctypes.byref(n)) == INVALID
        for args, code in [((-1, 100), INVALID), ((3, -1), INVALID), ((3, 1 << 30), UNSUPPORTED), (((1 << 20) + 1, 100), UNSUPPORTED), ((0, 0), OK)]:
            assert f(ctypes.byref(cfg), *args, ctypes.byref(n)) == code
    q = qk_cfg()
    assert L.rom_qk_norm_rope_backward_workspace_size(ctypes.byref(q), 5, ctypes.byref(n)) == OK
    assert norm_backward(L, ws_bytes=n.value - 1) == WORKSPACE
    assert L.rom_qk_norm_rope_backward_workspace_size(ctypes.byref(q), 5, None) == INVALID


@pytest.mark.parametrize("H,G,dk,dv", [(1, 1, 128, 128), (4, 2, 64, 64), (32, 32, 128, 128), (1024, 1, 8, 8)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_workspace_for_more_does_for_less(H, G, dk, dv, dtype):
    cfg = rb.make_linattn_config(H, G, dk, dv, dtype)
    for ask in (rb.linattn_ragged_workspace_size, rb.linattn_backward_workspace_size):
        last = 0
        for rows in list(range(0, 1200, 37)) + [4096, 5000, 16384, 100000, 1 << 20]:
            size = ask(cfg, 7, rows)
            assert size >= last and size >= ask(cfg, 1, rows)
            last = size


def test_binding_refuses_what_it_cannot_describe():
    with pytest.raises(ValueError):
        rb.rom_linattn_step(rb.make_linattn_config(1, 1, 8, 8, "f32"), None, None, None, None, None, None, None, None)
    with pytest.raises(KeyError):
        rb.make_linattn_config(1, 1, 8, 8, "f16")
    with pytest.raises(KeyError):
        rb.make_qk_config(1, 1, 8, 0, torch.float16)
    assert rb.make_linattn_config(1, 1, 64, 8, "f32").scale == 0.125

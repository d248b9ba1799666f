"""Linear attention with a decay per head, and the rotation of its queries and keys: what their documentation says of starts from zeros, of values that are not finite, of far
positions."""
import math
from fractions import Fraction

import pytest
import torch

from paper_2506_18145_b200 import binding as rb

import linattn_testlib as T
from linattn_testlib import Problem
from serving_testlib import same_bits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,lens", [(2, [130, 0, 64, 1]), (1, [2300, 0, 700])])
def test_without_initial_states_every_sequence_started_from_zeros(H, lens, dtype):
    """No pool to resume from: the flags that say `resume` have nothing to resume, and the gradient of a start from zeros is zeros."""
    slots = list(range(len(lens)))[::-1]
    asks = Problem(lens, H, 1, 64, 64, dtype, seed=2, tail=3, resume=[1] * len(lens), slots=slots, backward=True)
    fresh = Problem(lens, H, 1, 64, 64, dtype, seed=2, tail=3, resume=[0] * len(lens), slots=slots, backward=True)
    for a, b in zip(asks.run(s_in=None), fresh.run()):
        assert same_bits(a, b)
    *grads, ds = asks.run_backward(s_in=None)
    *want, ds_want = fresh.run_backward()
    for a, b in zip(grads, want):
        assert same_bits(a, b)
    for s in slots:
        assert (ds[s] == 0).all() and (ds_want[s] == 0).all()


def turns(pos, freq):
    """pos * freq in turns of a circle, less the whole ones, in rational arithmetic (pi to 60 places)."""
    two_pi = 2 * Fraction(3141592653589793238462643383279502884197169399375105820974944, 10 ** 60)
    t = Fraction(pos) * Fraction(freq) / two_pi
    return float(t - round(t))


@pytest.mark.parametrize("far", [5000, 2 ** 24, 2 ** 31 - 300])
def test_angles_of_far_positions_are_those_of_the_exact_product(far):
    """One in the first place of every pair, zero in the second: the pair's angle after the rotation is the position's.

    In units of 2^-24: the turn as a float, half a step in [1/4, 1/2] 2^-26 times 2 pi: 1.6; sine and cosine, an ulp each, 1.5 together; product, sum and root of each, 2: 5.1."""
    rows, d = 200, 128
    cfg = rb.make_qk_config(1, 1, d, d, "f32")
    x = torch.zeros((rows, d), device="cuda")
    x[:, :d // 2] = 1.0
    pos = torch.arange(far, far + rows, dtype=torch.int64).to(torch.int32)
    freq = (10000.0 ** (-torch.arange(d // 2, dtype=torch.float64) / 640)).float()      # (slowly falling: most of the angles are large)
    q, k = torch.empty_like(x), torch.empty_like(x)
    rb.rom_qk_norm_rope(cfg, x, x.clone(), None, None, pos.cuda(), freq.cuda(), q, k)
    y = q.double().cpu()
    got = torch.atan2(y[:, d // 2:], y[:, :d // 2]) / (2 * math.pi)
    want = torch.tensor([[turns(p, f) for f in freq.tolist()] for p in pos.tolist()], dtype=torch.float64)
    off = got - want
    off = (off - torch.round(off)).abs() * 2 * math.pi
    assert float(off.max()) <= 5.1 * 2.0 ** -24, f"{float(off.max()) * 2 ** 24:.2f} units"


def test_rows_beyond_32_bits_of_elements():
    """One sequence behind 2^31 elements of v and of the results; what lies ahead of it belongs to nobody, and is neither read nor written."""
    H, G, d, n, lead = 32, 16, 128, 200, 1 << 19
    rows = lead + n
    cfg = rb.make_linattn_config(H, G, d, d, "bf16")
    gen = torch.Generator().manual_seed(2)

    def tall(width):
        x = torch.empty((rows, width), dtype=torch.bfloat16, device="cuda")
        x[lead:] = torch.randn((n, width), generator=gen).bfloat16().cuda()
        return x

    q, k, v, do = tall(G * d), tall(G * d), tall(H * d), tall(H * d)
    g = (-torch.logspace(-0.5, -3, H)).cuda()
    start = torch.tensor([lead, rows], dtype=torch.int32, device="cuda")
    seqs = rb.make_ragged(rows, 1, start)
    ws = torch.empty(rb.linattn_backward_workspace_size(cfg, 1, rows), dtype=torch.uint8, device="cuda")
    o, dq, dk, dv = tall(H * d), tall(G * d), tall(G * d), tall(H * d)
    for x in (o, dq, dk, dv):
        x[:300], x[lead - 300:lead] = -7.0, -7.0
    s_out, ds_in = torch.empty((1, H, d, d), device="cuda"), torch.empty((1, H, d, d), device="cuda")
    rb.rom_linattn_ragged(cfg, seqs, q, k, v, g, None, s_out, o, ws)
    rb.rom_linattn_backward(cfg, seqs, do, q, k, v, g, None, None, dq, dk, dv, ds_in, ws)
    assert rb.rom_get_status(ws) == 0
    x = lambda t, m: t[lead:].double().view(n, m, d)  # noqa: E731
    zero = torch.zeros((H, d, d), dtype=torch.float64, device="cuda")
    scale = float(torch.tensor(cfg.scale, dtype=torch.float32))
    ref, S = T.forward(x(q, G), x(k, G), x(v, H), g.double(), zero, scale)
    size, Ssize = T.forward(x(q, G).abs(), x(k, G).abs(), x(v, H).abs(), g.double(), zero, scale)
    eo, es = T.units(n, d + 2, True)
    T.near(x(o, H), ref, size, eo, "bf16", "o")
    T.near(s_out[0], S, Ssize, es, "f32", "state")
    gref = T.backward(x(do, H), x(q, G), x(k, G), x(v, H), g.double(), zero, zero, scale)
    gsize = T.backward(x(do, H).abs(), x(q, G).abs(), x(k, G).abs(), x(v, H).abs(), g.double(), zero, zero, scale)
    for name, got, m, i in (("dq", dq, G, 0), ("dk", dk, G, 1), ("dv", dv, H, 2)):
        T.near(x(got, m), gref[i], gsize[i], eo, "bf16", name)
    assert (ds_in == 0).all()
    for y in (o, dq, dk, dv):
        assert (y[:300] == -7).all() and (y[lead - 300:lead] == -7).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_two_calls_at_once(dtype):
    """Two streams, a workspace each: what each call gives is what it gives alone."""
    problems = [Problem([900, 333, 1, 64], 4, 2, 128, 64, dtype, seed=8, backward=True), Problem([2500], 2, 2, 128, 128, dtype, seed=9, backward=True)]
    alone = [[*p.run(), *p.run_backward()] for p in problems]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in problems]
    for _ in range(3):
        got = []
        for p, st in zip(problems, streams):
            st.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(st):
                got.append([*p.run(), *p.run_backward()])
        torch.cuda.synchronize()
        for a, b in zip(alone, got):
            for x, y in zip(a, b):
                assert same_bits(x, y)
    for p in problems:
        assert rb.rom_get_status(p.ws) == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,rot,interleaved", [(128, 128, False), (96, 48, True), (40, 16, False)])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_norm_of_a_value_that_is_not_finite_stays_in_its_head_and_row(bad, d, rot, interleaved, dtype):
    rows, nq, nk = 37, 5, 2
    gen = torch.Generator().manual_seed(d)
    cfg = rb.make_qk_config(nq, nk, d, rot, dtype, interleaved=interleaved)
    new = lambda n: torch.randn((rows, n * d), generator=gen).to(T.TORCH[dtype]).cuda()  # noqa: E731
    q, k, gq, gk, w = new(nq), new(nk), new(nq), new(nk), torch.rand(d, generator=gen).cuda()
    pos, freq = torch.arange(rows, dtype=torch.int32, device="cuda"), torch.rand(rot // 2, generator=gen).cuda()
    ws = torch.empty(rb.qk_norm_rope_backward_workspace_size(cfg, rows), dtype=torch.uint8, device="cuda")

    def both():
        y = [torch.empty_like(q), torch.empty_like(k)]
        rb.rom_qk_norm_rope(cfg, q, k, w, w, pos, freq, *y)
        dx, dw = [torch.empty_like(q), torch.empty_like(k)], [torch.empty(d, device="cuda"), torch.empty(d, device="cuda")]
        rb.rom_qk_norm_rope_backward(cfg, gq, gk, q, k, w, w, pos, freq, *dx, *dw, ws)
        return y, dx, dw

    (y, dx, dw) = both()
    q[20, 3 * d + d - 1] = bad
    (y2, dx2, dw2) = both()
    assert same_bits(y[1], y2[1]) and same_bits(dx[1], dx2[1]) and same_bits(dw[1], dw2[1])
    for a, b in ((y[0], y2[0]), (dx[0], dx2[0])):
        other = torch.ones((rows, nq), dtype=torch.bool, device="cuda")
        other[20, 3] = False
        assert same_bits(a.view(rows, nq, d)[other], b.view(rows, nq, d)[other]) and not torch.isfinite(b.view(rows, nq, d)[20, 3, d - 1].float())

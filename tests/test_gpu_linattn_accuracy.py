"""Linear attention in bf16 against closed forms in 64 bits, to what its arithmetic leaves beside the rounding of the results themselves.

A result is one rounding of a number x that lies within `slack` of the exact one: rounding is monotone, so it lies between the rounded ends of [exact - slack, exact + slack]."""
import pytest
import torch

from paper_2506_18145_b200 import binding as rb

import linattn_testlib as T
from linattn_testlib import Problem

pytestmark = pytest.mark.gpu

SHAPES = [(2, 2, 16, 64), (4, 2, 64, 64), (2, 1, 128, 128), (2, 2, 128, 40), (3, 3, 24, 128)]
# Operands are sums of two bf16 numbers: the first, cut off, leaves less than 2^-7 of a number, of which the second loses half a step, 2^-8.
PARTS = 2.0 ** -15
STEP = 2.0 ** -23      # what a sum in the matrix instructions may lose a term, of the sum of its terms' sizes


def one_rounding(got, ref, slack, what):
    got, ref = got.double().reshape(ref.shape), ref.double()
    low, high = (ref - slack).to(torch.bfloat16).double(), (ref + slack).to(torch.bfloat16).double()
    wrong = ~((got >= low) & (got <= high))
    assert not wrong.any(), f"{what}: {int(wrong.sum())} of {wrong.numel()} are no rounding of the result, the first off by {float((got - ref)[wrong][0]):.3g} where {float(slack[wrong][0]):.3g} is left"


def by_heads(x, rows, n):
    return x[rows].reshape(x[rows].shape[0], n, -1)


@pytest.mark.parametrize("H,G,dk,dv", SHAPES)
@pytest.mark.parametrize("n", [1, 16, 37, 128])
def test_scores_keep_their_bits(n, H, G, dk, dv):
    """One chunk from a state of zeros: only scores, decayed, times values."""
    pr = Problem([n], H, G, dk, dv, "bf16", seed=n, lead=1, tail=2, resume=[0], backward=True)
    rows, q, k, v, do, S0, _ = pr.sequence(0)
    o, _ = pr.run(s_out=None)
    q_, k_, v_ = T._share(q, H), T._share(k, H), v.transpose(0, 1)
    D = T._decays(pr.g.double(), n)[0]
    P, Psize = abs(pr.scale) * (q_ @ k_.transpose(1, 2)).abs() * D, abs(pr.scale) * (q_.abs() @ k_.abs().transpose(1, 2)) * D
    ref, _ = T.forward(q, k, v, pr.g.double(), S0, pr.scale)
    slack = (PARTS * P + (dk + n + 8) * STEP * Psize) @ v_.abs()
    one_rounding(by_heads(o, rows, H), ref, slack.transpose(0, 1), "o")
    dq, dk_, dv_, _ = pr.run_backward(ds_out=None, ds_in=None, s_in=None)
    do_ = do.transpose(0, 1)
    A, Asize = abs(pr.scale) * (do_ @ v_.transpose(1, 2)).abs() * D, abs(pr.scale) * (do_.abs() @ v_.abs().transpose(1, 2)) * D
    left, right = PARTS * A + (dv + n + 8 + H // G) * STEP * Asize, PARTS * P + (dk + n + 8) * STEP * Psize
    ref = T.backward(do, q, k, v, pr.g.double(), S0, torch.zeros_like(S0), pr.scale)
    back = lambda x: x.transpose(0, 1).reshape(n, G, H // G, x.shape[2]).sum(2)  # noqa: E731
    one_rounding(by_heads(dq, rows, G), ref[0], back(left @ k_.abs()), "dq")
    one_rounding(by_heads(dk_, rows, G), ref[1], back(left.transpose(1, 2) @ q_.abs()), "dk")
    one_rounding(by_heads(dv_, rows, H), ref[2], (right.transpose(1, 2) @ do_.abs()).transpose(0, 1), "dv")


@pytest.mark.parametrize("H,G,dk,dv", SHAPES)
@pytest.mark.parametrize("n", [1, 33, 128, 300])
def test_the_state_keeps_its_bits(n, H, G, dk, dv):
    """Keys (or queries, or values) of zeros: the scores are zero, and every result is a product with the state that came in, decayed."""
    chunks = n / 128 + 1
    pr = Problem([n], H, G, dk, dv, "bf16", seed=n, tail=3, resume=[1], rates=[0.02 * 0.5 ** h for h in range(H)], backward=True)
    pr.k.zero_()
    rows, q, k, v, do, S0, dS = pr.sequence(0)
    ref, _ = T.forward(q, k, v, pr.g.double(), S0, pr.scale)
    size, _ = T.forward(q.abs(), k, v, pr.g.double(), S0.abs(), abs(pr.scale))
    unit = PARTS + (dk + 8 + 3 * chunks) * STEP
    one_rounding(by_heads(pr.run(s_out=None)[0], rows, H), ref, unit * size, "o")

    gen = torch.Generator().manual_seed(n)
    pr.k.copy_(torch.randn(pr.k.shape, generator=gen))
    pr.q.zero_()      # dk = v R^T, dv = k R: of ds_out alone
    rows, q, k, v, do, S0, dS = pr.sequence(0)
    got = pr.run_backward()
    ref = T.backward(do, q, k, v, pr.g.double(), S0, dS, pr.scale)
    size = T.backward(do.abs(), q, k.abs(), v.abs(), pr.g.double(), S0.abs(), dS.abs(), abs(pr.scale))
    unit = PARTS + (max(dk, dv) + H // G + 8 + 3 * chunks) * STEP
    one_rounding(by_heads(got[1], rows, G), ref[1], unit * size[1], "dk")
    one_rounding(by_heads(got[2], rows, H), ref[2], unit * size[2], "dv")

    pr.q.copy_(torch.randn(pr.q.shape, generator=gen))
    pr.v.zero_()      # dq = dout S^T: of s_in alone
    rows, q, k, v, do, S0, dS = pr.sequence(0)
    got = pr.run_backward()
    ref = T.backward(do, q, k, v, pr.g.double(), S0, dS, pr.scale)
    size = T.backward(do.abs(), q.abs(), k.abs(), v, pr.g.double(), S0.abs(), dS.abs(), abs(pr.scale))
    one_rounding(by_heads(got[0], rows, G), ref[0], unit * size[0], "dq")


def weighted(x, y, g, exponent):
    """sum_t lambda^exponent_t x_t y_t^T for every head, [H, dx, dy]; x, y [n, H, d]."""
    w = torch.exp(g[:, None] * exponent)      # [H, n]
    return torch.stack([(x[:, h] * w[h][:, None]).T @ y[:, h] for h in range(x.shape[1])])


@pytest.mark.parametrize("n,d", [(16384, 16), (131072, 16), (16384, 128)])
def test_long_sums_lose_no_more_than_short_ones(n, d):
    """One sequence of many heads, thousands of rows from cut to cut, hardly any decay: the last state and the gradient of the first one, which are sums over all rows.

    `near` allows 2^-19 of the norm, what 32 sums in the matrix instructions lose at most before they move to registers; how many rows there are does not matter."""
    H = 32
    pr = Problem([n], H, H, d, d, "bf16", seed=3, resume=[1], rates=[[0.0, 2.0 ** -11, 1e-5, 2.0 ** -7][h % 4] for h in range(H)], backward=True)
    g, slot = pr.g.double(), int(pr.p.slots[0])
    at = torch.arange(n, dtype=torch.float64, device="cuda")
    full = torch.exp(g * n)[:, None, None]
    _, s = pr.run()
    cut = lambda x: x.double().view(n, H, d)  # noqa: E731
    es = T.units(n, d, True)[1]
    S = weighted(cut(pr.k), cut(pr.v), g, n - 1 - at) + full * pr.s_in[slot].double()
    size = weighted(cut(pr.k).abs(), cut(pr.v).abs(), g, n - 1 - at) + full * pr.s_in[slot].double().abs()
    for h in range(4):      # (each rate of its own: the sums without decay are the largest)
        T.near(s[slot][h::4], S[h::4], size[h::4], es, "f32", f"state, rate {float(-pr.g[h]):.2g}")
    *_, ds = pr.run_backward()
    R = pr.scale * weighted(cut(pr.q), cut(pr.do), g, at + 1) + full * pr.ds_out[slot].double()
    size = pr.scale * weighted(cut(pr.q).abs(), cut(pr.do).abs(), g, at + 1) + full * pr.ds_out[slot].double().abs()
    for h in range(4):
        T.near(ds[slot][h::4], R[h::4], size[h::4], es, "f32", f"gradient of the state, rate {float(-pr.g[h]):.2g}")
    assert rb.rom_get_status(pr.ws) == 0


@pytest.mark.parametrize("dtype,n", [("bf16", 148 * 256 - 128), ("f32", 296 * 256 - 32)])
def test_a_slow_decay_over_every_cut(dtype, n):
    """One head, cut as often as it can be, 256 rows from cut to cut, and a decay whose power of 256 lies half way between two floats: nothing but the first state, decayed.

    A cut rounds each number once, 2^-24 of it at most and independent: at 296 cuts sqrt(296 / 3) 2^-24 = 2^-20.7 of the norm.  (One float for the power would be 2^-25 off at each cut,
    the same way: 296 2^-25 = 2^-16.8.)"""
    pr = Problem([n], 1, 1, 16, 16, dtype, seed=5, resume=[1], rates=[1.1230999916733708e-05], backward=True)
    slot, full = int(pr.p.slots[0]), torch.exp(pr.g.double()[0] * n)
    pr.k.zero_()
    s = pr.run()[1][slot].double()
    ref = full * pr.s_in[slot].double()
    assert (s - ref).norm() <= 2.0 ** -20 * ref.norm()
    pr.k.fill_(1.0)
    pr.q.zero_()
    ds = pr.run_backward()[3][slot].double()
    ref = full * pr.ds_out[slot].double()
    assert (ds - ref).norm() <= 2.0 ** -20 * ref.norm()


def on_places(got, ref, size, unit, store, places, what):
    """`near`, elementwise, at the places that a value which is not finite does not reach."""
    got, ref, tol = got.double()[places], ref[places], (unit * size * (1 + T.HALF_STEP[store]) + T.HALF_STEP[store] * ref.abs())[places] + 1e-37
    assert torch.isfinite(got).all(), f"{what}: not finite at {int((~torch.isfinite(got)).sum())} places"
    assert float(((got - ref).abs() / tol).max()) <= 1.0, f"{what}: {float(((got - ref).abs() / tol).max()):.2f} times the bound"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,G,dk,dv", [(4, 4, 64, 64), (4, 2, 128, 72), (6, 1, 40, 128)])
@pytest.mark.parametrize("which,bad", [("v", float("nan")), ("v", float("inf")), ("k", float("-inf")), ("q", float("nan")), ("do", float("inf")), ("do", float("nan"))])
@pytest.mark.parametrize("at", [173, 255])
def test_rows_beside_one_that_is_not_finite_keep_their_bits(at, which, bad, H, G, dk, dv, dtype):
    """One value of one row, in the middle or at the end of a chunk: what it does not reach is as exact as without it."""
    n, head = 400, 1
    pr = Problem([n, 150], H, G, dk, dv, dtype, seed=7, resume=[1, 0], backward=True)
    group = head * G // H
    place = 5
    x = getattr(pr, which)
    x[at, (head * dv if which in ("v", "do") else group * dk) + place] = 0.0
    rows, q, k, v, do, S0, dS = pr.sequence(0)
    ref, _ = T.forward(q, k, v, pr.g.double(), S0, pr.scale)
    size, _ = T.forward(q.abs(), k.abs(), v.abs(), pr.g.double(), S0.abs(), abs(pr.scale))
    gref = T.backward(do, q, k, v, pr.g.double(), S0, dS, pr.scale)
    gsize = T.backward(do.abs(), q.abs(), k.abs(), v.abs(), pr.g.double(), S0.abs(), dS.abs(), abs(pr.scale))
    x[at, (head * dv if which in ("v", "do") else group * dk) + place] = bad

    row = torch.arange(n, device="cuda")[:, None, None]
    heads = torch.arange(H, device="cuda")[None, :, None]
    shared = heads * G // H == group              # value heads that read the group's q and k
    groups = torch.arange(G, device="cuda")[None, :, None] == group
    cv, ck = torch.arange(dv, device="cuda")[None, None, :] == place, torch.arange(dk, device="cuda")[None, None, :] == place
    every_v, every_k = torch.ones_like(cv), torch.ones_like(ck)
    none = torch.zeros((1, 1, 1), dtype=torch.bool, device="cuda")
    mine = heads == head
    reached = {      # o, dq, dk, dv: rows from or up to it, one column or all
        "q": ((row == at) & shared & every_v, none, (row <= at) & groups & ck, (row <= at) & shared & every_v),
        "k": ((row >= at) & shared & every_v, (row >= at) & groups & ck, none, (row == at) & shared & every_v),
        "v": ((row >= at) & mine & cv, (row >= at) & groups & every_k, (row == at) & groups & every_k, none),
        "do": (none, (row == at) & groups & every_k, (row <= at) & groups & every_k, (row <= at) & mine & cv)}[which]
    parts = 2 * PARTS if dtype == "bf16" else 0.0
    unit = T.units(n, max(dk, dv) + H // G, False)[0] + parts
    o, _ = pr.run()
    dq, dk_, dv_, _ = pr.run_backward()
    for name, got, r, s, where in (("o", by_heads(o, rows, H), ref, size, reached[0]), ("dq", by_heads(dq, rows, G), gref[0], gsize[0], reached[1]),
                                   ("dk", by_heads(dk_, rows, G), gref[1], gsize[1], reached[2]), ("dv", by_heads(dv_, rows, H), gref[2], gsize[2], reached[3])):
        where = where.expand(r.shape)
        on_places(got, r, s, unit, dtype, ~where, name)
        assert not torch.isfinite(got.float()[where]).any(), f"{name}: finite where it cannot be"
    assert rb.rom_get_status(pr.ws) == 0

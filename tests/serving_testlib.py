"""Helpers of the serving tests: packed sequences and pools on the GPU, the oracle run sequence by sequence, and error bounds that follow the
arithmetic.  (Test infrastructure; not part of the product.)"""
from __future__ import annotations

import numpy as np
import torch

from oracle import rom_oracle as O
from paper_2506_18145_b200 import binding as rb

from rom_testlib import np64

TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
U32 = 2.0 ** -24                                   # half a step of fp32, relative
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


class Packed:
    """Sequences of the given lengths behind `lead` rows that belong to nobody and before `tail` more."""

    def __init__(self, lens, lead=0, tail=0, seed=0, n_slots=None, slots=None, resume=None):
        g = np.random.default_rng(seed)
        self.lens, self.n = list(lens), len(lens)
        self.start = lead + np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        self.rows = int(self.start[-1]) + tail
        self.n_slots = n_slots or self.n + 3
        self.slots = np.asarray(slots if slots is not None else g.permutation(self.n_slots)[:self.n], dtype=np.int32)
        self.resume = np.asarray(resume if resume is not None else g.integers(0, 2, self.n), dtype=np.int32)
        self.dev = [torch.from_numpy(v).cuda() for v in (self.start, self.slots, self.resume)]
        self.ragged = rb.make_ragged(self.rows, self.n_slots, *self.dev)

    def kept(self, i):
        return 0 <= self.slots[i] < self.n_slots

    def resumes(self, i):
        return bool(self.resume[i]) and self.kept(i)

    def mine(self):
        """Rows that belong to a sequence."""
        m = np.zeros(self.rows, dtype=bool)
        m[self.start[0]:self.start[-1]] = True
        return m


def randn(seed, shape, std=1.0, dtype=torch.float32):
    g = torch.Generator()
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(dtype)


def wide(t, left, right, fill=float("nan")):
    """t as a column slice of wider rows, the columns beside it filled."""
    rows, w = t.shape
    full = torch.full((rows, left + w + right), fill, dtype=t.dtype, device="cuda")
    full[:, left:left + w] = t.cuda()
    return full[:, left:left + w]


def pool_with_junk(seed, p, shape, std):
    """A pool whose slots that no sequence resumes from hold NaN."""
    pool = randn(seed, (p.n_slots,) + shape, std)
    used = {int(p.slots[i]) for i in range(p.n) if p.resumes(i)}
    for s in range(p.n_slots):
        if s not in used:
            pool[s] = float("nan")
    return pool


def conv_reference(x, w, b, past):
    """(y, |terms| summed, window) of one sequence, [n, De] and its window [k-1, De] before it."""
    k, n = w.shape[0], x.shape[0]
    line = np.concatenate([past, x])
    pre = np.tile(b if b is not None else np.zeros(w.shape[1]), (n, 1))
    size = np.abs(pre)
    for q in range(k):
        pre = pre + w[q] * line[q:q + n]
        size = size + np.abs(w[q] * line[q:q + n])
    return pre, size, line[n:]


def silu_bound(pre, err):
    """Error of SiLU(pre) computed in fp32 from a value `err` off: its slope is at most 1.1, exp and the quotient are a few units off,
    the exponent of exp by |pre| of them."""
    return 1.1 * err + (8.0 + 2.0 * np.abs(pre)) * U32 * np.abs(O.silu(pre))


def scan_reference(u, delta, A, Bm, Cm, D, z, h0, disc_mode):
    """(y, bound of its fp32 error, h_last, bound of its error) of one sequence.

    Every step of the recurrence rounds a few times and takes the decay a few units off (its exponent Delta A too, by |Delta A| units: less than
    half a unit of a each); what goes wrong by that in one step is at most 16 units of |h_{t-1}| + |B u / A| (zero-order hold: the input enters as
    w = -B u / A, of which 1 - a is taken) or + |Delta B u|, and decays with the state afterwards: G_t = a G_{t-1} + 16 U (|h_{t-1}| + |w|)."""
    n, De = u.shape
    h, G = np.array(h0), np.zeros_like(h0)
    y, bound = np.zeros((n, De)), np.zeros((n, De))
    gate = O.silu(z) if z is not None else np.ones((n, De))
    for t in range(n):
        x = delta[t][:, None] * A
        a = np.exp(x)
        bu = Bm[t][None, :] * u[t][:, None]
        inp = np.expm1(x) / A * bu if disc_mode == 0 else delta[t][:, None] * bu
        w = np.abs(bu / A) if disc_mode == 0 else np.abs(inp)
        G = a * G + 16.0 * U32 * (np.abs(h) + w)
        h = a * h + inp
        skip = D * u[t] if D is not None else 0.0 * u[t]
        v = h @ Cm[t] + skip
        e = G @ np.abs(Cm[t]) + 20.0 * U32 * (np.abs(h) @ np.abs(Cm[t]) + np.abs(skip))
        y[t] = v * gate[t]
        bound[t] = e * np.abs(gate[t]) + np.abs(v) * (silu_bound(z[t], 0.0) if z is not None else 0.0)
    return y, bound, h, G


def check(got, ref, bound, dtype, what):
    """|got - ref| <= the fp32 error's bound + half a step of the storage type."""
    got = np64(got)
    tol = bound * (1.0 + HALF_STEP[dtype]) + HALF_STEP[dtype] * np.abs(ref) + 1e-37
    off = np.abs(got - ref)
    assert np.all(np.isfinite(got)), f"{what}: not finite"
    worst = np.max(off / tol) if off.size else 0.0
    assert worst <= 1.0, f"{what}: {worst:.2f} times the bound, at {np.unravel_index(np.argmax(off / tol), off.shape)}"


def same_bits(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))

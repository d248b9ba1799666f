"""RMS norm of every head of q and k and its rotation by the position, forward and backward, against the formulas in 64 bits."""
import pytest
import torch

from paper_2506_18145_b200 import binding as rb

import linattn_testlib as T
from serving_testlib import HALF_STEP, U32, same_bits

pytestmark = pytest.mark.gpu

CASES = [  # rows, heads of q, of k, d, rot, interleaved
    (1, 1, 1, 8, 0, False), (1, 32, 32, 128, 128, False), (7, 3, 1, 80, 64, False), (7, 3, 2, 96, 48, True), (33, 5, 2, 256, 256, False), (33, 5, 2, 256, 192, True),
    (130, 2, 9, 24, 16, False), (130, 2, 9, 16, 16, True), (50, 40, 40, 64, 32, False), (3000, 8, 4, 40, 32, False), (5000, 16, 8, 128, 128, False), (5000, 16, 9, 128, 64, True)]


class Problem:
    def __init__(self, rows, nq, nk, d, rot, interleaved, dtype, seed=0, far=0, wide=8, eps=1e-6, std=1.7):
        g = torch.Generator().manual_seed(seed)
        self.rows, self.nq, self.nk, self.d, self.rot, self.inter, self.dtype, self.eps = rows, nq, nk, d, rot, interleaved, dtype, eps
        t = T.TORCH[dtype]
        self.x = (torch.randn((rows, (nq + nk) * d + wide), generator=g) * std).to(t).cuda()
        self.x[:, (nq + nk) * d:] = float("nan")
        self.q, self.k = self.x[:, :nq * d], self.x[:, nq * d:(nq + nk) * d]
        self.w = [(1 + 0.3 * torch.randn(d, generator=g)).cuda() for _ in range(2)]
        self.pos = (far + torch.randperm(rows, generator=g)).to(torch.int32).cuda()
        self.freq = (10000.0 ** (-torch.arange(rot // 2) / max(1, rot // 2))).float().cuda()
        self.dy = [torch.randn((rows, n * d), generator=g).to(t).cuda() for n in (nq, nk)]
        self.cfg = rb.make_qk_config(nq, nk, d, rot, dtype, eps, interleaved)

    def heads(self, x, n):
        return x.double().reshape(self.rows, n, self.d)

    def rot_args(self):
        return (self.pos, self.freq) if self.rot else (None, None)

    def forward(self, out=None, w=True):
        out = out or [torch.full((self.rows, n * self.d), -7.0, dtype=self.x.dtype, device="cuda") for n in (self.nq, self.nk)]
        rb.rom_qk_norm_rope(self.cfg, self.q, self.k, *(self.w if w else (None, None)), *self.rot_args(), *out)
        return out

    def backward(self, w=True):
        dx = torch.full_like(self.x, -7.0)
        dw = [torch.full((self.d,), -7.0, device="cuda") for _ in range(2)] if w else [None, None]
        ws = torch.full((rb.qk_norm_rope_backward_workspace_size(self.cfg, self.rows),), 0xFF, dtype=torch.uint8, device="cuda")
        n = self.nq * self.d
        rb.rom_qk_norm_rope_backward(self.cfg, *self.dy, self.q, self.k, *(self.w if w else (None, None)), *self.rot_args(), dx[:, :n], dx[:, n:n + self.nk * self.d], *dw, ws)
        return dx, dw

    def check_forward(self, out, w=True):
        for x, n, wt, y in ((self.q, self.nq, self.w[0], out[0]), (self.k, self.nk, self.w[1], out[1])):
            wt = wt.double() if w else torch.ones_like(wt).double()
            x = self.heads(x, n)
            ref = T.norm_rope(x, wt, self.pos, self.freq, self.rot, self.inter, self.eps)
            # the sum of d squares, the root and four products: d / 2 + 10 units of the normalised values; the angle's sine and cosine 4 units, of the pair's size
            flat = T.norm_rope(x, wt, self.pos, self.freq, 0, False, self.eps).abs()
            size = T.turn(flat, torch.zeros_like(self.pos).double()[:, None] * self.freq.double(), self.rot, self.inter) if self.rot else flat
            i = torch.arange(self.rot // 2, device="cuda")
            a, b = (2 * i, 2 * i + 1) if self.inter else (i, i + self.rot // 2)
            size[..., a] = size[..., b] = flat[..., a] + flat[..., b]
            T.near(y, ref, size, (self.d / 2 + 16) * U32, self.dtype, "norm and rotation")

    def check_backward(self, dx, dw, w=True):
        n = self.nq * self.d
        for x, m, wt, dy, g, gw in ((self.q, self.nq, self.w[0], self.dy[0], dx[:, :n], dw[0]), (self.k, self.nk, self.w[1], self.dy[1], dx[:, n:n + self.nk * self.d], dw[1])):
            wt = wt.double() if w else torch.ones_like(wt).double()
            x, dy = self.heads(x, m), self.heads(dy, m)
            ref, refw, sizew = T.norm_rope_backward(dy, x, wt, self.pos, self.freq, self.rot, self.inter, self.eps)
            r = torch.rsqrt((x * x).mean(-1, keepdim=True) + self.eps)
            pair = dy.abs()
            if self.rot:
                i = torch.arange(self.rot // 2, device="cuda")
                a, b = (2 * i, 2 * i + 1) if self.inter else (i, i + self.rot // 2)
                both = pair[..., a] + pair[..., b]
                pair[..., a], pair[..., b] = both, both
            gsize = pair * wt.abs()
            size = r * (gsize + (x * r).abs() * (gsize * (x * r).abs()).mean(-1, keepdim=True))
            T.near(g, ref, size, (2 * self.d + 32) * U32, self.dtype, "dx")
            if gw is not None:
                # a lane's sum of at most rows * heads terms, in fact of a few hundred, then of the blocks' in 64 bits
                terms = min(self.rows * m, 2048) + 64
                assert ((gw.double() - refw).abs() <= (terms + self.d + 32) * U32 * ((pair * (x * r).abs()).sum((0, 1))) + 1e-30).all()
                # as random roundings add up: sqrt(2048) 2^-24 / 2 of the norm of the terms' sum of absolute values at most
                assert (gw.double() - refw).norm() <= 2.0 ** -19 * sizew.norm()
        assert (dx[:, n + self.nk * self.d:] == -7).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,nq,nk,d,rot,inter", CASES)
def test_forward(rows, nq, nk, d, rot, inter, dtype):
    p = Problem(rows, nq, nk, d, rot, inter, dtype, seed=rows + d)
    p.check_forward(p.forward())
    p.check_forward(p.forward(w=False), w=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,nq,nk,d,rot,inter", CASES)
def test_backward(rows, nq, nk, d, rot, inter, dtype):
    p = Problem(rows, nq, nk, d, rot, inter, dtype, seed=rows + d + 1)
    dx, dw = p.backward()
    p.check_backward(dx, dw)
    again, dw2 = p.backward()
    assert same_bits(dx, again) and same_bits(dw[0], dw2[0]) and same_bits(dw[1], dw2[1])
    p.check_backward(*p.backward(w=False), w=False)


@pytest.mark.parametrize("far", [1_000_000, 2_147_000_000])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_positions_keep_their_angle(far, dtype):
    p = Problem(64, 4, 2, 128, 128, False, dtype, seed=1, far=far)
    p.check_forward(p.forward())
    p.check_backward(*p.backward())
    p.pos = -p.pos      # (a position before the first is an angle like any other)
    p.check_forward(p.forward())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place_zero_rows_and_values_that_are_not_finite(dtype):
    p = Problem(200, 4, 2, 64, 32, False, dtype, seed=2)
    p.x[5, :64] = 0.0      # a head of zeros stays zeros
    p.x[9, 3] = float("nan")
    p.x[11, 64 + 5] = float("inf")
    out = p.forward()
    assert (out[0][5, :64] == 0).all()
    bad = ~torch.isfinite(out[0].view(200, 4, 64).float()).all(-1)
    assert bad.sum() == 2 and bad[9, 0] and bad[11, 1] and torch.isfinite(out[1].float()).all()
    dx, dw = p.backward()
    bad = ~torch.isfinite(dx[:, :4 * 64].reshape(200, 4, 64).float()).all(-1)
    assert bad.sum() == 2 and bad[9, 0] and bad[11, 1]
    rb.rom_qk_norm_rope(p.cfg, p.q, p.k, *p.w, p.pos, p.freq, p.q, p.k)
    assert same_bits(p.q.contiguous().view(torch.uint8), out[0].view(torch.uint8)) and same_bits(p.k.contiguous(), out[1])


def test_no_rows():
    p = Problem(1, 2, 2, 64, 32, False, "bf16")
    p.rows, p.x = 0, p.x[:0]
    p.q, p.k, p.pos, p.dy = p.q[:0], p.k[:0], p.pos[:0], [d[:0].contiguous() for d in p.dy]
    p.forward()
    dx, dw = p.backward()
    assert (dw[0] == 0).all() and (dw[1] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_captured_and_replayed(dtype):
    p = Problem(300, 4, 4, 128, 128, False, dtype, seed=3)
    ref, (dx, dw) = p.forward(), p.backward()
    ws = torch.empty(rb.qk_norm_rope_backward_workspace_size(p.cfg, 300), dtype=torch.uint8, device="cuda")
    out, dx2, dw2 = [torch.empty_like(x) for x in ref], torch.full_like(dx, -7.0), [torch.empty_like(w) for w in dw]
    n = 4 * 128
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.forward(out)
        rb.rom_qk_norm_rope_backward(p.cfg, *p.dy, p.q, p.k, *p.w, p.pos, p.freq, dx2[:, :n], dx2[:, n:2 * n], *dw2, ws)
    for x in out:
        x.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip([*ref, dx, *dw], [*out, dx2, *dw2]):
        assert same_bits(a, b)

"""Linear attention with a decay per head, and the norm and rotation of its queries and keys, in 64 bits: closed forms over one sequence, and the error bounds of the
kernels' arithmetic.  (Test infrastructure; not part of the product.)"""
from __future__ import annotations

import torch

from paper_2506_18145_b200 import binding as rb

from serving_testlib import Packed, HALF_STEP, U32

TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}


def _share(x, H):
    """[n, G, d] -> [H, n, d]: value head h uses head h / (H / G)."""
    return x.repeat_interleave(H // x.shape[1], 1).transpose(0, 1)


def _decays(g, n):
    """lambda^{i-j} below and on the diagonal [H, n, n], lambda^{i+1} [H, n, 1], lambda^{n-1-j} [H, n, 1], lambda^n [H, 1, 1]."""
    i = torch.arange(n, dtype=torch.float64, device=g.device)
    gap = i[:, None] - i[None, :]
    D = torch.where(gap >= 0, torch.exp(g[:, None, None] * gap.clamp(min=0)), 0.0)
    row = lambda e: torch.exp(g[:, None] * e)[..., None]  # noqa: E731
    return D, row(i + 1), row(n - 1 - i), row(torch.tensor([float(n)], dtype=torch.float64, device=g.device))


def forward(q, k, v, g, S0, scale):
    """q, k [n, G, dk], v [n, H, dv], g [H], S0 [H, dk, dv] -> (o [n, H, dv], S [H, dk, dv])."""
    n, H = v.shape[0], v.shape[1]
    q, k, v = _share(q, H), _share(k, H), v.transpose(0, 1)
    D, up, down, full = _decays(g, n)
    o = scale * (((q @ k.transpose(1, 2)) * D) @ v + up * (q @ S0))
    return o.transpose(0, 1), (k * down).transpose(1, 2) @ v + full * S0


def backward(do, q, k, v, g, S0, dS, scale):
    """(dq, dk [n, G, dk], dv [n, H, dv], dS0 [H, dk, dv])."""
    n, H, G = v.shape[0], v.shape[1], q.shape[1]
    q, k, v, do = _share(q, H), _share(k, H), v.transpose(0, 1), do.transpose(0, 1)
    D, up, down, full = _decays(g, n)
    A = scale * (do @ v.transpose(1, 2)) * D
    P = scale * (q @ k.transpose(1, 2)) * D
    dq = A @ k + scale * up * (do @ S0.transpose(1, 2))
    dk = A.transpose(1, 2) @ q + down * (v @ dS.transpose(1, 2))
    dv = P.transpose(1, 2) @ do + down * (k @ dS)
    dS0 = scale * (q * up).transpose(1, 2) @ do + full * dS
    back = lambda x: x.transpose(0, 1).reshape(n, G, H // G, x.shape[2]).sum(2)  # noqa: E731
    return back(dq), back(dk), dv.transpose(0, 1), dS0


class Problem:
    """Packed sequences with inputs on the GPU.  Rows that belong to nobody hold NaN, and so do slots that nobody resumes from."""

    def __init__(self, lens, H, G, dk, dv, dtype, seed=0, lead=0, tail=0, resume=None, slots=None, n_slots=None, rates=None, wide=0, scale=None, flags=0, backward=False):
        self.p = Packed(lens, lead, tail, seed, n_slots, slots, resume)
        self.H, self.G, self.dk, self.dv, self.dtype = H, G, dk, dv, dtype
        self.cfg = rb.make_linattn_config(H, G, dk, dv, dtype, scale, flags)
        self.scale = float(torch.tensor(self.cfg.scale, dtype=torch.float32))
        gen = torch.Generator().manual_seed(seed + 17)
        rows, p = self.p.rows, self.p
        nobody = torch.from_numpy(~p.mine())

        def rows_of(width):
            full = torch.randn((rows, width + wide), generator=gen).to(TORCH[dtype])
            full[nobody] = float("nan")
            full[:, width:] = float("nan")
            return full.cuda()[:, :width]

        self.q, self.k, self.v, self.do = rows_of(G * dk), rows_of(G * dk), rows_of(H * dv), rows_of(H * dv).contiguous()
        rates = torch.logspace(-0.5, -3.3, H, dtype=torch.float64) if rates is None else torch.tensor(rates, dtype=torch.float64)
        self.g = (-rates).float().cuda()
        self.s_in = torch.randn((p.n_slots, H, dk, dv), generator=gen)
        used = {int(p.slots[i]) for i in range(p.n) if p.resumes(i)}
        for s in range(p.n_slots):
            if s not in used:
                self.s_in[s] = float("nan")
        self.s_in = self.s_in.cuda()
        self.ds_out = torch.randn((p.n_slots, H, dk, dv), generator=gen).cuda()
        size = (rb.linattn_backward_workspace_size if backward else rb.linattn_ragged_workspace_size)(self.cfg, p.n, rows)
        self.ws = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")      # (as fp32: NaN)

    def out(self, width, value=-7.0):
        return torch.full((self.p.rows, width), value, dtype=TORCH[self.dtype], device="cuda")

    def run(self, s_in="own", s_out="fresh", **kw):
        """(o, s_out) of the call; untouched places hold -7."""
        o = self.out(self.H * self.dv)
        if isinstance(s_out, str):
            s_out = torch.full_like(self.s_in, -7.0)
        rb.rom_linattn_ragged(self.cfg, self.p.ragged, self.q, self.k, self.v, self.g, self.s_in if isinstance(s_in, str) else s_in, s_out, o, self.ws, **kw)
        return o, s_out

    def run_backward(self, ds_out="own", ds_in="fresh", s_in="own", **kw):
        dq, dk, dv = self.out(self.G * self.dk), self.out(self.G * self.dk), self.out(self.H * self.dv)
        if isinstance(ds_in, str):
            ds_in = torch.full_like(self.s_in, -7.0)
        rb.rom_linattn_backward(self.cfg, self.p.ragged, self.do, self.q, self.k, self.v, self.g, self.s_in if isinstance(s_in, str) else s_in,
                                self.ds_out if isinstance(ds_out, str) else ds_out, dq, dk, dv, ds_in, self.ws, **kw)
        return dq, dk, dv, ds_in

    def sequence(self, i):
        """(rows, q, k, v, do, S0, dS) of sequence i in 64 bits."""
        p, a, b = self.p, int(self.p.start[i]), int(self.p.start[i + 1])
        cut = lambda x, n: x[a:b].double().reshape(b - a, n, x.shape[1] // n)  # noqa: E731
        S0 = self.s_in[int(p.slots[i])].double() if p.resumes(i) else torch.zeros((self.H, self.dk, self.dv), dtype=torch.float64, device="cuda")
        dS = self.ds_out[int(p.slots[i])].double() if p.kept(i) else torch.zeros_like(S0)
        return slice(a, b), cut(self.q, self.G), cut(self.k, self.G), cut(self.v, self.H), cut(self.do, self.H), S0, dS


def units(n, inner, bf16_matrix, wide_state=False):
    """(relative error of an output, of a state) against the same sums of absolute values, for a sequence of n rows and inner width `inner`.

    fp32: a product of `inner` terms, its factors (decay, scale: 4 roundings), a chunk's sum of at most 128 terms in its turn, the state's decay over the chunks (3 roundings in
    each of at most n / 32 + 1, and three a cut): inner + 128 + 3 (n / 32 + 2) + 16 units of 2^-24.
    bf16 on the matrix instructions, besides: the scores and the state that a chunk meets lose half a step each (no term passes both), keys that enter a state that is no
    result 2^-16; a state that is one is a sum of exact products, of whose running value every step of 16 rows may drop 2^-23."""
    e = (inner + 128 + 3 * (n / 32 + 2) + 16) * U32
    return (e + (HALF_STEP["bf16"] + 2.0 ** -16 if bf16_matrix else 0.0), e + ((n / 16 + 16) * 2 * U32 if bf16_matrix else 0.0))


def near(got, ref, size, unit, store, what):
    """|got - ref| <= unit * size + half a step of the storage type, everywhere; and in the 2-norm as independent roundings add up."""
    got, ref = got.double().reshape(ref.shape), ref.double()
    assert torch.isfinite(got).all(), f"{what}: not finite"
    if not ref.numel():
        return
    tol = unit * size * (1 + HALF_STEP[store]) + HALF_STEP[store] * ref.abs() + 1e-37
    worst = float(((got - ref).abs() / tol).max())
    assert worst <= 1.0, f"{what}: {worst:.2f} times the bound"
    if ref.numel() >= 512:
        # Three independent roundings of half a step 2^-8 at most (scores or state, stored partial sum, output), each of a variance of at most a third of its square: together
        # 2^-8 of the norm.  fp32: sums of up to 1000 random terms, sqrt(1000) 2^-24 / 2, twice.
        rel = float((got - ref).norm() / ref.norm().clamp(min=1e-30))
        # A state on the matrix instructions: 2^-24 of the running sum dropped by each step of 16 rows on average, at most 32 steps before it moves to registers: 2^-19.
        most = HALF_STEP["bf16"] if store == "bf16" else 2.0 ** -19
        assert rel <= most, f"{what}: {rel:.2e} of the norm"


def check_forward(pr, o, s_out, tensor=None, kept_untouched=True):
    """Every row, state, and what has to stay as it was."""
    tensor = pr.dtype == "bf16" if tensor is None else tensor
    g, p = pr.g.double(), pr.p
    o3 = o.view(p.rows, pr.H, pr.dv)
    for i in range(p.n):
        rows, q, k, v, _, S0, _ = pr.sequence(i)
        ref, S = forward(q, k, v, g, S0, pr.scale)
        size, Ssize = forward(q.abs(), k.abs(), v.abs(), g, S0.abs(), abs(pr.scale))      # (sums of absolute values: of the scale too)
        eo, es = units(q.shape[0], pr.dk, tensor)
        near(o3[rows], ref, size, eo, pr.dtype, f"o of sequence {i}")
        if s_out is not None and p.kept(i):
            near(s_out[int(p.slots[i])], S, Ssize, es, "f32", f"state of sequence {i}")
    nobody = torch.from_numpy(~p.mine()).cuda()
    assert (o[nobody] == -7).all()
    if s_out is not None and kept_untouched:
        named = {int(s) for s in p.slots}
        for s in range(p.n_slots):
            if s not in named:
                assert (s_out[s] == -7).all()


def check_backward(pr, dq, dk, dv, ds_in, tensor=None, no_state=False):
    tensor = pr.dtype == "bf16" if tensor is None else tensor
    g, p = pr.g.double(), pr.p
    shape = lambda x, n: x.view(p.rows, n, x.shape[1] // n)  # noqa: E731
    for i in range(p.n):
        rows, q, k, v, do, S0, dS = pr.sequence(i)
        if no_state:
            dS = torch.zeros_like(dS)
        ref = backward(do, q, k, v, g, S0, dS, pr.scale)
        size = backward(do.abs(), q.abs(), k.abs(), v.abs(), g, S0.abs(), dS.abs(), abs(pr.scale))
        eo, es = units(q.shape[0], max(pr.dk, pr.dv) + pr.H // pr.G, tensor)
        near(shape(dq, pr.G)[rows], ref[0], size[0], eo, pr.dtype, f"dq of sequence {i}")
        near(shape(dk, pr.G)[rows], ref[1], size[1], eo, pr.dtype, f"dk of sequence {i}")
        near(shape(dv, pr.H)[rows], ref[2], size[2], eo, pr.dtype, f"dv of sequence {i}")
        if ds_in is not None and p.kept(i):
            here = ds_in[int(p.slots[i])]
            if p.resumes(i):
                near(here, ref[3], size[3], es, "f32", f"ds of sequence {i}")
            else:
                assert (here == 0).all()
    nobody = torch.from_numpy(~p.mine()).cuda()
    for x in (dq, dk, dv):
        assert (x[nobody] == -7).all()
    if ds_in is not None:
        named = {int(s) for s in p.slots}
        for s in range(p.n_slots):
            if s not in named:
                assert (ds_in[s] == -7).all()


# ---------------------------------------------------------------------------------------------- norm and rotation
def turn(n, angle, rot, interleaved, way=1.0):
    """Pairs of the first `rot` places of [rows, heads, d] turned by angle [rows, rot/2]."""
    i = torch.arange(rot // 2, device=n.device)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    c, s = torch.cos(angle)[:, None], way * torch.sin(angle)[:, None]
    y = n.clone()
    y[..., a] = n[..., a] * c - n[..., b] * s
    y[..., b] = n[..., b] * c + n[..., a] * s
    return y


def norm_rope(x, w, pos, inv_freq, rot, interleaved, eps):
    """x [rows, heads, d] in 64 bits."""
    n = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps) * w
    return turn(n, pos.double()[:, None] * inv_freq.double(), rot, interleaved) if rot else n


def norm_rope_backward(dy, x, w, pos, inv_freq, rot, interleaved, eps):
    """(dx, dw, sum of |terms| of dw)."""
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + eps)
    hat = x * r
    dn = turn(dy, pos.double()[:, None] * inv_freq.double(), rot, interleaved, -1.0) if rot else dy
    g = dn * w
    return r * (g - hat * (g * hat).mean(-1, keepdim=True)), (dn * hat).sum((0, 1)), (dn * hat).abs().sum((0, 1))

"""Performance cases of linear attention with a decay for each head, and of what prepares its queries and keys.

A layer of that kind projects a row to q | k | v, normalises every head of q and k and rotates it by its position (`rom_qk_norm_rope`), and then runs the recurrence

    S_t = lambda_h S_{t-1} + k_t v_t^T,     o_t = scale q_t S_t

over packed prompts (`rom_linattn_ragged`), over one token of many sequences (`rom_linattn_step`), or backwards in training (`rom_linattn_backward`,
`rom_qk_norm_rope_backward`).  Value heads may share the heads of q and k.  Decays are a fixed schedule over the heads, a geometric series of rates from 1/2 down to 1/2048.

q, k and v are columns of one projection's rows where the projection is what the call reads (the norm, and v of the recurrence); q and k of the recurrence are the norm's
contiguous outputs, of unit mean square.  Positions run on from where a prompt resumes.
"""
import math
import random

import torch

own = False

CHUNK = 128      # rows of a chunk of the plain form


def _attn(name, n_seq, rows, H, G, dk, dv, dtype="bf16", tail=0, mix="prompts", resume=False, op="ragged"):
    return {"name": name, "op": op, "n_seq": n_seq, "rows": rows, "tail": tail, "mix": mix, "resume": resume, "H": H, "G": G, "dk": dk, "dv": dv, "dtype": dtype}


def _step(name, B, H, G, dk, dv, dtype="bf16", padded=0):
    return {"name": name, "op": "step", "B": B, "padded": padded, "H": H, "G": G, "dk": dk, "dv": dv, "dtype": dtype}


def _norm(name, rows, Hq, Hk, d, rot, dtype="bf16", op="norm", interleaved=False, far=0):
    return {"name": name, "op": op, "rows": rows, "Hq": Hq, "Hk": Hk, "d": d, "rot": rot, "interleaved": interleaved, "far": far, "dtype": dtype}


def listed():
    return [
        # one 16384-token prompt through a layer as wide as the largest of the benchmark: 32 heads of 128
        _attn("attn_long", 1, 16384, 32, 32, 128, 128),
        # prompts of uneven lengths in pieces that resume, heads of 64 whose queries and keys are shared by pairs, the buffer not filled to its end
        _attn("attn_prompts", 23, 8191, 32, 16, 64, 64, tail=5, resume=True),
        # continuous batching in full precision: most sequences bring one token, a few a piece of their prompt, all resume
        _attn("attn_continuous_f32", 37, 531, 8, 8, 64, 64, "f32", mix="continuous", resume=True),
        # one user's next token: latency counts
        _step("attn_token_1", 1, 32, 32, 128, 128),
        # a full serving batch, some of its rows padding of a captured graph: states in and out of HBM
        _step("attn_tokens_256", 256, 32, 32, 128, 128, padded=9),
        # the gradient of a training batch of eight sequences
        _attn("attn_backward", 8, 16384, 32, 32, 128, 128, op="backward"),
        # of a few uneven sequences in full precision, one head of queries and keys for all
        _attn("attn_backward_f32", 5, 1203, 8, 1, 48, 64, "f32", op="backward", resume=True),
        # norm and rotation of the training batch's queries and keys
        _norm("norm_train", 16384, 32, 32, 128, 128),
        # of one token far into its sequence
        _norm("norm_token_1", 1, 32, 32, 128, 128, far=1000000),
        # of a batch of tokens in full precision, half of each head rotated, pairs next to each other
        _norm("norm_tokens_f32", 67, 24, 8, 96, 48, "f32", interleaved=True, far=30000),
        # the gradient of the training batch's norm and rotation
        _norm("norm_backward", 16384, 32, 32, 128, 128, op="norm_backward"),
        # of an odd number of rows and unequal head counts in full precision
        _norm("norm_backward_f32", 777, 12, 3, 80, 64, "f32", op="norm_backward"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["ragged", "ragged", "ragged", "step", "step", "backward", "backward", "norm", "norm_backward"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if op in ("norm", "norm_backward"):
        rows, d = _log_int(rng, 1, 16384 if dtype == "bf16" else 4096), 8 * rng.randint(2, 16)
        c = _norm("", rows, rng.randint(1, 32), rng.randint(1, 32), d, 16 * rng.randint(0, d // 16), dtype, op, rng.random() < 0.3, rng.choice([0, 5000, 2000000]))
    else:
        G = rng.choice([1, 2, 4, 8, 16])
        H = G * rng.choice([1, 1, 2, 4] if G <= 8 else [1, 2])
        dk, dv = rng.choice([64, 128, 8 * rng.randint(2, 16)]), rng.choice([64, 128, 8 * rng.randint(2, 16)])
        if op == "step":
            B = _log_int(rng, 1, 256)
            c = _step("", B, H, G, dk, dv, dtype, padded=rng.choice([0, B // 7]))
        else:
            rows = _log_int(rng, 1, 16384 if dtype == "bf16" else 4096)
            n_seq = _log_int(rng, 1, min(rows, 128))
            c = _attn("", n_seq, rows, H, G, dk, dv, dtype, rng.choice([0, 0, rng.randint(0, rows - n_seq)]), rng.choice(["prompts", "prompts", "continuous"]),
                      rng.random() < 0.5, op)
    del c["name"]
    return c


# ---------------------------------------------------------------------------------------------- inputs
class _Draw:
    def __init__(self, seed, dtype):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)
        self.dtype = torch.float32 if dtype == "f32" else torch.bfloat16

    def normal(self, shape, std=1.0, dtype=None):
        return torch.randn(shape, generator=self.g, device="cuda", dtype=torch.float32).mul_(std).to(dtype or self.dtype)

    def normal32(self, shape, std=1.0):
        return self.normal(shape, std, torch.float32)

    def scattered(self, shape):
        """Zeros of the storage type: what an output buffer holds before the first call."""
        return torch.zeros(shape, device="cuda", dtype=self.dtype)


def _lengths(c, seed):
    """Lengths of the packed sequences, rows - tail in all; now and then one is empty."""
    rng = random.Random(seed * 7919 + c["rows"])
    n, used = c["n_seq"], c["rows"] - c["tail"]
    if c["mix"] == "continuous":
        weight = [0.0 if rng.random() < 0.75 else rng.expovariate(1.0) for _ in range(n)]
    else:
        weight = [rng.expovariate(1.0) + 0.05 for _ in range(n)]
    if not any(weight):
        weight[rng.randrange(n)] = 1.0
    base = min(1, used // n)
    left = used - base * n
    lens = [base + int(left * w / sum(weight)) for w in weight]
    lens[weight.index(max(weight))] += used - sum(lens)
    if n > 3 and rng.random() < 0.5:      # a request that was cancelled: nothing of it is left in the batch
        i, j = rng.randrange(n - 1), n - 1
        lens[j] += lens[i]
        lens[i] = 0
    return lens


def _prepare_attention(c, seed, s, d):
    H, G, dk, dv = c["H"], c["G"], c["dk"], c["dv"]
    rng = random.Random(seed)
    if c["op"] == "step":
        rows, n_slots = c["B"], c["B"] + 3
        slots = rng.sample(range(n_slots), rows - c["padded"]) + [-1] * c["padded"]
    else:
        rows, n_slots = c["rows"], c["n_seq"] + 3
        starts = [0]
        for n in _lengths(c, seed):
            starts.append(starts[-1] + n)
        slots = rng.sample(range(n_slots), c["n_seq"])
        s["seq_start"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
        s["resume"] = torch.tensor([int(c["resume"] and rng.random() < 0.8) for _ in slots], dtype=torch.int32, device="cuda")
    s["slot"] = torch.tensor(slots, dtype=torch.int32, device="cuda")
    s["q"], s["k"] = d.normal((rows, G * dk)), d.normal((rows, G * dk))
    s["v"] = d.normal((rows, 2 * G * dk + H * dv))[:, 2 * G * dk:]
    rate = torch.logspace(-1.0, -11.0, H, base=2.0, dtype=torch.float64)
    s["log_decay"] = (-rate).float().cuda()
    s["s_in"], s["s_out"] = d.normal32((n_slots, H, dk, dv)), d.normal32((n_slots, H, dk, dv))
    if c["op"] == "backward":
        s["dout"], s["ds_out"], s["ds_in"] = d.normal((rows, H * dv)), s.pop("s_out").mul_(0.1), torch.zeros((n_slots, H, dk, dv), device="cuda")
        s["dq"], s["dk"], s["dv"] = d.scattered((rows, G * dk)), d.scattered((rows, G * dk)), d.scattered((rows, 2 * G * dk + H * dv))[:, 2 * G * dk:]
    else:
        s["o"] = d.scattered((rows, H * dv))


def _prepare_norm(c, seed, s, d):
    rows, Hq, Hk, w = c["rows"], c["Hq"], c["Hk"], c["d"]
    wide = (Hq + 2 * Hk) * w      # q | k | v of one projection
    x = d.normal((rows, wide), 1.7)
    s["q"], s["k"] = x[:, :Hq * w], x[:, Hq * w:(Hq + Hk) * w]
    s["w_q"], s["w_k"] = 1.0 + d.normal32((w,), 0.2), 1.0 + d.normal32((w,), 0.2)
    s["pos"] = (torch.randint(0, c["far"] + 1, (1,), generator=d.g, device="cuda") + torch.arange(rows, device="cuda")).to(torch.int32)
    i = torch.arange(c["rot"] // 2, device="cuda", dtype=torch.float64)
    s["inv_freq"] = torch.exp(-math.log(10000.0) * 2.0 * i / max(1, c["rot"])).float()
    if c["op"] == "norm":
        s["q_out"], s["k_out"] = d.scattered((rows, Hq * w)), d.scattered((rows, Hk * w))
    else:
        s["dq_out"], s["dk_out"] = d.normal((rows, Hq * w)), d.normal((rows, Hk * w))
        dx = d.scattered((rows, wide))
        s["dq"], s["dk"] = dx[:, :Hq * w], dx[:, Hq * w:(Hq + Hk) * w]
        s["dw_q"], s["dw_k"] = torch.zeros(w, device="cuda"), torch.zeros(w, device="cuda")


def prepare(case, seed):
    c, d = case, _Draw(seed, case["dtype"])
    s = {"case": dict(c)}
    (_prepare_norm if c["op"].startswith("norm") else _prepare_attention)(c, seed, s, d)
    if own:
        from paper_2506_18145_b200 import binding as rb
        if c["op"].startswith("norm"):
            s["cfg"] = rb.make_qk_config(c["Hq"], c["Hk"], c["d"], c["rot"], c["dtype"], eps=EPS, interleaved=c["interleaved"])
            size = rb.qk_norm_rope_backward_workspace_size(s["cfg"], c["rows"]) if c["op"] == "norm_backward" else 0
        else:
            s["cfg"] = rb.make_linattn_config(c["H"], c["G"], c["dk"], c["dv"], c["dtype"])
            size = 0
            if c["op"] != "step":
                s["seqs"] = rb.make_ragged(c["rows"], c["n_seq"] + 3, s["seq_start"], s["slot"], s["resume"])
                ask = rb.linattn_backward_workspace_size if c["op"] == "backward" else rb.linattn_ragged_workspace_size
                size = ask(s["cfg"], c["n_seq"], c["rows"])
        s["ws"] = torch.empty(size, dtype=torch.uint8, device="cuda") if size else None
    return s


EPS = 1e-6


# ---------------------------------------------------------------------------------------------- one pass
def run(s):
    c = s["case"]
    if own:
        return _run_own(s, c)
    return {"ragged": _plain_ragged, "step": _plain_step, "backward": _plain_backward, "norm": _plain_norm, "norm_backward": _plain_norm_backward}[c["op"]](s, c)


def _run_own(s, c):
    from paper_2506_18145_b200 import binding as rb
    op = c["op"]
    if op == "ragged":
        rb.rom_linattn_ragged(s["cfg"], s["seqs"], s["q"], s["k"], s["v"], s["log_decay"], s["s_in"], s["s_out"], s["o"], s["ws"])
        return {"o": s["o"], "state": s["s_out"]}
    if op == "step":
        rb.rom_linattn_step(s["cfg"], s["q"], s["k"], s["v"], s["log_decay"], s["slot"], s["s_in"], s["s_out"], s["o"])
        return {"o": s["o"], "state": s["s_out"]}
    if op == "backward":
        rb.rom_linattn_backward(s["cfg"], s["seqs"], s["dout"], s["q"], s["k"], s["v"], s["log_decay"], s["s_in"], s["ds_out"], s["dq"], s["dk"], s["dv"], s["ds_in"], s["ws"])
        return {"dq": s["dq"], "dk": s["dk"], "dv": s["dv"], "dstate": s["ds_in"]}
    if op == "norm":
        rb.rom_qk_norm_rope(s["cfg"], s["q"], s["k"], s["w_q"], s["w_k"], s["pos"], s["inv_freq"], s["q_out"], s["k_out"])
        return {"q": s["q_out"], "k": s["k_out"]}
    rb.rom_qk_norm_rope_backward(s["cfg"], s["dq_out"], s["dk_out"], s["q"], s["k"], s["w_q"], s["w_k"], s["pos"], s["inv_freq"], s["dq"], s["dk"], s["dw_q"], s["dw_k"], s["ws"])
    return {"dq": s["dq"], "dk": s["dk"], "dw_q": s["dw_q"], "dw_k": s["dw_k"]}


def _write_slots(pool, slot, value, keep):
    """pool[slot] = value for the rows that `keep` holds for; the others go to one spare row that is not returned."""
    n = pool.shape[0]
    wide = torch.cat([pool, pool[:1]])
    wide[torch.where(keep, slot, n)] = value
    pool.copy_(wide[:n])


def _power(s, exponent):
    """lambda_h ** exponent, [H, ...], zero where the exponent is negative (in 64 bits: far positions)."""
    e = exponent.double()
    x = s["log_decay"].double().view(-1, *[1] * e.dim()) * e.clamp(min=0)
    return torch.where(e >= 0, torch.exp(x), 0.0).float()


class _Chunks:
    """The packed rows laid out so that every sequence starts a chunk: which row each place holds, which sequence each chunk belongs to."""

    def __init__(self, s, c, reverse=False):
        start = s["seq_start"].long()
        self.start, self.length = start, start[1:] - start[:-1]
        count = (self.length + CHUNK - 1) // CHUNK
        self.first = torch.cumsum(count, 0) - count
        self.nc = (c["rows"] + CHUNK - 1) // CHUNK + c["n_seq"]
        chunk = torch.arange(self.nc, device="cuda")
        self.seq = (chunk[:, None] >= (self.first + count)[None, :]).sum(1).clamp(max=c["n_seq"] - 1)
        self.before = chunk - self.first[self.seq]      # chunks of the sequence ahead of this one
        at = self.before[:, None] * CHUNK + torch.arange(CHUNK, device="cuda")
        self.live = (at >= 0) & (at < self.length[self.seq][:, None])
        place = self.length[self.seq][:, None] - 1 - at if reverse else at
        self.row = torch.where(self.live, start[self.seq][:, None] + place, 0)
        self.count = self.live.sum(1)

    def heads(self, x, n, H):
        """[rows, n * d] -> [chunks, H, CHUNK, d] in fp32, zeros where a place holds no row; n heads shared by H."""
        x = x.float().reshape(x.shape[0], n, -1).repeat_interleave(H // n, 1)
        return torch.where(self.live[:, :, None, None], x[self.row], 0.0).transpose(1, 2)

    def back(self, y, out):
        """[chunks, H, CHUNK, d] into the rows of `out` that belong to a sequence."""
        flat = y.transpose(1, 2).reshape(self.nc * CHUNK, -1).to(out.dtype)
        wide = torch.cat([out, out[:1]])
        wide[torch.where(self.live, self.row, out.shape[0]).reshape(-1)] = flat
        out.copy_(wide[:-1])


def _recurrence(s, ch, q, k, v, init, scale, early=0):
    """o_i = q_i S_i and the last state of every sequence, S_i = lambda S_{i-1} + scale k_i v_i^T, q, k, v [chunks, H, CHUNK, d].
    `early`: the initial state meets the first row undecayed."""
    i = torch.arange(CHUNK, device="cuda")
    p = torch.matmul(q, k.transpose(2, 3)) * _power(s, i[:, None] - i[None, :]) * scale
    o = torch.matmul(p, v)
    tail = _power(s, torch.where(ch.live, ch.count[:, None] - 1 - i, -1)).transpose(0, 1)      # [chunks, H, CHUNK]
    own_state = torch.matmul((k * tail[..., None] * scale).transpose(2, 3), v)      # [chunks, H, dk, dv]
    n = torch.arange(ch.nc, device="cuda")
    gap = torch.where((ch.seq[:, None] == ch.seq[None, :]) & (ch.before[:, None] >= 0), n[:, None] - n[None, :] - 1, -1)
    mix = _power(s, torch.where(gap >= 0, gap * CHUNK, -1))      # [H, chunks, chunks]
    flat = own_state.transpose(0, 1).reshape(mix.shape[0], ch.nc, -1)
    into = torch.bmm(mix, flat).view(mix.shape[0], ch.nc, *own_state.shape[2:]).transpose(0, 1)
    lead = ch.before * CHUNK      # rows of the sequence ahead of the chunk
    since = torch.where(ch.before > 0, lead - early, lead)
    into = into + _power(s, since).t()[:, :, None, None] * init[ch.seq]
    first = torch.where(ch.before > 0, 0, early)[:, None]
    o = o + _power(s, torch.where(ch.live, i + 1 - first, -1)).transpose(0, 1)[..., None] * torch.matmul(q, into)
    last = (ch.first + (ch.length + CHUNK - 1) // CHUNK - 1).clamp(min=0)
    end = _power(s, ch.count[last] - first[last, 0]).t()[:, :, None, None] * into[last] + own_state[last]
    return o, torch.where((ch.length > 0)[:, None, None, None], end, init)


def _initial(s):
    return torch.where((s["resume"] == 0)[:, None, None, None], 0.0, s["s_in"][s["slot"].long()])


def _plain_ragged(s, c):
    H, G, ch = c["H"], c["G"], _Chunks(s, c)
    scale = c["dk"] ** -0.5
    o, last = _recurrence(s, ch, ch.heads(s["q"], G, H) * scale, ch.heads(s["k"], G, H), ch.heads(s["v"], H, H), _initial(s), 1.0)
    ch.back(o, s["o"])
    _write_slots(s["s_out"], s["slot"].long(), last, torch.ones_like(s["slot"], dtype=torch.bool))
    return {"o": s["o"], "state": s["s_out"]}


def _plain_step(s, c):
    H, G, B, slot = c["H"], c["G"], c["B"], s["slot"].long()
    live = slot >= 0
    q, k = (x.float().view(B, G, -1).repeat_interleave(H // G, 1) for x in (s["q"], s["k"]))
    lam = torch.exp(s["log_decay"])[:, None, None]
    S = lam * s["s_in"][slot.clamp(min=0)] + k[..., :, None] * s["v"].float().view(B, H, -1)[..., None, :]
    o = (c["dk"] ** -0.5 * torch.matmul(q[..., None, :], S)).view(B, -1)
    s["o"].copy_(torch.where(live[:, None], o.to(s["o"].dtype), s["o"]))
    _write_slots(s["s_out"], slot, S, live)
    return {"o": s["o"], "state": s["s_out"]}


def _plain_backward(s, c):
    H, G, dk, dv, ch = c["H"], c["G"], c["dk"], c["dv"], _Chunks(s, c)
    scale = dk ** -0.5
    do, v, k = ch.heads(s["dout"], H, H), ch.heads(s["v"], H, H), ch.heads(s["k"], G, H)
    dq, _ = _recurrence(s, ch, do * scale, v, k, _initial(s).transpose(2, 3), 1.0)
    shared = lambda g: g.reshape(ch.nc, G, H // G, CHUNK, dk).sum(2)  # noqa: E731
    ch.back(shared(dq), s["dq"])
    del dq
    rv = _Chunks(s, c, reverse=True)
    do, v, k, q = rv.heads(s["dout"], H, H), rv.heads(s["v"], H, H), rv.heads(s["k"], G, H), rv.heads(s["q"], G, H)
    at_end = s["ds_out"][s["slot"].long()]
    dv_, R = _recurrence(s, rv, k, q, do, at_end, scale, early=1)
    rv.back(dv_, s["dv"])
    del dv_
    dk_, _ = _recurrence(s, rv, v, do, q, at_end.transpose(2, 3), scale, early=1)
    rv.back(shared(dk_), s["dk"])
    lam = torch.exp(s["log_decay"])[None, :, None, None]
    ds = torch.where((ch.length > 0)[:, None, None, None], lam * R, R)
    ds = torch.where((s["resume"] == 0)[:, None, None, None], 0.0, ds)
    _write_slots(s["ds_in"], s["slot"].long(), ds, torch.ones_like(s["slot"], dtype=torch.bool))
    return {"dq": s["dq"], "dk": s["dk"], "dv": s["dv"], "dstate": s["ds_in"]}


def _angles(s):
    a = s["pos"].double()[:, None, None] * s["inv_freq"].double()
    return torch.cos(a).float(), torch.sin(a).float()


def _rotate(n, cos, sin, c):
    """Pairs of the first `rot` places of [rows, heads, d] turned by the angles."""
    rot = c["rot"]
    if c["interleaved"]:
        a, b = n[..., 0:rot:2], n[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(2)
    else:
        a, b = n[..., :rot // 2], n[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, n[..., rot:]], -1)


def _plain_norm(s, c):
    cos, sin = _angles(s)

    def one(x, w, out):
        x = x.float().reshape(x.shape[0], -1, c["d"])
        n = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w
        return out.copy_(_rotate(n, cos, sin, c).flatten(1).to(out.dtype))

    return {"q": one(s["q"], s["w_q"], s["q_out"]), "k": one(s["k"], s["w_k"], s["k_out"])}


def _plain_norm_backward(s, c):
    cos, sin = _angles(s)

    def one(x, w, dy, dx, dw):
        x, dy = x.float().reshape(x.shape[0], -1, c["d"]), dy.float().view(x.shape[0], -1, c["d"])
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        dn, hat = _rotate(dy, cos, -sin, c), x * r
        g = dn * w
        dx.copy_((r * (g - hat * (g * hat).mean(-1, keepdim=True))).flatten(1).to(dx.dtype))
        return dx, dw.copy_((dn * hat).flatten(0, 1).sum(0))

    dq, dw_q = one(s["q"], s["w_q"], s["dq_out"], s["dq"], s["dw_q"])
    dk, dw_k = one(s["k"], s["w_k"], s["dk_out"], s["dk"], s["dw_k"])
    return {"dq": dq, "dk": dk, "dw_q": dw_q, "dw_k": dw_k}


# ---------------------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    if c["op"].startswith("norm"):
        n = c["rows"] * (c["Hq"] + c["Hk"]) * c["d"]
        back = c["op"] == "norm_backward"
        return {"bytes": n * e * (3 if back else 2) + 4 * c["rows"] + 2 * c["rot"] + 8 * c["d"] * (2 if back else 1), "flops": n * (14 if back else 8)}
    H, G, dk, dv = c["H"], c["G"], c["dk"], c["dv"]
    state = H * dk * dv
    if c["op"] == "step":
        rows = seqs = read = c["B"] - c["padded"]
    else:
        rows, seqs = c["rows"] - c["tail"], c["n_seq"]
        read = 0.8 * seqs if c["resume"] else 0
    qk, vo = rows * G * dk * e, rows * H * dv * e
    if c["op"] == "backward":      # the gradient of an initial state is written for every sequence, the last one's is read for every one
        return {"bytes": 4 * qk + 3 * vo + (read + 2 * seqs) * state * 4 + 4 * H, "flops": rows * state * 10}
    return {"bytes": 2 * qk + 2 * vo + (read + seqs) * state * 4 + 4 * H, "flops": rows * state * 4}


# ---------------------------------------------------------------------------------------------- in 64 bits, from the definitions
def exact(case, seed):
    s = prepare(case, seed)
    s = {k: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v for k, v in s.items()}
    if case["op"].startswith("norm"):
        return _exact_norm(s, case)
    return (_exact_backward if case["op"] == "backward" else _exact_attention)(s, case)


def _sequences(s):
    """(slot, resumes, first row, length), the longest first; a generated token is a sequence of one row that resumes, none without a slot."""
    slots = s["slot"].tolist()
    if "seq_start" not in s:
        return [(q, True, i, 1) for i, q in enumerate(slots) if q >= 0]
    st = s["seq_start"].tolist()
    return sorted([(q, bool(r), st[i], st[i + 1] - st[i]) for i, (q, r) in enumerate(zip(slots, s["resume"].tolist()))], key=lambda q: -q[3])


def _exact_attention(s, c):
    """All sequences side by side, token by token."""
    H, G, dk, dv = c["H"], c["G"], c["dk"], c["dv"]
    share = torch.arange(H, device="cuda") // (H // G)
    q, k, v = s["q"].reshape(-1, G, dk), s["k"].reshape(-1, G, dk), s["v"].reshape(-1, H, dv)
    lam, o = torch.exp(s["log_decay"])[:, None, None], s["o"].view(-1, H, dv)
    seqs = _sequences(s)
    S = torch.stack([s["s_in"][a] if r else torch.zeros_like(s["s_in"][a]) for a, r, _, _ in seqs])
    lens, first = [n for _, _, _, n in seqs], torch.tensor([f for _, _, f, _ in seqs], device="cuda")
    live = len(lens)
    for t in range(lens[0]):
        while lens[live - 1] <= t:
            live -= 1
        r = first[:live] + t
        S[:live].mul_(lam).add_(k[r][:, share, :, None] * v[r][:, :, None, :])
        o[r] = dk ** -0.5 * torch.einsum("nha,nhac->nhc", q[r][:, share], S[:live])
    for i, (slot, _, _, _) in enumerate(seqs):
        s["s_out"][slot] = S[i]
    return {"o": s["o"], "state": s["s_out"]}


def _exact_backward(s, c):
    H, G, dk, dv = c["H"], c["G"], c["dk"], c["dv"]
    share = torch.arange(H, device="cuda") // (H // G)
    q, k, v, do = s["q"].reshape(-1, G, dk), s["k"].reshape(-1, G, dk), s["v"].reshape(-1, H, dv), s["dout"].view(-1, H, dv)
    lam, scale = torch.exp(s["log_decay"])[:, None, None], dk ** -0.5
    dq, dk_, dv_ = s["dq"].view(-1, G, dk), s["dk"].view(-1, G, dk), torch.zeros_like(v)
    seqs = _sequences(s)
    lens, first = [n for _, _, _, n in seqs], torch.tensor([f for _, _, f, _ in seqs], device="cuda")
    S = torch.stack([s["s_in"][a] if r else torch.zeros_like(s["s_in"][a]) for a, r, _, _ in seqs])
    live = len(lens)
    for t in range(lens[0]):
        while lens[live - 1] <= t:
            live -= 1
        r = first[:live] + t
        S[:live].mul_(lam).add_(k[r][:, share, :, None] * v[r][:, :, None, :])
        dq[r] = scale * torch.einsum("nhc,nhac->nha", do[r], S[:live]).view(live, G, H // G, dk).sum(2)
    R = torch.stack([s["ds_out"][a] for a, _, _, _ in seqs])      # the gradient of the state behind row t, and then lambda times it
    live = 0
    for t in range(lens[0] - 1, -1, -1):
        while live < len(lens) and lens[live] > t:
            live += 1
        r = first[:live] + t
        R[:live].add_(scale * q[r][:, share, :, None] * do[r][:, :, None, :])
        dk_[r] = torch.einsum("nhac,nhc->nha", R[:live], v[r]).view(live, G, H // G, dk).sum(2)
        dv_[r] = torch.einsum("nhac,nha->nhc", R[:live], k[r][:, share])
        R[:live].mul_(lam)
    s["dv"].copy_(torch.where((torch.arange(c["rows"], device="cuda") < c["rows"] - c["tail"])[:, None], dv_.flatten(1), s["dv"]))
    for i, (slot, resumes, _, _) in enumerate(seqs):
        s["ds_in"][slot] = R[i] if resumes else 0.0
    return {"dq": s["dq"], "dk": s["dk"], "dv": s["dv"], "dstate": s["ds_in"]}


def _exact_norm(s, c):
    """As one matrix a row: y = M (x w / |x|), M the rotation; its gradient by the transpose and by the quotient rule."""
    d, rot = c["d"], c["rot"]
    i = torch.arange(rot // 2, device="cuda")
    a, b = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + rot // 2)
    angle = s["pos"].double()[:, None, None] * s["inv_freq"]

    def turn(n, way):
        y = n.clone()
        y[..., a] = n[..., a] * torch.cos(angle) - way * n[..., b] * torch.sin(angle)
        y[..., b] = n[..., b] * torch.cos(angle) + way * n[..., a] * torch.sin(angle)
        return y

    found = {}
    for name in ("q", "k"):
        x, w = s[name].reshape(c["rows"], -1, d), s["w_" + name]
        size = torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
        if c["op"] == "norm":
            found[name] = turn(w * x / size, 1.0).flatten(1)
            continue
        dn = turn(s["d" + name + "_out"].view(c["rows"], -1, d), -1.0)
        found["d" + name] = (dn * w / size - x * (dn * w * x).sum(-1, keepdim=True) / (d * size ** 3)).flatten(1)
        found["dw_" + name] = (dn * x / size).sum((0, 1))
    return found

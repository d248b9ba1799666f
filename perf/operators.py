"""Performance cases of the serving operators: prompts and generated tokens of many sequences in one call.

A server of Routing-Mamba layers holds one conv window and one scan state per live sequence, in pools indexed by slot.  Prompts of
different lengths arrive packed one behind the other in a single buffer (`rom_conv_ragged`, `rom_scan_ragged`); generated tokens come one
per sequence (`rom_conv_step`, `rom_scan_step`); the hybrid model's FFN-MoE then runs on those few tokens (`rom_ffn_moe_step`).

Widths, dt ranks, expert counts and dtypes are those of the seeded workloads in `paper_2506_18145_b200/synth.py`.  Activations are O(1),
Delta is log-uniform in [1e-3, 1e-1] as at the start of training, A is negative and near -(n+1).  x and z are the two halves of one
projection's rows (pitch 2 d_inner), B and C columns of the x Proj's fp32 rows (pitch dt_rank + 2 d_state): what the calls are handed in use.
"""
import math
import random

import torch

own = False

N_STATE, D_CONV = 16, 4


def _conv(name, n_seq, rows, d_inner, dtype="bf16", tail=0, mix="prompts", resume=False):
    return {"name": name, "op": "conv_ragged", "n_seq": n_seq, "rows": rows, "tail": tail, "mix": mix, "resume": resume, "d_inner": d_inner, "dtype": dtype}


def _scan(name, n_seq, rows, d_inner, dtype="bf16", tail=0, mix="prompts", resume=False, disc_mode=0):
    return {"name": name, "op": "scan_ragged", "n_seq": n_seq, "rows": rows, "tail": tail, "mix": mix, "resume": resume, "d_inner": d_inner, "dtype": dtype,
            "disc_mode": disc_mode}


def _step(name, op, B, d_inner, dtype="bf16", padded=0, disc_mode=0):
    return {"name": name, "op": op, "B": B, "padded": padded, "d_inner": d_inner, "dtype": dtype, "disc_mode": disc_mode}


def _ffn(name, B, d_model, d_ff, E, K, dtype="bf16"):
    return {"name": name, "op": "ffn_step", "B": B, "d_model": d_model, "d_ff": d_ff, "E": E, "K": K, "dtype": dtype}


def listed():
    return [
        # a batch of a few long prompts through a 1.3B layer, the buffer not filled to its end
        _conv("conv_prompts", 5, 16384, 4096, tail=37),
        # continuous batching in full precision: most sequences bring one token, a few a piece of their prompt, all resume
        _conv("conv_continuous_f32", 37, 531, 512, "f32", mix="continuous", resume=True),
        # the scan behind those two: one 16384-token prompt, the longest sequence of the benchmark
        _scan("scan_long", 1, 16384, 4096),
        # prompts of uneven lengths through a 353M layer, in pieces that resume; Euler form of B-bar
        _scan("scan_prompts", 23, 8191, 2048, tail=5, resume=True, disc_mode=1),
        # the full-precision configuration on a small mixed batch
        _scan("scan_continuous_f32", 37, 531, 512, "f32", mix="continuous", resume=True),
        # one user's next token: latency counts
        _step("conv_token_1", "conv_step", 1, 4096),
        _step("scan_token_1", "scan_step", 1, 4096),
        # a full serving batch, some of its rows padding of a captured graph: states in and out of HBM
        _step("conv_tokens_512", "conv_step", 512, 4096, padded=19),
        _step("scan_tokens_512", "scan_step", 512, 4096, padded=19),
        # the FFN-MoE of one token, hidden width 4 x d_model as in the benchmark
        _ffn("ffn_token_1", 1, 2048, 8192, 8, 1),
        # of a batch of 64, two experts of sixteen each: every expert's weights are read
        _ffn("ffn_tokens_64", 64, 2048, 8192, 16, 2),
        # of a few tokens in full precision
        _ffn("ffn_tokens_f32", 5, 256, 1024, 4, 2, "f32"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["conv_ragged", "scan_ragged", "scan_ragged", "conv_step", "scan_step", "ffn_step", "ffn_step"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if op in ("conv_ragged", "scan_ragged"):
        d_inner = 64 * rng.randint(4, 64) if dtype == "bf16" else 64 * rng.randint(4, 16)
        rows = _log_int(rng, 1, 16384 if dtype == "bf16" else 4096)
        n_seq = _log_int(rng, 1, min(rows, 128))
        kw = {"tail": rng.choice([0, 0, rng.randint(0, rows - n_seq)]), "mix": rng.choice(["prompts", "prompts", "continuous"]), "resume": rng.random() < 0.5}
        c = _conv("", n_seq, rows, d_inner, dtype, **kw) if op == "conv_ragged" else _scan("", n_seq, rows, d_inner, dtype, disc_mode=rng.randint(0, 1), **kw)
    elif op in ("conv_step", "scan_step"):
        B = _log_int(rng, 1, 512)
        c = _step("", op, B, 64 * rng.randint(4, 64), dtype, padded=rng.choice([0, B // 7]), disc_mode=rng.randint(0, 1))
    else:
        E = rng.choice([4, 8, 8, 16])
        d_model, wide = (64 * rng.randint(4, 32), rng.choice([2, 3, 4])) if dtype == "bf16" else (64 * rng.randint(2, 8), 4)
        c = _ffn("", _log_int(rng, 1, 64), d_model, -(-d_model * wide // 128) * 128, E, rng.choice([1, 1, 2]), dtype)
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

    def uniform(self, shape):
        return torch.rand(shape, generator=self.g, device="cuda", dtype=torch.float32)


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


def _prepare_ragged(c, seed, s, d):
    lens, n = _lengths(c, seed), c["n_seq"]
    starts = [0]
    for k in lens:
        starts.append(starts[-1] + k)
    rng = random.Random(seed)
    n_slots = n + 3
    slot = rng.sample(range(n_slots), n)
    s["seq_start"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    s["slot"] = torch.tensor(slot, dtype=torch.int32, device="cuda")
    s["resume"] = torch.tensor([int(c["resume"] and rng.random() < 0.8) for _ in lens], dtype=torch.int32, device="cuda")
    return n_slots


def _conv_inputs(s, d, rows, De, n_slots):
    s["x"] = d.normal((rows, 2 * De))[:, :De]
    s["w_conv"], s["b_conv"] = d.normal((D_CONV, De), 0.5), d.normal32((De,), 0.1)
    s["state_in"], s["state_out"] = d.normal32((n_slots, D_CONV - 1, De)), d.normal32((n_slots, D_CONV - 1, De))
    s["y"] = torch.zeros((rows, De), dtype=d.dtype, device="cuda")


def _scan_inputs(s, d, rows, De, n_slots):
    R = De // 32
    x_dbl = d.normal32((rows, R + 2 * N_STATE))
    n = torch.arange(1, N_STATE + 1, dtype=torch.float32, device="cuda")
    s["u"], s["z"] = d.normal((rows, De)), d.normal((rows, 2 * De))[:, De:]
    s["delta"] = torch.exp(d.uniform((rows, De)) * (math.log(1e-1) - math.log(1e-3)) + math.log(1e-3))
    s["A"] = (-n[None, :] * (0.5 + d.uniform((De, N_STATE)))).contiguous()
    s["Bm"], s["Cm"] = x_dbl[:, R:R + N_STATE], x_dbl[:, R + N_STATE:]
    s["D"] = 1.0 + d.normal32((De,), 0.1)
    s["h0"], s["h_last"] = d.normal32((n_slots, De, N_STATE), 0.2), d.normal32((n_slots, De, N_STATE), 0.2)
    s["y"] = torch.zeros((rows, De), dtype=d.dtype, device="cuda")


def prepare(case, seed):
    c, d = case, _Draw(seed, case["dtype"])
    s = {"case": dict(c)}
    if c["op"] in ("conv_ragged", "scan_ragged"):
        n_slots = _prepare_ragged(c, seed, s, d)
        (_conv_inputs if c["op"] == "conv_ragged" else _scan_inputs)(s, d, c["rows"], c["d_inner"], n_slots)
        dims = (1, c["rows"], 64, c["d_inner"], 1, 1)
    elif c["op"] in ("conv_step", "scan_step"):
        B, n_slots = c["B"], c["B"] + 3
        slots = random.Random(seed).sample(range(n_slots), B - c["padded"]) + [-1] * c["padded"]
        s["slot"] = torch.tensor(slots, dtype=torch.int32, device="cuda")
        (_conv_inputs if c["op"] == "conv_step" else _scan_inputs)(s, d, B, c["d_inner"], n_slots)
        dims = (B, 1, 64, c["d_inner"], 1, 1)
    else:
        B, Dm, F, E, K = c["B"], c["d_model"], c["d_ff"], c["E"], c["K"]
        s["W_gu"], s["W_down"] = d.normal((E, 2 * F, Dm), Dm ** -0.5), d.normal((E, Dm, F), F ** -0.5)
        s["x"] = d.normal((B, Dm))
        logit = d.normal32((B, E))
        s["topk_idx"] = torch.topk(logit, K, dim=1).indices.to(torch.int32).contiguous()
        s["gates"] = torch.softmax(logit, 1).gather(1, s["topk_idx"].long()).contiguous()
        s["out"] = torch.zeros((B, Dm), dtype=d.dtype, device="cuda")
        dims = (B, 1, Dm, 64, E, K)
    if own:
        from paper_2506_18145_b200 import binding as rb
        B, L, Dm, De, E, K = dims
        s["cfg"] = cfg = rb.make_config(B, L, Dm, De, N_STATE, D_CONV, 16, E, K, c["dtype"], disc_mode=c.get("disc_mode", 0))
        if "seq_start" in s:
            s["ragged"] = rb.make_ragged(c["rows"], n_slots, s["seq_start"], s["slot"], s["resume"])
        size = {"scan_ragged": lambda: rb.scan_ragged_workspace_size(cfg, c["n_seq"], c["rows"]), "ffn_step": lambda: rb.ffn_moe_step_workspace_size(cfg, c["d_ff"])}
        if c["op"] in size:
            s["ws"] = torch.empty(size[c["op"]](), dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------- one pass
def run(s):
    c = s["case"]
    if own:
        return _run_own(s, c)
    return {"conv_ragged": _plain_conv_ragged, "scan_ragged": _plain_scan_ragged, "conv_step": _plain_conv_step, "scan_step": _plain_scan_step,
            "ffn_step": _plain_ffn}[c["op"]](s, c)


def _run_own(s, c):
    from paper_2506_18145_b200 import binding as rb
    op = c["op"]
    if op == "conv_ragged":
        rb.rom_conv_ragged(s["cfg"], s["ragged"], s["x"], s["w_conv"], s["b_conv"], s["state_in"], s["state_out"], s["y"])
        return {"y": s["y"], "state": s["state_out"]}
    if op == "scan_ragged":
        rb.rom_scan_ragged(s["cfg"], s["ragged"], s["u"], s["delta"], s["A"], s["Bm"], s["Cm"], s["D"], s["z"], s["h0"], s["h_last"], s["y"], s["ws"])
        return {"y": s["y"], "state": s["h_last"]}
    if op == "conv_step":
        rb.rom_conv_step(s["cfg"], s["x"], s["w_conv"], s["b_conv"], s["slot"], s["state_in"], s["state_out"], s["y"])
        return {"y": s["y"], "state": s["state_out"]}
    if op == "scan_step":
        rb.rom_scan_step(s["cfg"], s["u"], s["delta"], s["A"], s["Bm"], s["Cm"], s["D"], s["z"], s["slot"], s["h0"], s["h_last"], s["y"])
        return {"y": s["y"], "state": s["h_last"]}
    rb.rom_ffn_moe_step(s["cfg"], c["d_ff"], s["W_gu"], s["W_down"], s["x"], s["topk_idx"], s["gates"], s["out"], s["ws"])
    return {"out": s["out"]}


def _silu(v):
    return v / (1.0 + torch.exp(-v))


def _rows_of(s):
    """For every packed row: its sequence (n_seq behind the last one), its place in it; for every sequence: its first and last row."""
    start = s["seq_start"].long()
    row = torch.arange(s["y"].shape[0], device="cuda")
    seq = (row[:, None] >= start[None, 1:]).sum(1)
    return row, seq, row - start[seq.clamp(max=len(start) - 2)], start


def _write_slots(pool, slot, value, keep):
    """pool[slot] = value for the rows that `keep` holds for; the others go to one spare row that is not returned."""
    n = pool.shape[0]
    wide = torch.cat([pool, pool[:1]])
    wide[torch.where(keep, slot, n)] = value
    pool.copy_(wide[:n])


def _plain_conv_ragged(s, c):
    row, seq, at, start = _rows_of(s)
    slot = s["slot"].long()
    fresh = s["resume"] == 0
    win = torch.where(fresh[:, None, None], 0.0, s["state_in"][slot])      # [n_seq, 3, De]
    x, w = s["x"].float(), s["w_conv"].float()
    own_seq = seq.clamp(max=len(start) - 2)
    back = [torch.where((at >= k)[:, None], x[(row - k).clamp(min=0)], win[own_seq, (D_CONV - 1 - k + at).clamp(max=D_CONV - 2)]) for k in (3, 2, 1)]
    pre = s["b_conv"] + back[0] * w[0] + back[1] * w[1] + back[2] * w[2] + x * w[3]
    y = torch.where((seq < len(start) - 1)[:, None], _silu(pre).to(s["y"].dtype), s["y"])
    s["y"].copy_(y)
    length = start[1:] - start[:-1]
    j = torch.arange(D_CONV - 1, device="cuda")
    from_end = length[:, None] - (D_CONV - 1) + j[None, :]      # place in the sequence of window entry j; negative: in the old window
    new = torch.where((from_end >= 0)[:, :, None], x[(start[:-1, None] + from_end).clamp(0, len(row) - 1)],
                      win.gather(1, (from_end + D_CONV - 1).clamp(0, D_CONV - 2)[:, :, None].expand(-1, -1, win.shape[2])))
    _write_slots(s["state_out"], slot, new, torch.ones_like(fresh))
    return {"y": s["y"], "state": s["state_out"]}


def _decay_input(s, c, u, delta):
    """exp(Delta A) and B-bar u of rows [..., De, 1], for all 16 states."""
    x = delta[..., None] * s["A"]
    inp = u[..., None] * s["Bm"][:, None, :]
    return torch.exp(x), (torch.expm1(x) / s["A"] if c["disc_mode"] == 0 else delta[..., None]) * inp


def _scan_output(s, h, u):
    y = (h * s["Cm"][:, None, :]).sum(-1) + s["D"] * u
    return (y * _silu(s["z"].float())).to(s["y"].dtype)


def _plain_scan_ragged(s, c):
    """The recurrence as a scan by doubling: after the step of width k, (a, b) of a row is the map over its last 2k rows."""
    row, seq, at, start = _rows_of(s)
    n_seq, slot = len(start) - 1, s["slot"].long()
    valid = seq < n_seq
    init = torch.where((s["resume"] == 0)[:, None, None], 0.0, s["h0"][slot])
    u = s["u"].float()
    a, b = _decay_input(s, c, u, s["delta"])
    first = torch.where(s["seq_start"][:-1] < s["seq_start"][1:], start[:-1], len(row))      # (an empty sequence has no first row)
    b = torch.cat([b, b[:1]])
    a = torch.cat([a, a[:1]])
    b[first] += a[first] * init
    a[first] = 0.0
    a, b = a[:-1], b[:-1]
    k = 1
    while k < len(row):
        b = torch.cat([b[:k], b[k:] + a[k:] * b[:-k]])
        a = torch.cat([a[:k], a[k:] * a[:-k]])
        k *= 2
    s["y"].copy_(torch.where(valid[:, None], _scan_output(s, b, u), s["y"]))
    length = start[1:] - start[:-1]
    last = torch.where((length > 0)[:, None, None], b[(start[1:] - 1).clamp(min=0)], init)
    _write_slots(s["h_last"], slot, last, torch.ones_like(slot, dtype=torch.bool))
    return {"y": s["y"], "state": s["h_last"]}


def _plain_conv_step(s, c):
    slot = s["slot"].long()
    live = slot >= 0
    x, w = s["x"].float(), s["w_conv"].float()
    win = torch.cat([s["state_in"][slot.clamp(min=0)], x[:, None, :]], 1)      # [B, 4, De]
    y = _silu(s["b_conv"] + (win * w[None]).sum(1)).to(s["y"].dtype)
    s["y"].copy_(torch.where(live[:, None], y, s["y"]))
    _write_slots(s["state_out"], slot, win[:, 1:], live)
    return {"y": s["y"], "state": s["state_out"]}


def _plain_scan_step(s, c):
    slot = s["slot"].long()
    live = slot >= 0
    u = s["u"].float()
    a, b = _decay_input(s, c, u, s["delta"])
    h = a * s["h0"][slot.clamp(min=0)] + b
    s["y"].copy_(torch.where(live[:, None], _scan_output(s, h, u), s["y"]))
    _write_slots(s["h_last"], slot, h, live)
    return {"y": s["y"], "state": s["h_last"]}


def _plain_ffn(s, c):
    x, F, idx, gates = s["x"].float(), c["d_ff"], s["topk_idx"].long(), s["gates"]
    if c["B"] * c["K"] <= c["E"]:      # few choices: only the chosen experts' weights
        W_gu, W_down = s["W_gu"][idx].float(), s["W_down"][idx].float()      # [B, K, ...]
        gu = torch.matmul(W_gu, x[:, None, :, None])[..., 0]
        h = _silu(gu[..., :F]) * gu[..., F:]
        out = (torch.matmul(W_down, h[..., None])[..., 0] * gates[..., None]).sum(1)
    else:                              # all experts on all tokens, weighted by the gate (zero where not chosen)
        g = (gates[..., None] * (idx[..., None] == torch.arange(c["E"], device="cuda"))).sum(1)      # [B, E]
        gu = torch.matmul(x, s["W_gu"].float().transpose(1, 2))      # [E, B, 2F]
        h = _silu(gu[..., :F]) * gu[..., F:]
        out = (torch.matmul(h, s["W_down"].float().transpose(1, 2)) * g.t()[:, :, None]).sum(0)
    s["out"].copy_(out.to(s["out"].dtype))
    return {"out": s["out"]}


# ---------------------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    if c["op"] in ("conv_ragged", "scan_ragged", "conv_step", "scan_step"):
        De = c["d_inner"]
        if c["op"].endswith("ragged"):
            rows, seqs = c["rows"] - c["tail"], c["n_seq"]
            read = 0.8 * seqs if c["resume"] else 0
        else:
            rows = seqs = read = c["B"] - c["padded"]
        if c["op"].startswith("conv"):
            return {"bytes": rows * De * 2 * e + (D_CONV * e + 4) * De + (read + seqs) * (D_CONV - 1) * De * 4, "flops": rows * De * (2 * D_CONV + 4)}
        return {"bytes": rows * (De * (3 * e + 4) + 8 * N_STATE) + De * (4 * N_STATE + 4) + (read + seqs) * De * N_STATE * 4, "flops": rows * De * (N_STATE * 7 + 6)}
    B, Dm, F, E, K = c["B"], c["d_model"], c["d_ff"], c["E"], c["K"]
    experts = E * (1.0 - (1.0 - K / E) ** B)      # experts that B tokens choose, on average
    return {"bytes": experts * 3 * F * Dm * e + 2 * B * Dm * e + 8 * B * K, "flops": 6.0 * B * K * F * Dm}


# ---------------------------------------------------------------------------------------------- in 64 bits, from the definitions
def exact(case, seed):
    s = prepare(case, seed)
    s = {k: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v for k, v in s.items()}
    return {"conv_ragged": _exact_conv, "scan_ragged": _exact_scan, "conv_step": _exact_conv, "scan_step": _exact_scan, "ffn_step": _exact_ffn}[case["op"]](s, case)


def _sequences(s):
    """(slot, resumes, first row, length) of every sequence; a generated token is a sequence of one row that resumes, none without a slot."""
    slots = s["slot"].tolist()
    if "seq_start" not in s:
        return [(q, True, i, 1) for i, q in enumerate(slots) if q >= 0]
    st = s["seq_start"].tolist()
    return [(q, bool(r), st[i], st[i + 1] - st[i]) for i, (q, r) in enumerate(zip(slots, s["resume"].tolist()))]


def _exact_conv(s, c):
    y, state = s["y"], s["state_out"]
    for slot, resumes, first, n in _sequences(s):
        past = s["state_in"][slot] if resumes else torch.zeros_like(s["state_in"][slot])
        line = torch.cat([past, s["x"][first:first + n]])
        if n:
            v = s["b_conv"] + sum(s["w_conv"][q] * line[q:q + n] for q in range(D_CONV))
            y[first:first + n] = v * torch.sigmoid(v)
        state[slot] = line[n:]
    return {"y": y, "state": state}


def _exact_scan(s, c):
    """All sequences side by side, step by step."""
    y, state, A = s["y"], s["h_last"], s["A"]
    seqs = sorted(_sequences(s), key=lambda q: -q[3])
    h = torch.stack([s["h0"][q] if r else torch.zeros_like(s["h0"][q]) for q, r, _, _ in seqs])
    first = torch.tensor([f for _, _, f, _ in seqs], device="cuda")
    lens = [n for _, _, _, n in seqs]
    gate = s["z"] * torch.sigmoid(s["z"])
    live = len(lens)
    for t in range(lens[0] if lens else 0):
        while lens[live - 1] <= t:
            live -= 1
        r = first[:live] + t
        dl, u = s["delta"][r][:, :, None], s["u"][r][:, :, None]
        decay = torch.exp(dl * A)
        bu = s["Bm"][r][:, None, :] * u
        h[:live] = decay * h[:live] + (torch.expm1(dl * A) / A * bu if c["disc_mode"] == 0 else dl * bu)
        y[r] = (torch.einsum("bcn,bn->bc", h[:live], s["Cm"][r]) + s["D"] * u[:, :, 0]) * gate[r]
    for i, (slot, _, _, _) in enumerate(seqs):
        state[slot] = h[i]
    return {"y": y, "state": state}


def _exact_ffn(s, c):
    out = torch.zeros_like(s["x"])
    F = c["d_ff"]
    for e in range(c["E"]):
        for k in range(c["K"]):
            t = torch.nonzero(s["topk_idx"][:, k] == e)[:, 0]
            if len(t):
                g, v = s["x"][t] @ s["W_gu"][e, :F].t(), s["x"][t] @ s["W_gu"][e, F:].t()
                out[t] += s["gates"][t, k, None] * ((g * torch.sigmoid(g) * v) @ s["W_down"][e].t())
    return {"out": out}

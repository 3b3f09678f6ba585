"""Position rotation on the way into the KV cache, and differential attention over it: what is measured, and at what sizes.

  append  crop every agent to its kept prefix, append n tokens from the unrotated projections: K rotated by its positions on
          the way into the pages, V as it is, Q rotated beside them.  A bf16 cache's pools come back whole, of a cache in
          8 bits the values held from the first page that changed on
  rotate  the same rotation of one tensor alone (queries, or keys kept elsewhere), by positions on one axis or on several
          (time, height, width)
  diff    differential attention of every agent's last n positions: heads 2i and 2i + 1 of Q are the two maps of head i,
          kv-heads 2j and 2j + 1 hold their keys and, side by side, the value of width 2d that both maps weigh:
          O = softmax(q1 k1) V - lambda softmax(q2 k2) V, then (where the model has it) the norm of each head's 2d columns

With ``own`` false the operators are computed from elementary torch operations, angles in 64 bits, the rest in 32.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5  # of the heads' norm


def _append(name, B, L, hq, hkv, d, ps, T, n, bits=16, T_lo=None, rot=0, pairs="halves", sections="", pos0=-1, base=10000.0):
    return {"name": name, "op": "append", "B": B, "L": L, "hq": hq, "hkv": hkv, "d": d, "ps": ps, "T": T, "n": n, "bits": bits,
            "T_lo": T if T_lo is None else T_lo, "rot": rot or d, "pairs": pairs, "sections": sections, "pos0": pos0, "base": base}


def _rotate(name, B, L, hq, d, n, rot=0, pairs="halves", sections="", pos0=0, base=10000.0):
    return {"name": name, "op": "rotate", "B": B, "L": L, "hq": hq, "hkv": 1, "d": d, "ps": 16, "T": n, "n": n, "bits": 16, "T_lo": n,
            "rot": rot or d, "pairs": pairs, "sections": sections, "pos0": pos0, "base": base}


def _diff(name, B, hq, hkv, d, ps, T, n=1, T_lo=None, norm=True):
    return {"name": name, "op": "diff", "B": B, "hq": hq, "hkv": hkv, "d": d, "ps": ps, "T": T, "T_lo": T if T_lo is None else T_lo,
            "n": n, "norm": norm}


def listed():
    return [
        # one token of one small agent: latency
        _append("append_tiny", 1, 1, 8, 8, 64, 16, 640, 1),
        # a decode step's write: a token for each of 16 agents, all layers; evicted sessions, so positions far past the lengths
        _append("append_step", 16, 32, 32, 8, 128, 16, 700, 1, T_lo=101, pos0=120001),
        # a forget request's write: 1638 tokens of one agent, all layers of a 32-layer model
        _append("append_suffix", 1, 32, 32, 8, 128, 16, 2005, 1638, base=500000.0),
        # the same step into a cache in 8 bits
        _append("append_step_8", 16, 32, 32, 8, 128, 16, 700, 1, bits=8, T_lo=101),
        # ragged prompts into large pages in 8 bits: 64-wide heads, half of the columns rotated, neighbours paired
        _append("append_ragged_8", 8, 2, 8, 8, 64, 64, 1000, 333, bits=8, T_lo=401, rot=32, pairs="neighbours"),
        # one token's queries of 16 agents, three axes: latency
        _rotate("rotate_step", 16, 1, 32, 128, 1, sections="16,24,24", pos0=4001),
        # frames of video: queries of 4 agents x 1500 tokens, 8 layers, three axes
        _rotate("rotate_frames", 4, 8, 32, 128, 1500, sections="16,24,24", pos0=77, base=1000000.0),
        # one token of one small agent: latency
        _diff("diff_tiny", 1, 8, 8, 64, 16, 640),
        # a decode step of 16 agents with ordinary sessions
        _diff("diff_decode", 16, 32, 8, 128, 16, 8192, T_lo=2048),
        # one agent with a very long session, wide groups, large pages
        _diff("diff_long", 1, 64, 8, 128, 64, 120001),
        # a few re-read tokens of 8 agents on long prefixes
        _diff("diff_few", 8, 32, 8, 128, 16, 32784, n=16, norm=False),
        # a forget request's suffix: one layer of 1638 tokens on 16k
        _diff("diff_suffix", 1, 32, 8, 128, 16, 16384, n=1638),
    ]


HEADS = [(8, 8, 64), (32, 8, 128), (64, 8, 128), (16, 2, 128), (32, 8, 64), (8, 4, 64), (16, 4, 128)]


def draw(rng):
    """One more case: sizes spread over their logarithm, from a token to the listed cases' longest."""
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["append", "append", "rotate", "diff", "diff", "diff"])
    hq, hkv, d = rng.choice(HEADS)
    ps = rng.choice([8, 16, 16, 32, 64, 128])
    B = spread(1, 16)
    rot = rng.choice([d, d, d // 2, d // 4])
    pairs = rng.choice(["halves", "halves", "neighbours"])
    sections = ""
    if rng.random() < 0.4:
        t = rng.randint(1, rot // 2 - 2)
        h = rng.randint(1, rot // 2 - t - 1)
        sections = "%d,%d,%d" % (t, h, rot // 2 - t - h)
    pos0 = spread(1, 200000) if sections or rng.random() < 0.5 else -1
    base = rng.choice([10000.0, 500000.0, 1000000.0])
    if op == "append":
        L, n = spread(1, 32), spread(1, 2000)
        while L * B * n * hq * d > 2.1e8:
            L, B, n = max(1, L * 3 // 4), max(1, B - 1), max(1, n * 3 // 4)
        T = n + spread(1, 600) - 1
        T_lo = n + spread(1, T - n + 1) - 1
        c = _append("", B, L, hq, hkv, d, ps, T, n, rng.choice([16, 16, 8]), T_lo, rot, pairs, sections, pos0, base)
    elif op == "rotate":
        L, n = spread(1, 8), spread(1, 2000)
        while L * B * n * hq * d > 1.9e8:
            L, B, n = max(1, L * 3 // 4), max(1, B - 1), max(1, n * 3 // 4)
        c = _rotate("", B, L, hq, d, n, rot, pairs, sections, pos0, base)
    else:
        T = spread(17, 60000)
        n = rng.choice([1, 1, spread(1, 40), spread(1, 2000)])
        T = max(T, n)
        while B * hq * n * T > 8e8 or B * T * hkv * d > 2.5e8:
            B, T, n = max(1, B - 1), max(17, T * 3 // 4), max(1, n * 3 // 4)
        T = max(T, n)
        T_lo = min(T, max(n, spread(max(1, T // 4), T)))
        c = _diff("", B, hq, hkv, d, ps, T, n, T_lo, rng.random() < 0.7)
    del c["name"]
    return c


def _lens(c):
    """The agents' session lengths (the appended or attended positions included): T down to T_lo."""
    return [c["T"] - (c["T"] - c["T_lo"]) * i // max(1, c["B"] - 1) for i in range(c["B"])]


def _gen(seed, what):
    return torch.Generator("cuda").manual_seed(int(seed) * 16 + what)


def _randn(seed, what, shape):
    return torch.randn(shape, generator=_gen(seed, what), device="cuda")


def _valid(lens, T):
    return torch.arange(T, device="cuda")[None] < torch.tensor(lens, device="cuda")[:, None]


def _session(c, seed, what, L=1):
    """K or V (what = 1, 2) of every agent, bf16 [L][B][T][Hkv][d]: columns of unequal size, some tokens far larger."""
    g = _gen(seed, what)
    shape = (L, c["B"], c["T"], c["hkv"], c["d"])
    col = torch.exp(0.5 * torch.randn((L, 1, 1, c["hkv"], c["d"]), generator=g, device="cuda"))
    tok = 1 + 7 * (torch.rand((L, c["B"], c["T"], 1, 1), generator=g, device="cuda") < 0.01).float()
    x = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    for layer in range(L):
        x[layer] = torch.randn(shape[1:], generator=g, device="cuda") * col[layer] * tok[layer]
    return x


def _queries(c, seed):
    """Unrotated, or attended as they are: bf16 [L][B n][Hq][d] ([B n][Hq][d] for diff)."""
    lead = () if c["op"] == "diff" else (c["L"],)
    return _randn(seed, 3, lead + (c["B"] * c["n"], c["hq"], c["d"])).to(torch.bfloat16)


def _lambda(c, seed):
    """fp32 [Hq / 2]: learned, around the 0.2 to 0.8 that the layers start from."""
    return 0.5 + 0.15 * _randn(seed, 4, (c["hq"] // 2,))


def _gain(c, seed):
    """fp32 [2 d]: learned, with the factor 1 - lambda_init in it."""
    return 0.4 * (1 + 0.1 * _randn(seed, 5, (2 * c["d"],))) if c["norm"] else None


def _freq(c):
    """Radians per position of each pair, and the axis of each pair."""
    half = c["rot"] // 2
    sections = [int(x) for x in c["sections"].split(",")] if c["sections"] else [half]
    return [c["base"] ** (-i / half) for i in range(half)], [a for a, m in enumerate(sections) for _ in range(m)]


def _positions(c, seed):
    """int32 [axes][B n], or None for the positions that the tokens have in their sequences.  Several axes: a token's frame
    and its place in a 30 x 40 grid, after pos0 positions of text; one agent's text is longer than the next one's."""
    if c["pos0"] < 0:
        return None
    i = torch.arange(c["n"], device="cuda")[None]
    start = c["pos0"] + 97 * torch.arange(c["B"], device="cuda")[:, None] + int(torch.randint(0, 1000, (1,), generator=torch.Generator().manual_seed(int(seed))))
    axes = [i // 1200, i // 40 % 30, i % 40] if c["sections"] else [i]
    return torch.stack([(start + a).flatten() for a in axes]).int()


# ---------------------------------------------------------------- the plain form's arithmetic
def _rotated(c, x, pos):
    """x [L][N][H][d] -> fp32, pos int [axes][N]."""
    freq, axis = _freq(c)
    angle = pos.double()[axis].t() * torch.tensor(freq, dtype=torch.float64, device="cuda")
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    y = x.float()
    r = y[..., : c["rot"]]
    a, b = (r[..., 0::2], r[..., 1::2]) if c["pairs"] == "neighbours" else r.chunk(2, dim=-1)
    a, b = a * cos - b * sin, b * cos + a * sin
    r = torch.stack((a, b), dim=-1).flatten(-2) if c["pairs"] == "neighbours" else torch.cat((a, b), dim=-1)
    return torch.cat((r, y[..., c["rot"]:]), dim=-1)


def _pow2(e):
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _quantise(x, ps):
    """x fp32 [..][T][Hkv][d], T a multiple of ps -> the values pages of ps tokens hold: e4m3 codes times 2^e, e the least
    exponent with the page's largest magnitude at most 448 * 2^e."""
    pages = x.unflatten(-3, (x.shape[-3] // ps, ps))
    m, e = torch.frexp(pages.abs().amax(dim=(-3, -1), keepdim=True))
    e = torch.where(m == 0, torch.full_like(e, -126), torch.clamp(e - 9 + (m > 0.875).int(), min=-126))
    return ((pages * _pow2(-e)).to(torch.float8_e4m3fn).float() * _pow2(e)).flatten(-4, -3)


# ---------------------------------------------------------------- a case's state
def _order(c, seed):
    pages = sum(-(-t // c["ps"]) for t in _lens(c)) + 4
    return torch.randperm(pages, generator=torch.Generator().manual_seed(int(seed))).tolist()


def _cu(counts):
    cu = [0]
    for n in counts:
        cu.append(cu[-1] + n)
    return cu


def prepare(case, seed):
    c, lens = case, _lens(case)
    B, n, ps = c["B"], c["n"], c["ps"]
    s = {"case": c, "lens": lens, "t": torch.tensor(lens, device="cuda"), "Q": _queries(c, seed)}
    L = c["L"] if c["op"] == "append" else 1
    s["pos"] = None if c["op"] == "diff" else _positions(c, seed)
    valid = _valid(lens, c["T"])
    if c["op"] == "diff":
        s["lam"], s["gain"] = _lambda(c, seed), _gain(c, seed)
    if c["op"] != "rotate":
        K, V = _session(c, seed, 1, L), _session(c, seed, 2, L)
    else:
        K = V = torch.zeros((1, B, c["T"], 1, c["d"]), dtype=torch.bfloat16, device="cuda")
    if c["op"] == "append":  # the tokens to append, packed; the cache holds K of the kept prefixes as it is
        new = valid & (torch.arange(c["T"], device="cuda")[None] >= s["t"][:, None] - n)
        s["K"], s["V"] = K[:, new].contiguous(), V[:, new].contiguous()
    order = _order(c, seed)
    pools = None
    if c["op"] == "append" and c["bits"] == 16:
        pools = [torch.zeros((L, len(order), c["hkv"], ps, c["d"]), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        s["pools"] = pools
    if own:
        from paper_2609_04875_gb300 import PagedKVCache, Rope
        cache = PagedKVCache(L, c["hkv"], c["d"], ps, len(order), B, -(-c["T"] // ps), init_free_order=order,
                             **({"kv_bits": c.get("bits", 16)} if pools is None else {"k_pool": pools[0], "v_pool": pools[1]}))
        seqs = [cache.seq_create() for _ in range(B)]
        cache.append_kv_batch(seqs, K[:, valid].contiguous(), V[:, valid].contiguous(), _cu(lens))
        s |= {"cache": cache, "seqs": seqs}
        if c["op"] != "diff":
            freq, axis = _freq(c)
            s["rope"] = Rope(freq, axis=axis, interleaved=c["pairs"] == "neighbours")
        torch.cuda.synchronize()
        return s
    if s["pos"] is None and c["op"] != "diff":
        s["pos"] = ((s["t"] - n)[:, None] + torch.arange(n, device="cuda")[None]).flatten()[None].int()
    if c["op"] == "diff":
        s["k"], s["v"] = K[0], V[0]
    elif pools is not None:
        # every agent's pages in the order they are taken, and where its new tokens lie
        page = torch.tensor(order, device="cuda")
        first = torch.tensor(_cu([-(-t // ps) for t in lens])[:-1], device="cuda")
        at = torch.arange(c["T"], device="cuda")[None].expand(B, -1)
        where = page[(first[:, None] + at // ps).clamp(max=len(order) - 1)]
        for pool, x in ((pools[0], K), (pools[1], V)):
            for layer in range(L):
                pool[layer].permute(0, 2, 1, 3)[where[valid], (at % ps)[valid]] = x[layer][valid]
        s["page"], s["slot"] = where[new], (at % ps)[new]
    elif c["op"] == "append":
        # the kept tokens' values on the first page that changes, [L][B][ps][Hkv][d] fp32
        base = (s["t"] - n) // ps * ps
        at = base[:, None] + torch.arange(ps, device="cuda")[None]
        s["kept"] = at < s["t"][:, None] - n
        rows = torch.arange(B, device="cuda")[:, None]
        wide = -c["T"] % ps
        held = [_quantise(torch.nn.functional.pad(x.float() * valid[:, :, None, None], (0, 0, 0, 0, 0, wide)), ps) for x in (K, V)]
        s["old"] = [x[:, rows, at.clamp(max=x.shape[2] - 1)] for x in held]
    return s


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    c, cache, seqs, lens = s["case"], s["cache"], s["seqs"], s["lens"]
    n = c["n"]
    cu = [n * i for i in range(c["B"] + 1)]
    if c["op"] == "diff":
        return {"out": cache.diff_attn_batch(seqs, 0, s["Q"], cu, s["lam"], gain=s["gain"], eps=EPS)}
    if c["op"] == "rotate":
        return {"out": cache.rotate_batch(seqs, s["Q"], cu, s["rope"], positions=s["pos"])}
    # (the last agent first: its pages go back first, so that every pass finds each agent's pages where they were)
    cache.crop_batch(seqs[::-1], [t - n + 1 for t in lens[::-1]])
    q = cache.append_kv_rope_batch(seqs, s["K"], s["V"], cu, s["rope"], Q=s["Q"], positions=s["pos"])
    if c["bits"] == 16:
        return {"K": s["pools"][0], "V": s["pools"][1], "Q": q}
    begin = [(t - n) // c["ps"] * c["ps"] for t in lens]
    k, v = cache.read_kv_batch(seqs, begin, _cu([t - b for t, b in zip(lens, begin)]))
    return {"K": k, "V": v, "Q": q}


def _run_plain(s):
    c, t, B, n, d = s["case"], s["t"], s["case"]["B"], s["case"]["n"], s["case"]["d"]
    if c["op"] == "rotate":
        return {"out": _rotated(c, s["Q"], s["pos"]).to(torch.bfloat16)}
    if c["op"] == "append":
        k, q = _rotated(c, s["K"], s["pos"]), _rotated(c, s["Q"], s["pos"]).to(torch.bfloat16)
        if c["bits"] == 16:
            for pool, x in ((s["pools"][0], k.to(torch.bfloat16)), (s["pools"][1], s["V"])):
                pool.permute(1, 3, 0, 2, 4)[s["page"], s["slot"]] = x.transpose(0, 1)
            return {"K": s["pools"][0], "V": s["pools"][1], "Q": q}
        ps = c["ps"]
        off = (t - n) % ps  # of the first new token on the first page that changes
        width = -(-(ps - 1 + n) // ps) * ps
        rows = torch.arange(B, device="cuda")[:, None]
        place = off[:, None] + torch.arange(n, device="cuda")[None]
        held = torch.arange(width, device="cuda")[None] < (off + n)[:, None]
        out = {"Q": q}
        for name, new, old in (("K", k, s["old"][0]), ("V", s["V"].float(), s["old"][1])):
            x = torch.zeros((c["L"], B, width, c["hkv"], d), device="cuda")
            x[:, :, :ps] = old * s["kept"][:, :, None, None]
            x[:, rows, place] = new.view(c["L"], B, n, c["hkv"], d)
            out[name] = _quantise(x, ps)[:, held].to(torch.bfloat16)
        return out
    hq, hkv, T = c["hq"], c["hkv"], c["T"]
    g = hq // hkv
    # [B][pair][map][head of the pair, query][d], and the pairs' values side by side
    q = s["Q"].float().view(B, n, hkv // 2, g, 2, d).permute(0, 2, 4, 3, 1, 5).reshape(B, hkv // 2, 2, g * n, d)
    k = s["k"].float().view(B, T, hkv // 2, 2, d).permute(0, 2, 3, 4, 1)
    v = s["v"].float().view(B, T, hkv // 2, 1, 2 * d).permute(0, 2, 3, 1, 4)
    x = (q @ k).mul_(1.0 / math.sqrt(d))
    last = t[:, None] - n + torch.arange(n, device="cuda")[None]
    seen = torch.arange(T, device="cuda")[None, None] <= last[:, :, None]
    x = x.view(B, hkv // 2, 2, g, n, T).masked_fill_(~seen[:, None, None, None], -math.inf)
    x = x.sub_(x.amax(dim=-1, keepdim=True)).exp_()
    x = x.div_(x.sum(dim=-1, keepdim=True)).view(B, hkv // 2, 2, g * n, T)
    o = x @ v
    o = o.view(B, hkv // 2, 2, g, n, 2 * d)
    o = o[:, :, 0] - s["lam"].view(hkv // 2, g, 1, 1) * o[:, :, 1]
    if s["gain"] is not None:
        o = o * (1.0 / ((o * o).mean(dim=-1, keepdim=True) + EPS).sqrt()) * s["gain"]
    return {"out": o.permute(0, 3, 1, 2, 4).reshape(B * n, hq // 2, 2 * d).to(torch.bfloat16)}


def work(case):
    c, lens = case, _lens(case)
    if c["op"] == "diff":
        pairs = sum(c["n"] * t - c["n"] * (c["n"] - 1) // 2 for t in lens)
        return {"bytes": 4.0 * sum(lens) * c["hkv"] * c["d"] + 4.0 * c["B"] * c["n"] * c["hq"] * c["d"], "flops": 6.0 * pairs * c["hq"] * c["d"]}
    q = c["L"] * c["B"] * c["n"] * c["hq"] * c["d"] * 2
    flops = 3.0 * q / 2 * c["rot"] / c["d"]
    if c["op"] == "rotate":
        return {"bytes": 2.0 * q, "flops": flops}
    new = c["L"] * c["B"] * c["n"] * c["hkv"] * c["d"] * 2
    flops *= (c["hq"] + c["hkv"]) / c["hq"]
    if c["bits"] == 16:
        return {"bytes": 2.0 * q + 4.0 * new, "flops": flops}
    back = c["L"] * sum(c["n"] + (t - c["n"]) % c["ps"] for t in lens) * c["hkv"] * c["d"] * 2
    return {"bytes": 2.0 * q + 2.0 * new + new + back + 2.0 * back, "flops": flops + 4.0 * new}


# ---------------------------------------------------------------- 64 bits, from the definition
def _turned(c, x, pos):
    """x fp64 [..][N][H][d]; pos int [axes][N]: each pair of columns as a complex number, times e^(i angle)."""
    freq, axis = _freq(c)
    half = c["rot"] // 2
    one, two = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if c["pairs"] == "neighbours" else (slice(0, half), slice(half, 2 * half))
    turn = torch.stack([torch.polar(torch.ones_like(p), p) for p in (pos[a].double() * f for a, f in zip(axis, freq))], dim=-1)
    z = torch.complex(x[..., one], x[..., two]) * turn[:, None]
    y = x.clone()
    y[..., one], y[..., two] = z.real, z.imag
    return y


def _two(e):
    """2^e, exactly."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _page_values(x, ps):
    """The values pages of ps tokens hold for x, fp64 [T][Hkv][d]: steps of 2^(exponent - 3) of a value over the page's scale,
    at least 2^-9, ties to even."""
    T = x.shape[0]
    pages = torch.cat([x, x.new_zeros((-T % ps,) + x.shape[1:])]).view(-1, ps, *x.shape[1:])
    a = pages.abs().amax(dim=(1, 3))[:, None, :, None]
    e = torch.where(a == 0, torch.zeros_like(a), torch.ceil(torch.log2(a / 448)))
    e = torch.where(a > 448 * _two(e), e + 1, torch.where(a <= 448 * _two(e - 1), e - 1, e))
    scale = _two(torch.clamp(e, min=-126))
    y = pages / scale
    step = _two(torch.clamp(torch.frexp(y)[1] - 4, min=-9))
    return (torch.round(y / step) * step * scale).view(-1, *x.shape[1:])[:T]


def exact(case, seed):
    c, lens = case, _lens(case)
    B, n, ps, d = c["B"], c["n"], c["ps"], c["d"]
    Q = _queries(c, seed)
    if c["op"] == "diff":
        K, V = _session(c, seed, 1)[0], _session(c, seed, 2)[0]
        lam, gain, g = _lambda(c, seed).double(), _gain(c, seed), c["hq"] // c["hkv"]
        out = torch.empty((B * n, c["hq"] // 2, 2 * d), dtype=torch.float64, device="cuda")
        for b, t in enumerate(lens):
            past = torch.arange(t, device="cuda")[None] > torch.arange(t - n, t, device="cuda")[:, None]
            rows = slice(b * n, (b + 1) * n)
            for h in range(c["hq"] // 2):
                j = h // g
                v = torch.cat([V[b, :t, 2 * j], V[b, :t, 2 * j + 1]], dim=1).double()
                maps = [torch.softmax((Q[rows, 2 * h + m].double() @ K[b, :t, 2 * j + m].double().t() / math.sqrt(d)).masked_fill(past, -math.inf), dim=1)
                        for m in range(2)]
                out[rows, h] = (maps[0] - lam[h] * maps[1]) @ v
        if gain is not None:
            out = out / torch.sqrt(out.square().sum(dim=-1, keepdim=True) / (2 * d) + EPS) * gain.double()
        return {"out": out}
    pos = _positions(c, seed)
    if pos is None:
        pos = torch.tensor([t - n + i for t in lens for i in range(n)], device="cuda")[None]
    q = torch.stack([_turned(c, x.double(), pos) for x in Q])
    if c["op"] == "rotate":
        return {"out": q}
    K, V = _session(c, seed, 1, c["L"]), _session(c, seed, 2, c["L"])
    new = [torch.cat([x[:, b, t - n: t] for b, t in enumerate(lens)], dim=1) for x in (K, V)]
    if c["bits"] == 8:
        found = {"K": [], "V": [], "Q": q}
        for name, x, y in (("K", K, torch.stack([_turned(c, z.double(), pos) for z in new[0]])), ("V", V, new[1].double())):
            for layer in range(c["L"]):
                for b, t in enumerate(lens):
                    p0 = (t - n) // ps * ps
                    # the kept tokens stood on a full page before the crop; the page is quantised again with the new ones
                    old = _page_values(x[layer, b, p0: min(t, p0 + ps)].double(), ps)[: t - n - p0]
                    found[name].append(_page_values(torch.cat([old, y[layer, b * n: (b + 1) * n]]), ps))
            found[name] = torch.cat(found[name]).view(c["L"], -1, c["hkv"], d)
        return found
    # the pools, page by page
    order = _order(c, seed)
    pools = [torch.zeros((c["L"], len(order), c["hkv"], ps, d), dtype=torch.float64, device="cuda") for _ in range(2)]
    for layer in range(c["L"]):
        turned = _turned(c, new[0][layer].double(), pos)
        taken = iter(order)
        for b, t in enumerate(lens):
            pages = torch.tensor([next(taken) for _ in range(-(-t // ps))], device="cuda")
            for pool, x, y in ((pools[0], K, turned), (pools[1], V, new[1][layer].double())):
                z = torch.zeros((len(pages) * ps, c["hkv"], d), dtype=torch.float64, device="cuda")
                z[: t - n] = x[layer, b, : t - n].double()
                z[t - n: t] = y[b * n: (b + 1) * n]
                pool[layer, pages] = z.view(-1, ps, c["hkv"], d).transpose(1, 2)
    return {"K": pools[0], "V": pools[1], "Q": q}

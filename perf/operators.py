"""The measured work of the operators that serve a model after its prefill, through the library's public entry points:

  rotary   tsa_rotary: rotary positions on Q and K
  write    tsa_cache_write: new rows of K and V into a paged cache, bf16 or 8 bits with a power-of-two scale per row
  read     tsa_cache_read: sequences of that cache back as contiguous bf16 tensors
  attend   tsa_attend_cache: attention of the new tokens of a ragged batch over the cache

Every operator has a plain form here too (`own` false): elementary torch operations in 32 bits, angles in 64."""
from __future__ import annotations

import itertools
import math
import random

import torch

own = False

E4M3_MAX = 448.0


def listed():
    return [
        # the next token of 61 sequences, some of them far into a long context: half of the head rotated, pairs side by side
        dict(kind="rotary", name="rotary_step", B=1, L=61, Hq=32, Hkv=8, d=64, rot=32, interleaved=1, scaling="parts", factor=8.0, original=32768,
             base=10000.0, far=1, fused=1),
        # a long prompt, out of the rows that a fused projection leaves into one tensor per head, stretched context
        dict(kind="rotary", name="rotary_prompt", B=1, L=32768, Hq=32, Hkv=8, d=128, rot=128, interleaved=0, scaling="wavelength", factor=8.0,
             original=8192, base=500000.0, far=0, fused=1),
        # the next token of 61 sequences into 8 bits
        dict(kind="write", name="write_step_e4m3", n=61, new=1, kv=9000, mix=0, Hkv=8, d=128, page=16, e4m3=1, lens=1),
        # prompts of different lengths into 8 bits
        dict(kind="write", name="write_prompts_e4m3", n=7, new=12000, kv=12000, mix=0, Hkv=8, d=128, page=64, e4m3=1, lens=2),
        # a few short sequences back, to score against them
        dict(kind="read", name="read_batch_bf16", n=7, kv=2500, Hkv=4, d=64, page=32, e4m3=0, lens=3),
        # a long context back into bf16
        dict(kind="read", name="read_64k_e4m3", n=1, kv=65536, Hkv=8, d=128, page=64, e4m3=1, lens=4),
        # one user, one token, a short context: the smallest call
        _attend(name="decode_one", n=1, new=1, kv=701, page=16, lens=5),
        # a serving batch of ragged contexts
        _attend(name="decode_ragged", n=48, new=1, kv=16384, page=16, lens=6),
        # few users with very long contexts in 8 bits
        _attend(name="decode_long_e4m3", n=4, new=1, kv=131072, page=64, e4m3=1, lens=7),
        # drafted tokens checked at once on a model with a sliding window and seven query heads per KV head, old pages dropped
        _attend(name="verify_window_e4m3", n=9, new=5, kv=32768, Hq=28, Hkv=4, page=16, e4m3=1, window=4096, lens=8),
        # one piece of a long prompt
        _attend(name="chunk_2k", n=1, new=2048, kv=32768, page=64, lens=9),
        # two prompts that arrive while six sequences decode
        _attend(name="mixed", n=8, new=1500, kv=6000, page=32, mix=6, lens=10),
    ]


def _attend(**kw):
    return dict(dict(kind="attend", Hq=32, Hkv=8, d=128, e4m3=0, window=0, mix=0, pad=0), **kw)


_HEADS = [(4, 4), (8, 8), (12, 4), (16, 2), (28, 4), (32, 8), (32, 8), (32, 32), (40, 8)]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    big = {k: max(_cost(c) for c in listed() if c["kind"] == k) for k in ("rotary", "write", "read", "attend")}
    while True:
        kind = rng.choice(["rotary", "rotary", "write", "write", "read", "attend", "attend", "attend", "attend"])
        Hq, Hkv = rng.choice(_HEADS)
        d = rng.choice([64, 128, 128])
        if kind == "rotary":
            c = dict(kind=kind, B=rng.choice([1, 1, 2, 3]), L=_log(rng, 1, 32768), Hq=Hq, Hkv=Hkv, d=d, rot=rng.choice([d, d, d // 2, d // 4]),
                     interleaved=rng.choice([0, 0, 1]), scaling=rng.choice(["none", "linear", "base", "parts", "wavelength"]),
                     factor=rng.choice([2.0, 4.0, 8.0]), original=rng.choice([4096, 8192, 32768]), base=rng.choice([10000.0, 500000.0]),
                     far=rng.choice([0, 0, 1]), fused=rng.choice([0, 1]))
        elif kind == "read":
            c = dict(kind=kind, n=_log(rng, 1, 16), kv=_log(rng, 1, 65536), Hkv=Hkv, d=d, page=rng.choice([16, 16, 32, 64, 128, 256]),
                     e4m3=rng.choice([0, 1]), lens=rng.randrange(1 << 30))
        else:
            new = rng.choice([1, 1, rng.randrange(2, 9), _log(rng, 9, 8192)])
            n = _log(rng, 1, 64) if new < 9 else _log(rng, 1, 8)
            c = dict(kind=kind, n=n, new=new, kv=max(new, _log(rng, 16, 131072)), mix=rng.randrange(n) if new > 8 else 0, Hkv=Hkv, d=d,
                     page=rng.choice([16, 16, 32, 64, 128, 256]), e4m3=rng.choice([0, 1]), lens=rng.randrange(1 << 30))
            if kind == "attend":
                c.update(Hq=Hq, window=rng.choice([0, 0, 0, 128, 1000, 4096]), pad=rng.choice([0, 0, 3]))
        if kind in ("read", "attend") and c["n"] * c["kv"] * c["Hkv"] * c["d"] > 4 * 131072 * 8 * 128:
            continue
        # (the plain form of attend lays out n x max new x heads x max kv scores)
        if kind == "attend" and c["n"] * c["new"] * c["Hq"] * c["kv"] > 2.2e9:
            continue
        if kind == "write" and c["n"] * c["kv"] * c["Hkv"] * c["d"] > 2 * 131072 * 8 * 128:
            continue
        if _cost(c) <= big[kind]:
            return c


def _cost(case):
    w = work(case)
    return w["flops"] / 1.0e15 + w["bytes"] / 4.0e12


# ---- shapes of a case

def _lens(c):
    """New tokens and cached tokens (the new ones among them) of every sequence.  The last `mix` sequences add one token; the longest
    context is exactly `kv` long, and one sequence adds exactly `new`."""
    r = random.Random(c["lens"])
    n, most = c["n"], c.get("new", 1)
    kv = [c["kv"]] + [_log(r, max(1, c["kv"] // 40), c["kv"]) for _ in range(n - 1)]
    new = [most] + [r.randrange(max(1, most // 3), most + 1) for _ in range(n - 1)]
    new = [min(1 if i >= n - c.get("mix", 0) else x, kv[i]) for i, x in enumerate(new)]
    if c["kind"] == "write" and c["new"] == c["kv"]:        # whole prompts
        new = kv
    both = list(zip(new, kv))
    r.shuffle(both)
    return [x for x, _ in both], [x for _, x in both]


def _seen(new, kv, window):
    """Pairs of a query and a key that it sees, and keys that any query sees, of one sequence."""
    if not window:
        return new * (kv - new) + new * (new + 1) // 2, kv
    pairs = sum(min(p + 1, window) for p in range(kv - new, kv)) if new < 4096 or kv - new < window else new * window
    return pairs, min(kv, new + window - 1)


def work(case):
    c = case
    if c["kind"] == "rotary":
        rows = c["B"] * c["L"] * (c["Hq"] + c["Hkv"])
        return {"bytes": 4 * rows * c["d"], "flops": 3 * rows * c["rot"]}
    new, kv = _lens(c)
    row = c["Hkv"] * (c["d"] + 1 if c["e4m3"] else 2 * c["d"])       # one token's K (or V) in the cache
    if c["kind"] == "write":
        return {"bytes": 2 * sum(new) * (row + 2 * c["Hkv"] * c["d"]), "flops": 4 * sum(new) * c["Hkv"] * c["d"]}
    if c["kind"] == "read":
        return {"bytes": 2 * sum(kv) * row + 4 * c["n"] * c["kv"] * c["Hkv"] * c["d"], "flops": 2 * sum(kv) * c["Hkv"] * c["d"]}
    seen = [_seen(a, b, c["window"]) for a, b in zip(new, kv)]
    return {"bytes": 2 * row * sum(k for _, k in seen) + sum(new) * c["Hq"] * (4 * c["d"] + 4), "flops": 4 * c["d"] * c["Hq"] * sum(p for p, _ in seen)}


# ---- what a program has in hand

def _frequencies(c):
    """Radians per position of every pair, and the factor on the rotated columns, in plain Python."""
    rot, base, f, orig = c["rot"], c["base"], c["factor"], c["original"]
    if c["scaling"] == "base":
        base = base * f ** (rot / (rot - 2.0))
    freq = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    gain = 1.0
    if c["scaling"] == "linear":
        freq = [x / f for x in freq]
    elif c["scaling"] == "parts":
        # pairs that turn more than 32 times within the original length stay, those below one turn are stretched, a ramp between
        at = lambda turns: rot * math.log(orig / (turns * 2 * math.pi)) / (2 * math.log(base))
        lo, hi = max(0, math.floor(at(32.0))), min(rot - 1, math.ceil(at(1.0)))
        ramp = [min(1.0, max(0.0, (i - lo) / (hi - lo if hi > lo else 0.001))) for i in range(rot // 2)]
        freq = [x * (1 - t) + x / f * t for x, t in zip(freq, ramp)]
        gain = 0.1 * math.log(f) + 1.0
    elif c["scaling"] == "wavelength":
        # pairs with more than 4 turns in the original length stay, below one turn they are stretched, linear in the turns between
        turns = [orig * x / (2 * math.pi) for x in freq]
        mix = [min(1.0, max(0.0, (t - 1.0) / (4.0 - 1.0))) for t in turns]
        freq = [x * m + x / f * (1 - m) for x, m in zip(freq, mix)]
    return freq, gain


def _pow2(e):
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _quantise(x):
    """Rows of x as e4m3 values and E8M0 bytes: the smallest power of two with which the row's largest magnitude fits."""
    amax = x.float().abs().amax(-1)
    m, e = torch.frexp(amax)
    e = torch.where(m > 0.875, e - 8, e - 9).clamp(-126, 127)
    e = torch.where(amax > 0, e, torch.zeros_like(e))
    q = (x.float() * _pow2(-e)[..., None]).to(torch.float8_e4m3fn)
    return q, (e + 127).to(torch.uint8)


def _values(pages, scales):
    x = pages.float()
    return x if scales is None else x * _pow2(scales.to(torch.int32) - 127)[..., None]


def _rows(g, *shape):
    """N(0,1) rows whose columns differ in size, as keys and values of a model do."""
    gain = torch.exp(0.5 * torch.randn(shape[-1], generator=g, device="cuda"))
    return (torch.randn(*shape, generator=g, device="cuda") * gain).bfloat16()


def _inputs(c, seed):
    """Tensors of a case, on the GPU."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    s = dict(case=c)
    if c["kind"] == "rotary":
        B, L, Hq, Hkv, d = c["B"], c["L"], c["Hq"], c["Hkv"], c["d"]
        if c["fused"]:
            s["qkv"] = _rows(g, B, L, (Hq + 2 * Hkv) * d)
            s["Q"] = s["qkv"][..., :Hq * d].unflatten(-1, (Hq, d)).transpose(1, 2)               # [B,H,L,d] views of the rows
            s["K"] = s["qkv"][..., Hq * d:(Hq + Hkv) * d].unflatten(-1, (Hkv, d)).transpose(1, 2)
        else:
            s["Q"], s["K"] = _rows(g, B, Hq, L, d), _rows(g, B, Hkv, L, d)
        top = 1 << 20 if c["far"] else 4096
        s["positions"] = torch.randint(0, top, (B, L), generator=g, device="cuda", dtype=torch.int32) if c["far"] else \
            (torch.randint(0, top, (B, 1), generator=g, device="cuda", dtype=torch.int32) + torch.arange(L, device="cuda", dtype=torch.int32))
        return s
    n, Hkv, d, page = c["n"], c["Hkv"], c["d"], c["page"]
    new, kv = _lens(c)
    per = -(-c["kv"] // page)
    need = [-(-k // page) for k in kv]
    # a pool in use: the pages of a sequence anywhere in it, -1 behind the last one and where no query looks any more
    order = torch.randperm(sum(need) + 3, generator=g, device="cuda").to(torch.int32)
    first = ints([0] + list(itertools.accumulate(need)))[:n, None]
    gone = ints([max(0, (k - q + 1 - c["window"]) // page) if c.get("window") else 0 for q, k in zip(new, kv)])
    p = torch.arange(per, device="cuda", dtype=torch.int32)
    table = torch.where((p >= gone[:, None]) & (p < ints(need)[:, None]), order[(first + p).clamp(max=sum(need)).long()], -1).to(torch.int32)
    s.update(table=table, kv_len=ints(kv), n_pages=sum(need) + 3)
    if c["kind"] != "read":
        s.update(cu_q=ints([0] + list(itertools.accumulate(new))), n_tokens=sum(new) + c.get("pad", 0), max_q=max(new))
    pools = (s["n_pages"], Hkv, page, d)
    if c["kind"] == "write":
        s["K"], s["V"] = _rows(g, s["n_tokens"], Hkv, d), _rows(g, s["n_tokens"], Hkv, d)
        s["kp"], s["vp"] = (torch.zeros(pools, dtype=torch.float8_e4m3fn if c["e4m3"] else torch.bfloat16, device="cuda") for _ in "kv")
        s["ks"], s["vs"] = (torch.zeros(pools[:3], dtype=torch.uint8, device="cuda") if c["e4m3"] else None for _ in "kv")
        return s
    s["kp"], s["vp"], s["ks"], s["vs"] = _rows(g, *pools), _rows(g, *pools), None, None
    if c["e4m3"]:
        s["kp"], s["ks"] = _quantise(s["kp"])
        s["vp"], s["vs"] = _quantise(s["vp"])
    if c["kind"] == "attend":
        s["Q"] = _rows(g, s["n_tokens"], c["Hq"], d)
        s["O"] = torch.zeros(s["n_tokens"], c["Hq"], d, dtype=torch.bfloat16, device="cuda")
        s["lse"] = torch.zeros(s["n_tokens"], c["Hq"], device="cuda")
    return s


def prepare(case, seed):
    s, c = _inputs(case, seed), case
    if c["kind"] == "rotary":
        s["freq"], s["gain"] = _frequencies(c)
        s["Qo"], s["Ko"] = (torch.empty(x.shape, dtype=x.dtype, device="cuda") for x in (s["Q"], s["K"]))
    if c["kind"] == "read":
        s["K"], s["V"] = (torch.empty(c["n"], c["Hkv"], c["kv"], c["d"], dtype=torch.bfloat16, device="cuda") for _ in "kv")
    if own:
        from paper_2602_03216_amd import binding as tsa
        if c["kind"] == "rotary":
            s["desc"] = tsa.make_rotary_desc(c["B"], c["Hq"], c["Hkv"], c["L"], c["d"], s["freq"], interleaved=c["interleaved"], gain=s["gain"],
                                             q_strides=s["Q"].stride()[:3], k_strides=s["K"].stride()[:3])
        else:
            s["desc"] = tsa.make_cache_desc(c["n"], s.get("n_tokens", 0), c.get("Hq", c["Hkv"]), c["Hkv"], c["d"], c["page"], s["n_pages"],
                                            s["table"].shape[1], tsa.TSA_CACHE_E4M3 if c["e4m3"] else tsa.TSA_CACHE_BF16,
                                            max_q=s.get("max_q", 0), window=c.get("window", 0))
        if c["kind"] == "attend":
            s["ws"] = tsa.alloc_attend_cache_workspace(s["desc"])
    return s


# ---- one pass

def run(s):
    kind = s["case"]["kind"]
    if own:
        from paper_2602_03216_amd import binding as tsa
        if kind == "rotary":
            tsa.tsa_rotary(s["desc"], s["Q"], s["K"], s["Qo"], s["Ko"], positions=s["positions"])
            return s["Qo"], s["Ko"]
        if kind == "write":
            tsa.tsa_cache_write(s["desc"], s["K"], s["V"], s["cu_q"], s["kv_len"], s["table"], s["kp"], s["vp"], s["ks"], s["vs"])
            return s["kp"], s["vp"], s["ks"], s["vs"]
        if kind == "read":
            tsa.tsa_cache_read(s["desc"], s["kp"], s["vp"], s["kv_len"], s["table"], s["case"]["kv"], s["K"], s["V"], s["ks"], s["vs"])
            return s["K"], s["V"]
        tsa.tsa_attend_cache(s["desc"], s["Q"], s["kp"], s["vp"], s["cu_q"], s["kv_len"], s["table"], s["O"], s["ws"], lse=s["lse"],
                             k_scales=s["ks"], v_scales=s["vs"])
        return s["O"], s["lse"]
    return {"rotary": _plain_rotary, "write": _plain_write, "read": _plain_read, "attend": _plain_attend}[kind](s)


def _plain_rotary(s):
    c = s["case"]
    rot, half = c["rot"], c["rot"] // 2
    angle = s["positions"].double()[:, None, :, None] * torch.tensor(s["freq"], dtype=torch.float64, device="cuda")
    cos, sin = (torch.cos(angle) * s["gain"]).float(), (torch.sin(angle) * s["gain"]).float()

    def turn(x, out):
        out[..., rot:] = x[..., rot:]
        a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if c["interleaved"] else (x[..., :half], x[..., half:rot])
        a, b = a.float(), b.float()
        u, v = (a * cos - b * sin).to(out.dtype), (a * sin + b * cos).to(out.dtype)
        if c["interleaved"]:
            out[..., 0:rot:2], out[..., 1:rot:2] = u, v
        else:
            out[..., :half], out[..., half:rot] = u, v
        return out

    return turn(s["Q"], s["Qo"]), turn(s["K"], s["Ko"])


def _plain_write(s):
    page, cu = s["case"]["page"], s["cu_q"].long()
    t = torch.arange(s["n_tokens"], device="cuda")
    seq = torch.searchsorted(cu[1:], t, right=True)
    pos = s["kv_len"].long()[seq] - (cu[seq + 1] - t)
    p, o = s["table"].long()[seq, pos // page], pos % page

    def put(x, pages, scales):
        if scales is None:
            pages[p, :, o] = x
        else:
            q, e = _quantise(x)
            pages.view(torch.uint8)[p, :, o] = q.view(torch.uint8)
            scales[p, :, o] = e

    put(s["K"], s["kp"], s["ks"])
    put(s["V"], s["vp"], s["vs"])
    return s["kp"], s["vp"], s["ks"], s["vs"]


def _rows_of(s, pages, scales):
    """[n, Hkv, kv, d] in 32 bits: the rows of every sequence in order."""
    c = s["case"]
    at = s["table"].clamp(min=0).long()
    x = _values(pages.view(torch.uint8)[at].view(pages.dtype) if scales is not None else pages[at], None if scales is None else scales[at])
    return x.transpose(1, 2).flatten(2, 3)[:, :, :c["kv"]]


def _plain_read(s):
    c = s["case"]
    there = (torch.arange(c["kv"], device="cuda") < s["kv_len"][:, None])[:, None, :, None]
    for_ = lambda pages, scales, out: out.copy_(torch.where(there, _rows_of(s, pages, scales), 0.0))
    return for_(s["kp"], s["ks"], s["K"]), for_(s["vp"], s["vs"], s["V"])


def _plain_attend(s):
    c = s["case"]
    n, Hq, Hkv, d, mq, Lk = c["n"], c["Hq"], c["Hkv"], c["d"], s["max_q"], c["kv"]
    cu, kv = s["cu_q"].long(), s["kv_len"].long()
    q_len = cu[1:] - cu[:-1]
    K, V = _rows_of(s, s["kp"], s["ks"]), _rows_of(s, s["vp"], s["vs"])
    tok = (cu[:-1, None] + torch.arange(mq, device="cuda")).clamp(max=s["n_tokens"] - 1)                      # [n, mq]
    Q = s["Q"][tok].float().view(n, mq, Hkv, Hq // Hkv, d).permute(0, 2, 1, 3, 4).reshape(n, Hkv, -1, d)
    x = torch.matmul(Q, K.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(d)).view(n, Hkv, mq, Hq // Hkv, Lk)
    p = (kv - q_len)[:, None] + torch.arange(mq, device="cuda")                                              # position of a query
    key = torch.arange(Lk, device="cuda")
    hidden = key > p[..., None]
    if c["window"]:
        hidden |= key <= p[..., None] - c["window"]
    x.masked_fill_(hidden[:, None, :, None, :], float("-inf"))
    m = x.amax(-1, keepdim=True)
    x.sub_(m).exp_()
    l = x.sum(-1, keepdim=True)
    O = torch.matmul(x.view(n, Hkv, -1, Lk), V).view(n, Hkv, mq, Hq // Hkv, d) / l
    lse = (m + torch.log(l)).squeeze(-1)
    t = torch.arange(s["n_tokens"], device="cuda")
    seq = torch.searchsorted(cu[1:].contiguous(), t, right=True)
    there = seq < n
    seq = seq.clamp(max=n - 1)
    j = (t - cu[seq]).clamp(max=mq - 1)
    s["O"].copy_(torch.where(there[:, None, None], O[seq, :, j].reshape(-1, Hq, d).to(s["O"].dtype), s["O"]))
    s["lse"].copy_(torch.where(there[:, None], lse[seq, :, j].reshape(-1, Hq), s["lse"]))
    return s["O"], s["lse"]


# ---- the definitions in 64 bits

def exact(case, seed):
    c, s = case, _inputs(case, seed)
    two_to = lambda e: ((e.to(torch.int64) + 1023) << 52).view(torch.float64)              # (a library's power may be a bit off)
    if c["kind"] == "rotary":
        freq, gain = _frequencies(c)
        a = s["positions"].double()[:, None, :, None] * torch.tensor(freq, dtype=torch.float64, device="cuda")
        z = torch.polar(torch.full_like(a, gain), a)

        def turn(x):
            x = x.double()
            r, rest = x[..., :c["rot"]], x[..., c["rot"]:]
            pairs = r.unflatten(-1, (-1, 2)) if c["interleaved"] else torch.stack(r.chunk(2, -1), -1)
            y = torch.view_as_real(torch.complex(pairs[..., 0].contiguous(), pairs[..., 1].contiguous()) * z)
            y = y.flatten(-2) if c["interleaved"] else torch.cat([y[..., 0], y[..., 1]], -1)
            return torch.cat([y, rest], -1)

        return turn(s["Q"]), turn(s["K"])
    new, kv = _lens(c)
    rows = [torch.tensor([[p // c["page"], p % c["page"]] for p in range(k)], device="cuda") for k in kv]
    if c["kind"] == "write":
        if c["e4m3"]:
            # every value of the format from its bits, and the nearest of them (of two as near, the one with an even code)
            code = torch.arange(127, device="cuda", dtype=torch.float64)
            ex, ma = torch.div(code, 8, rounding_mode="floor"), code % 8
            value = torch.where(ex == 0, ma * 2.0 ** -9, (1 + ma / 8) * two_to(ex - 7))

            def packed(x):
                x = x.double()
                big = x.abs().amax(-1, keepdim=True)
                e = torch.ceil(torch.log2(big / E4M3_MAX))
                e = torch.where(big > E4M3_MAX * two_to(e), e + 1, torch.where(big <= E4M3_MAX * two_to(e - 1), e - 1, e))
                y = x.abs() / two_to(e)
                hi = torch.searchsorted(value, y.contiguous()).clamp(1, 126)
                lo = hi - 1
                down, up = y - value[lo], value[hi] - y
                at = torch.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
                return value[at] * torch.sign(x), (e.squeeze(-1) + 127).to(torch.uint8)
        else:
            packed = lambda x: (x.double(), None)
        out = []
        for src in ("K", "V"):
            q, e = packed(s[src])
            pool = torch.zeros(s["kp"].shape, dtype=torch.float64, device="cuda")
            exps = torch.zeros(s["kp"].shape[:3], dtype=torch.uint8, device="cuda")
            at = 0
            for i in range(c["n"]):
                where = rows[i][kv[i] - new[i]:]
                page = s["table"][i].long()[where[:, 0]]
                pool[page, :, where[:, 1]] = q[at:at + new[i]]
                if e is not None:
                    exps[page, :, where[:, 1]] = e[at:at + new[i]]
                at += new[i]
            out.append((pool, exps if e is not None else None))
        return out[0][0], out[1][0], out[0][1], out[1][1]

    def sequence(pages, scales, i, first=0):
        """[Hkv, kv - first, d]: the cached rows from `first` on."""
        where = rows[i][first:]
        page = s["table"][i].long()[where[:, 0]].clamp(min=0)
        x = (pages.view(torch.uint8) if scales is not None else pages)[page, :, where[:, 1]]
        x = x.view(pages.dtype).double()
        if scales is not None:
            x = x * two_to(scales[page, :, where[:, 1]].to(torch.int64) - 127)[..., None]
        return x.transpose(0, 1)

    if c["kind"] == "read":
        K, V = (torch.zeros(c["n"], c["Hkv"], c["kv"], c["d"], dtype=torch.float64, device="cuda") for _ in "kv")
        for i in range(c["n"]):
            K[i, :, :kv[i]], V[i, :, :kv[i]] = sequence(s["kp"], s["ks"], i), sequence(s["vp"], s["vs"], i)
        return K, V
    O, lse, at, g = s["O"].double(), s["lse"].double(), 0, c["Hq"] // c["Hkv"]
    for i in range(c["n"]):
        first = max(0, kv[i] - new[i] - c["window"] + 1) if c["window"] else 0
        K, V = sequence(s["kp"], s["ks"], i, first), sequence(s["vp"], s["vs"], i, first)
        p = torch.arange(kv[i] - new[i], kv[i], device="cuda")[:, None]
        key = torch.arange(first, kv[i], device="cuda")
        there = key <= p
        if c["window"]:
            there &= key > p - c["window"]
        for h in range(c["Hq"]):
            x = s["Q"][at:at + new[i], h].double() @ K[h // g].T.contiguous() / c["d"] ** 0.5
            x = torch.where(there, x, -math.inf)
            lse[at:at + new[i], h] = torch.logsumexp(x, -1)
            O[at:at + new[i], h] = torch.softmax(x, -1) @ V[h // g]
        at += new[i]
    return O, lse

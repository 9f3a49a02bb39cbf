"""The work of a receiver that uses its KV cache, as it is timed: new keys and
values are appended to the cache (with key and query norm and the position
rotation), rows of a cache are read back, and packed queries attend over it, as
whole prompts, as questions behind a transferred context and one token at a time.
Caches are bf16, fp32 or 4-bit, contiguous or paged.

4-bit caches hold, for every row and head, codes in groups of 32 channels:
value = scale * (code - 8), scale a bf16 number with at most 5 significant bits,
codes 1 .. 15.  Channel c = 32 g + 4 j + i of a head of D channels is nibble
(D / 8) j + 4 g + i of its D / 2 bytes (low nibble first).

With `own` false the plain forms run: elementary torch operations in fp32, rounded
once at the end.  With `own` true the same tensors go through the package's
KVCache.
"""

import math
import random

import torch

own = False

DEV = "cuda"
GROUP = 32
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _append(name=None, **kw):
    c = dict(kind="append", cache="bf16", dtype="bf16", n=8, lo=1, hi=1, seed=1, start=400, H=8, G=4, D=128,
             block=16, norm=False)
    c.update(kw)
    return c if name is None else dict(name=name, **c)


def _read(name=None, **kw):
    c = dict(kind="read", cache="q4", dtype="bf16", n=4, lo=1000, hi=8191, seed=1, start=0, H=8, G=1, D=128, block=16)
    c.update(kw)
    return c if name is None else dict(name=name, **c)


def _attend(name=None, **kw):
    # lo .. hi: query tokens of a sequence; past_lo .. past_hi: cached tokens before them
    c = dict(kind="attend", cache="bf16", dtype="bf16", n=1, lo=1, hi=1, past_lo=0, past_hi=0, seed=1, H=8, G=4,
             D=128, block=0)
    c.update(kw)
    return c if name is None else dict(name=name, **c)


def listed():
    return [
        # One decoding step of a batch of 32 receivers: a token each, its query rotated in the same call.
        _append("append_step", n=32, start=500),
        # Eight ragged prompts into a paged cache of a model with key and query norm and seven query heads a KV head.
        _append("append_prompt", n=8, lo=1021, hi=8191, seed=3, start=0, H=4, G=7, norm=True),
        # A long prompt into a 4-bit cache, and its rows as the cache now holds them (what the next agent gets).
        _append("append_q4", cache="q4", n=1, lo=8191, hi=8191, start=129, H=8, G=4),
        # The message of an agent that keeps its caches in 4 bits, read back as a sender cache.
        _read("read_q4", n=4, lo=2048, hi=16384, seed=5),
        # The smallest model of the tests: fp32, narrow heads, a few short texts.
        _attend("attend_tiny_f32", cache="f32", dtype="f32", n=3, lo=1, hi=256, seed=2, H=4, G=2, D=32),
        # An ordinary batch of prompts, packed, of different lengths.
        _attend("attend_prompts", n=6, lo=257, hi=4096, seed=7),
        # One long prompt: the native prefill that a transfer is compared with.
        _attend("attend_long", n=1, lo=8192, hi=8192),
        # Short questions behind transferred contexts of 4K to 32K tokens.
        _attend("attend_question", n=4, lo=17, hi=96, past_lo=4096, past_hi=32768, seed=4, block=16),
        # One receiver's decoding step after a short context: latency.
        _attend("step_single", n=1, past_lo=1000, past_hi=1000, block=16),
        # A ragged batch's decoding step, seven query heads a KV head.
        _attend("step_batch", n=32, past_lo=500, past_hi=16384, seed=9, H=4, G=7, block=16),
        # Four receivers of very long contexts, held in 4 bits.
        _attend("step_q4_long", cache="q4", n=4, past_lo=131071, past_hi=131071, block=16),
        # The questions again, behind contexts held in 4 bits.
        _attend("question_q4", cache="q4", n=4, lo=17, hi=96, past_lo=4096, past_hi=32768, seed=6, block=16),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "append", "read", "prompt", "prompt", "question", "step", "step"])
    H = rng.choice([1, 2, 4, 8, 10])
    G = rng.choice([1, 2, 4, 5, 7, 8])
    D = rng.choice([64, 128, 128])
    seed = rng.randrange(1 << 20)
    block = rng.choice([0, 8, 16, 16, 32, 64])
    cache = rng.choice(["bf16", "bf16", "q4"])
    if kind == "append":
        n = _log_int(rng, 1, 64)
        hi = _log_int(rng, 1, max(2, 16000 // n))
        cache = rng.choice([cache, cache, cache, "f32"])
        norm = cache != "q4" and rng.random() < 0.5
        return _append(cache=cache, dtype="f32" if cache == "f32" else "bf16", n=n, lo=rng.randint(1, hi), hi=hi, seed=seed, start=rng.randrange(0, 700), H=H, G=G,
                       D=D, block=block, norm=norm)
    if kind == "read":
        n = _log_int(rng, 1, 16)
        hi = _log_int(rng, 1, max(2, 32000 // n))
        return _read(cache=cache, n=n, lo=rng.randint(1, hi), hi=hi, seed=seed, start=rng.randrange(0, 300), H=H, D=D,
                     block=block)
    if kind == "prompt":
        if rng.random() < 0.2:
            n = rng.randint(1, 6)
            return _attend(cache="f32", dtype="f32", n=n, lo=1, hi=_log_int(rng, 16, 600), seed=seed, H=min(H, 4),
                           G=min(G, 4), D=rng.choice([32, 64, 128]), block=block)
        n = _log_int(rng, 1, 16)
        most = min(8192, int(math.sqrt(8192.0 * 8192 * 32 * 128 / (n * H * G * D))))
        hi = _log_int(rng, 16, max(17, most))
        return _attend(cache=cache, n=n, lo=rng.randint(1, hi), hi=hi, seed=seed, H=H, G=G, D=D, block=block)
    n = _log_int(rng, 1, 48 if kind == "step" else 8)
    most = min(131072, 4 * 131072 * 8 * 36 // (n * H * (36 if cache == "q4" else 128)))
    past = _log_int(rng, 64, max(65, most if kind == "step" else min(most, 32768)))
    lo, hi = (1, 1) if kind == "step" else (rng.randint(1, 16), _log_int(rng, 17, 128))
    return _attend(cache=cache, n=n, lo=lo, hi=hi, past_lo=rng.randint(1, past), past_hi=past, seed=seed, H=H, G=G, D=D,
                   block=block)


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _lengths(rng, n, lo, hi):
    return [lo if lo == hi else min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(max(lo, 0.5)), math.log(hi)))))))
            for _ in range(n)]


def _shape_of(case):
    """New tokens and tokens already cached of every sequence: sizes, the same for every seed of the inputs."""
    rng = random.Random(case["seed"])
    new = _lengths(rng, case["n"], case["lo"], case["hi"])
    if case["kind"] == "attend":
        if case["past_hi"] > 0:
            past = _lengths(rng, case["n"], case["past_lo"], case["past_hi"])
        else:
            past = [0] * case["n"]
    else:
        past = [rng.randrange(0, case["start"] + 1) if case["n"] > 1 else case["start"] for _ in range(case["n"])]
    return new, past


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _channel_scales(g, H, D):
    """Channels of different size, as caches have them: 10 ** U(-0.5, 0.5)."""
    return 10.0 ** (torch.rand((H, D), generator=g, device=DEV) - 0.5)


def _rope_table(n_pos, D, theta=500000.0):
    """cos and sin of every position and channel pair, fp32 [n_pos][D/2][2]."""
    inv = (theta ** (-torch.arange(0, D, 2, dtype=torch.float64, device=DEV) / D)).float().double()
    a = torch.arange(n_pos, dtype=torch.float64, device=DEV)[:, None] * inv[None, :]
    return torch.stack((a.cos(), a.sin()), dim=-1).float().contiguous()


def _scales5(g, shape):
    """Scales as a 4-bit cache holds them: 5 significant bits, around 0.25."""
    s = 0.25 * torch.exp(0.5 * torch.randn(shape, generator=g, device=DEV))
    return ((s.view(torch.int32) + 0x40000) & -0x80000).view(torch.float32).to(torch.bfloat16)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    new, past = _shape_of(case)
    n, H, G, D, block = case["n"], case["H"], case["G"], case["D"], case["block"]
    dt = DTYPES[case["dtype"]]
    T = sum(new)
    total = [a + b for a, b in zip(new, past)]
    ptr = [0]
    for a in new:
        ptr.append(ptr[-1] + a)
    st = dict(case=case, T=T, max_new=max(new), max_total=max(total), tok_ptr=_i32(ptr), start=_i32(past),
              kv_len=_i32(total))
    # where the rows of a sequence are: a block table, or the sequences one after another
    if block:
        need = [-(-t // block) for t in total]
        n_blocks = sum(need) + -(-sum(need) // 10)
        perm = torch.randperm(n_blocks, generator=g, device=DEV).to(torch.int32)
        table = torch.zeros((n, max(need)), dtype=torch.int32, device=DEV)
        at = 0
        for i, k in enumerate(need):
            table[i, :k] = perm[at:at + k]
            at += k
        rows = n_blocks * block
        st["table"], st["row0"] = table, None
    else:
        rows = sum(total)
        at = [0]
        for t in total:
            at.append(at[-1] + t)
        st["table"], st["row0"] = None, _i32(at[:-1])
    st["rows"] = rows
    # the cache, as earlier calls left it
    if case["cache"] == "q4":
        low = torch.randint(1, 16, (2, H, rows, D // 2), generator=g, device=DEV, dtype=torch.uint8)
        high = torch.randint(1, 16, (2, H, rows, D // 2), generator=g, device=DEV, dtype=torch.uint8)
        st["codes"] = low | (high << 4)
        del low, high
        st["scales"] = _scales5(g, (2, H, rows, D // GROUP))
    else:
        kv = torch.randn((2, rows, H, D), generator=g, device=DEV, dtype=dt)
        kv *= _channel_scales(g, H, D).to(dt)
        st["kv"] = kv
    q_scale = 1.5 if case["kind"] == "attend" else 1.0
    st["q"] = (torch.randn((T, H * G, D), generator=g, device=DEV) * q_scale).to(dt)
    if case["kind"] == "append":
        scale = _channel_scales(g, H, D)
        st["k"] = (torch.randn((T, H, D), generator=g, device=DEV) * scale).to(dt)
        st["v"] = torch.randn((T, H, D), generator=g, device=DEV).to(dt)
        st["rope"] = _rope_table(max(total), D)
        st["k_norm"] = st["q_norm"] = None
        if case["norm"]:
            st["k_norm"] = 1.0 + 0.2 * torch.randn(D, generator=g, device=DEV)
            st["q_norm"] = 1.0 + 0.2 * torch.randn(D, generator=g, device=DEV)
        st["q_out"] = torch.empty_like(st["q"])
    if case["kind"] != "attend":
        st["k_out"] = torch.empty((T, H, D), dtype=dt, device=DEV)
        st["v_out"] = torch.empty((T, H, D), dtype=dt, device=DEV)
    else:
        st["out"] = torch.empty_like(st["q"])
    if own:
        from paper_2609_32259_gb300 import pipeline

        if case["cache"] == "q4":
            st["cache"] = pipeline.KVCache(kind="q4", H=H, D=D, n_seq=n, codes=st["codes"][None],
                                           scales=st["scales"][None], block_table=st["table"], block_size=block,
                                           row0=st["row0"])
        else:
            st["cache"] = pipeline.KVCache(kind=case["cache"], H=H, D=D, n_seq=n, kv=st["kv"][None],
                                           block_table=st["table"], block_size=block, row0=st["row0"])
    return st


# ---------------------------------------------------------------------------
# The plain forms
# ---------------------------------------------------------------------------
def _token_rows(st):
    """Sequence and cache row of every new token."""
    T = st["T"]
    tok = torch.arange(T, device=DEV)
    seq = torch.searchsorted(st["tok_ptr"][1:].long(), tok, right=True)
    at = tok - st["tok_ptr"].long()[seq] + st["start"].long()[seq]
    return seq, at, _rows_of(st, seq, at)


def _rows_of(st, seq, at):
    block = st["case"]["block"]
    if block:
        return st["table"].long()[seq, at // block] * block + at % block
    return st["row0"].long()[seq] + at


def _rope(x, table):
    """Rotates the pairs (i, i + D/2) of x [T, heads, D] by table [T, D/2, 2]."""
    half = x.shape[-1] // 2
    a, b = x[..., :half], x[..., half:]
    c, s = table[:, None, :, 0], table[:, None, :, 1]
    return torch.cat((a * c - b * s, b * c + a * s), dim=-1)


def _norm(x, w):
    return x if w is None else x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + 1e-6) * w


def _held_in_4_bits(x):
    """The values that a 4-bit cache holds for x [..., D]."""
    y = x.reshape(*x.shape[:-1], -1, GROUP)
    s = y.abs().amax(dim=-1, keepdim=True) / 7.0
    s = ((s.view(torch.int32) + 0x40000) & -0x80000).view(torch.float32)
    code = torch.where(s > 0, torch.round(y / s).clamp(-7, 7), torch.zeros_like(y))
    return (code * s).reshape(x.shape)


def _unpacked(st, which, rows):
    """fp32 values [*rows.shape, H, D] of a 4-bit cache's rows."""
    case = st["case"]
    H, D = case["H"], case["D"]
    flat = rows.reshape(-1)
    b = st["codes"][which][:, flat]  # [H, R, D/2]
    code = torch.stack((b & 15, b >> 4), dim=-1).reshape(H, -1, 8, D // GROUP, 4)
    code = code.permute(1, 0, 3, 2, 4).reshape(-1, H, D // GROUP, GROUP)
    s = st["scales"][which][:, flat].permute(1, 0, 2).float()
    return ((code.float() - 8.0) * s[..., None]).reshape(*rows.shape, H, D)


def _plain_append(st):
    case = st["case"]
    seq, at, rows = _token_rows(st)
    dt = st["q"].dtype
    table = st["rope"][at]
    k = _rope(_norm(st["k"].float(), st["k_norm"]), table)
    v = st["v"].float()
    q = _rope(_norm(st["q"].float(), st["q_norm"]), table).to(dt)
    if case["cache"] == "q4":
        return {"q": q, "k": _held_in_4_bits(k).to(dt), "v": _held_in_4_bits(v).to(dt)}
    st["kv"][0, rows] = k.to(dt)
    st["kv"][1, rows] = v.to(dt)
    return {"q": q, "kv": st["kv"]}


def _plain_read(st):
    _, _, rows = _token_rows(st)
    dt = DTYPES[st["case"]["dtype"]]
    if st["case"]["cache"] == "q4":
        return {"k": _unpacked(st, 0, rows).to(dt), "v": _unpacked(st, 1, rows).to(dt)}
    return {"k": st["kv"][0, rows].to(dt), "v": st["kv"][1, rows].to(dt)}


def _plain_attend(st):
    case = st["case"]
    n, H, G, D = case["n"], case["H"], case["G"], case["D"]
    Lq, Lk = st["max_new"], st["max_total"]
    # sequences padded to the longest one
    qi = torch.arange(Lq, device=DEV)
    kj = torch.arange(Lk, device=DEV)
    nq = (st["tok_ptr"][1:] - st["tok_ptr"][:-1]).long()
    nk = st["kv_len"].long()
    tok = st["tok_ptr"][:-1].long()[:, None] + qi[None, :]
    there = qi[None, :] < nq[:, None]
    at = torch.minimum(kj[None, :], nk[:, None] - 1)
    rows = _rows_of(st, torch.arange(n, device=DEV)[:, None].expand(n, Lk), at)
    if case["cache"] == "q4":
        k, v = _unpacked(st, 0, rows), _unpacked(st, 1, rows)
    else:
        k, v = st["kv"][0, rows].float(), st["kv"][1, rows].float()
    q = st["q"].float()[tok.clamp(max=st["T"] - 1)] * (1.0 / math.sqrt(D))
    q = q.reshape(n, Lq, H, G, D).permute(0, 2, 3, 1, 4).reshape(n, H, G * Lq, D)
    s = (q @ k.permute(0, 2, 3, 1)).reshape(n, H, G, Lq, Lk)
    seen = kj[None, None, :] <= (nk - nq)[:, None, None] + qi[None, :, None]
    s.masked_fill_(~seen[:, None, None], -math.inf)
    top = s.amax(dim=-1, keepdim=True)
    s.sub_(torch.where(torch.isinf(top), torch.zeros_like(top), top)).exp_()
    total = s.sum(dim=-1, keepdim=True)
    o = s.reshape(n, H, G * Lq, Lk) @ v.permute(0, 2, 1, 3)
    o = o.reshape(n, H, G, Lq, D) / torch.where(total > 0, total, torch.ones_like(total))
    return o.permute(0, 3, 1, 2, 4).reshape(n, Lq, H * G, D)[there].to(DTYPES[case["dtype"]])


def run(state):
    st = state
    kind = st["case"]["kind"]
    if not own:
        return {"append": _plain_append, "read": _plain_read, "attend": _plain_attend}[kind](st)
    cache = st["cache"]
    if kind == "append":
        cache.append(0, st["k"], st["v"], st["tok_ptr"], st["start"], rope=st["rope"], q=st["q"], q_out=st["q_out"],
                     k_norm=st["k_norm"], q_norm=st["q_norm"], eps=1e-6)
        if st["case"]["cache"] == "q4":
            cache.read(0, st["k_out"], st["v_out"], st["tok_ptr"], st["start"])
            return {"q": st["q_out"], "k": st["k_out"], "v": st["v_out"]}
        return {"q": st["q_out"], "kv": st["kv"]}
    if kind == "read":
        cache.read(0, st["k_out"], st["v_out"], st["tok_ptr"], st["start"])
        return {"k": st["k_out"], "v": st["v_out"]}
    cache.attend(0, st["q"], st["out"], st["tok_ptr"], st["kv_len"], max_q_len=st["max_new"],
                 max_kv_len=st["max_total"])
    return st["out"]


# ---------------------------------------------------------------------------
# 64-bit values, sequence by sequence and head by head
# ---------------------------------------------------------------------------
def _held_exact(x):
    out = torch.empty_like(x)
    for c in range(0, x.shape[-1], GROUP):
        y = x[..., c:c + GROUP]
        a = y.abs().max(dim=-1, keepdim=True).values / 7
        mant, exp = torch.frexp(a)
        s = torch.ldexp(torch.floor(mant * 32 + 0.5), exp - 5)
        out[..., c:c + GROUP] = torch.where(s > 0, torch.round(y / s).clamp(-7, 7) * s, torch.zeros_like(y))
    return out


def _exact_rotated(x, norm, pos, table):
    y = x.double()
    if norm is not None:
        y = y / torch.sqrt((y ** 2).sum(-1, keepdim=True) / y.shape[-1] + 1e-6) * norm.double()
    D = y.shape[-1]
    z = torch.complex(y[..., : D // 2], y[..., D // 2:])
    t = table.double()[pos]
    z = z * torch.complex(t[..., 0], t[..., 1])[:, None, :]
    return torch.cat((z.real, z.imag), dim=-1)


def _seq_rows(st, s, lo, hi):
    at = torch.arange(lo, hi, device=DEV)
    if st["table"] is None:
        return int(st["row0"][s]) + at
    b = st["case"]["block"]
    return st["table"][s].long()[torch.div(at, b, rounding_mode="floor")] * b + at % b


def _exact_rows(st, which, rows, h):
    """Rows of one head of the cache in fp64."""
    case = st["case"]
    D = case["D"]
    if case["cache"] != "q4":
        return st["kv"][which, rows, h].double()
    b = st["codes"][which, h, rows].long()
    s = st["scales"][which, h, rows].double()
    c = torch.arange(D, device=DEV)
    grp, j, i = c // GROUP, (c % GROUP) // 4, c % 4
    nib = (D // 8) * j + 4 * grp + i
    return (((b[:, nib // 2] >> (4 * (nib % 2))) & 15) - 8).double() * s[:, grp]


def exact(case, seed):
    st = prepare(case, seed)
    new, past = _shape_of(case)
    H, G, D = case["H"], case["G"], case["D"]
    if case["kind"] == "attend":
        out = torch.empty((st["T"], H * G, D), dtype=torch.float64, device=DEV)
        t0 = 0
        for s, (a, b) in enumerate(zip(new, past)):
            rows = _seq_rows(st, s, 0, a + b)
            for h in range(H):
                k, v = _exact_rows(st, 0, rows, h), _exact_rows(st, 1, rows, h)
                for g in range(G):
                    for i0 in range(0, a, 4096):
                        i1 = min(a, i0 + 4096)
                        m = b + i1
                        x = st["q"][t0 + i0:t0 + i1, h * G + g].double() @ k[:m].T / math.sqrt(D)
                        x += torch.full_like(x, -math.inf).triu_(diagonal=b + i0 + 1)
                        out[t0 + i0:t0 + i1, h * G + g] = torch.softmax(x, dim=-1) @ v[:m]
            t0 += a
        return out
    rows, pos = [], []
    for s, (a, b) in enumerate(zip(new, past)):
        rows.append(_seq_rows(st, s, b, a + b))
        pos.append(torch.arange(b, a + b, device=DEV))
    rows, pos = torch.cat(rows), torch.cat(pos)
    if case["kind"] == "read":
        return {w: torch.stack([_exact_rows(st, i, rows, h) for h in range(H)], dim=1) for i, w in enumerate("kv")}
    q = _exact_rotated(st["q"], st["q_norm"], pos, st["rope"])
    k = _exact_rotated(st["k"], st["k_norm"], pos, st["rope"])
    v = st["v"].double()
    if case["cache"] == "q4":
        return {"q": q, "k": _held_exact(k), "v": _held_exact(v)}
    kv = st["kv"].double()
    kv[0, rows], kv[1, rows] = k, v
    return {"q": q, "kv": kv}


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    new, past = _shape_of(case)
    H, G, D = case["H"], case["G"], case["D"]
    es = 4 if case["dtype"] == "f32" else 2
    row = 2 * H * (D // 2 + 2 * (D // GROUP) if case["cache"] == "q4" else D * (4 if case["cache"] == "f32" else 2))
    T = sum(new)
    if case["kind"] == "attend":
        pairs = sum(a * b + a * (a + 1) // 2 for a, b in zip(new, past))
        return {"bytes": 2 * T * H * G * D * es + sum(a + b for a, b in zip(new, past)) * row,
                "flops": 4 * D * H * G * pairs}
    if case["kind"] == "read":
        return {"bytes": T * row + 2 * T * H * D * es, "flops": 2 * T * H * D}
    positions = len(set().union(*(range(b, a + b) for a, b in zip(new, past)))) if T < 100000 else T
    moved = 2 * T * H * D * es + T * row + 2 * T * H * G * D * es + positions * D * 4
    if case["cache"] == "q4":
        moved += T * row + 2 * T * H * D * es  # read back
    return {"bytes": moved, "flops": T * (H + H * G) * D * 3}

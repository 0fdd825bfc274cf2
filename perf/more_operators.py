"""Cases of the 4-bit key/value cache (LVQ4 codes: writing, reading back, attention
for single tokens, a few tokens and prompt chunks) and of rotary positions.

A cache is a pool of pages; a page holds `page` token positions of every head in
blocks of 16 tokens.  A token's key (and value) of a head is a bias b, a scale s and
4-bit codes: value = b + s code.  A block is 16 d + 128 bytes:
  keys    [d / 16][8 g][4 c][2 l][2 t]: tokens g + 8 t, dims 4 c + l in the low and
          4 c + l + 2 in the high half of a byte
  values  [d / 16][8 g][4 c][2 l][2 t]: dims g + 8 t, tokens 2 c + l in the low and
          2 c + l + 8 in the high half of a byte
  float16 [16 tokens][4]: key scale, key bias, value scale, value bias
"""
import math
import random

import torch

own = False

B = 16  # tokens of a block
DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
F16_MOST = 65504.0


def listed():
    return [
        # a decode step's new token of 32 running sequences, written and read back: latency counts
        dict(name="append one token", op="write", type="bf16", batch=32, heads=8, d=128, page=64, past=2000, new=1, fused=True, even=False),
        # the prompts that one scheduling step admits, out of the rows of a fused projection
        dict(name="write prompts", op="write", type="bf16", batch=12, heads=8, d=128, page=64, past=7, new=2500, fused=True, even=False),
        # a short sequence's keys and values in 32 bits, as an index over its keys would take them
        dict(name="read one sequence", op="read", type="f32", batch=1, heads=2, d=96, page=32, past=37, new=257, even=True),
        # long sequences moved out of the cache in 16 bits
        dict(name="read long sequences", op="read", type="bf16", batch=4, heads=8, d=128, page=64, past=0, new=32768, even=False),
        # one user's next token on a short context: latency counts
        dict(name="decode one", op="attend", type="bf16", batch=1, heads=8, group=4, d=128, page=64, past=332, new=1, causal=True, window=0, lse=False, even=True),
        # a full server's decode step, sequences of all lengths
        dict(name="decode batch", op="attend", type="bf16", batch=96, heads=8, group=4, d=128, page=64, past=10001, new=1, causal=True, window=0, lse=False, even=False),
        # one very long document, merged with other parts by its log-sum-exp
        dict(name="decode long", op="attend", type="f16", batch=1, heads=8, group=8, d=128, page=128, past=262150, new=1, causal=True, window=0, lse=True, even=True),
        # five guessed tokens checked at once, wide heads, a sliding window
        dict(name="verify in a window", op="attend", type="bf16", batch=16, heads=2, group=8, d=256, page=32, past=5000, new=5, causal=True, window=1024, lse=False, even=False),
        # a chunk of two long prompts behind what the cache holds of them
        dict(name="prompt chunk", op="attend", type="bf16", batch=2, heads=8, group=4, d=128, page=64, past=6144, new=2048, causal=True, window=0, lse=False, even=False),
        # whole prompts of a small model with ungrouped heads
        dict(name="whole prompts", op="attend", type="f16", batch=4, heads=16, group=1, d=64, page=16, past=0, new=4096, causal=True, window=0, lse=True, even=False),
        # the query and key rows of a decode step, out of a fused projection's rows: latency counts
        dict(name="rotate a step", op="rotate", type="bf16", batch=64, heads=8, group=4, d=128, dims=128, layout="half", scaling="none", past=8191, new=1, fused=True, back=False, even=False),
        # the gradients of prompts' rotated queries and keys, neighbouring dims of half of each head, a stretched context
        dict(name="rotate gradients", op="rotate", type="bf16", batch=12, heads=8, group=4, d=128, dims=64, layout="interleaved", scaling="turns", past=30000, new=2500, fused=False, back=True, even=False),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    d = rng.choice([64, 64, 80, 96, 128, 128, 128, 192, 256])
    page = rng.choice([16, 32, 64, 128])
    heads = rng.choice([1, 2, 3, 4, 8, 8, 16])
    op = rng.choice(["write", "read", "attend", "attend", "attend", "attend", "rotate", "rotate"])
    if op in ("write", "read"):
        case = dict(op=op, type=rng.choice(["bf16", "bf16", "f16", "f32"]), batch=log(1, 64), heads=heads, d=d, page=page,
                    past=rng.choice([0, log(1, 4000)]), new=log(1, 8000), even=rng.random() < 0.3)
        if op == "write":
            case["fused"] = rng.random() < 0.5
        while case["batch"] * case["new"] * heads * d > 30e6:
            case["new"] = max(1, case["new"] // 2)
        return case
    group = rng.choice([1, 2, 4, 4, 6, 7, 8, 16])
    if op == "rotate":
        d = rng.choice([d, d, d, rng.randrange(20, 200, 2)])
        dims = rng.choice([d, d, d // 4 * 2, 2 * rng.randrange(2, d // 2 + 1)])
        case = dict(op="rotate", type=rng.choice(["bf16", "bf16", "f16", "f32"]), batch=log(1, 64), heads=heads, group=group, d=d, dims=dims,
                    layout=rng.choice(["half", "interleaved"]), scaling=rng.choice(["none", "none", "linear", "base", "index", "turns"]),
                    past=rng.choice([0, log(1, 4000), log(1000, 1000000)]), new=rng.choice([1, log(1, 8000)]), fused=rng.random() < 0.5,
                    back=rng.random() < 0.3, even=rng.random() < 0.3)
        while case["batch"] * case["new"] * heads * (group + 1) * d > 150e6:
            case["new"] = max(1, case["new"] // 2)
        return case
    kind = rng.choice(["decode", "decode", "few", "prompt"])
    new = 1 if kind == "decode" else log(2, 16) if kind == "few" else log(17, 3000)
    typ = rng.choice(["bf16", "bf16", "f16", "f32" if kind != "prompt" else "bf16"])
    batch = log(1, 100 if kind == "decode" else 16)
    past = rng.choice([0, log(1, 4000)]) if kind == "prompt" else log(1, 60000 if kind == "decode" else 16000)
    case = dict(op="attend", type=typ, batch=batch, heads=heads, group=group, d=d, page=page, past=past, new=new,
                causal=rng.random() < 0.85, window=0, lse=rng.random() < 0.5, even=rng.random() < 0.3)
    if case["causal"] and rng.random() < 0.25:
        case["window"] = log(20, 4000)
    most = 30e6 if typ == "f32" else 300e6
    while case["batch"] * (case["past"] + new) * heads * d > most or \
            case["batch"] * (case["past"] + new) * new * heads * group * d > 100e9:
        if case["batch"] > 1:
            case["batch"] //= 2
        elif case["past"] > 0:
            case["past"] //= 2
        else:
            new = case["new"] = new // 2
    return case


def sizes(case):
    """Tokens held before and new tokens of each sequence: the first one has the
    case's own numbers, the others (unless even) fractions of them."""
    rng = random.Random(case["batch"] * 7919 + case["past"] * 31 + case["new"])
    past, new = [], []
    for i in range(case["batch"]):
        f = 1.0 if i == 0 or case["even"] else 0.05 + 0.95 * rng.random()
        past.append(int(case["past"] * f))
        n = case["new"]
        new.append(n if n <= 16 else max(1, int(n * (1.0 if i == 0 or case["even"] else 0.05 + 0.95 * rng.random()))))
    return past, new


# ---- the format


def bits_up(y):
    """float64 y >= 0 as the smallest float16 that is not below it."""
    h = y.float().half()
    return torch.where(h.double() < y, (h.view(torch.int16) + 1).view(torch.float16), h)


def bits_down(y):
    """float32 y as the largest float16 that is not above it."""
    h = y.half()
    i = h.view(torch.int16)
    # one step down: a positive number's bits less one, a negative one's (and zero's) magnitude one more
    down = torch.where(h > 0, i - 1, torch.where(h < 0, i + 1, torch.full_like(i, -32767)))
    return torch.where(h.float() > y, down.view(torch.float16), h)


def quantise(x):
    """Scale and bias (float16) and codes (uint8) of vectors x [..., d]."""
    x = x.float()
    fine = torch.isfinite(x)
    some = fine.any(-1)
    big = torch.full_like(x, math.inf)
    lo = torch.where(some, torch.where(fine, x, big).amin(-1), torch.zeros_like(x[..., 0])).clamp(-F16_MOST, F16_MOST)
    hi = torch.where(some, torch.where(fine, x, -big).amax(-1), torch.zeros_like(lo)).clamp(-F16_MOST, F16_MOST)
    b = bits_down(lo)
    s = bits_up((hi.double() - b.double()) / 15)
    step = torch.where(s > 0, s, torch.ones_like(s)).double()
    q = ((x.double() - b.double()[..., None]) / step[..., None]).round()  # in 64 bits: values between two codes
    q = torch.nan_to_num(q, nan=0.0).clamp(0, 15)
    return s, b, torch.where((s > 0)[..., None], q, torch.zeros_like(q)).to(torch.uint8)


def pack(name, c):
    """Codes [..., 16 tokens, d] as a block's bytes [..., 8 d]."""
    n, d = c.dim() - 2, c.shape[-1]
    lead = list(range(n))
    if name == "k":  # token 8 t + g, dim 16 w + 4 c + 2 h + l
        c = c.view(*c.shape[:n], 2, 8, d // 16, 4, 2, 2).permute(*lead, n + 2, n + 1, n + 3, n + 5, n, n + 4)
    else:  # token 8 h + 2 c + l, dim 16 w + 8 t + g
        c = c.view(*c.shape[:n], 2, 4, 2, d // 16, 2, 8).permute(*lead, n + 3, n + 5, n + 1, n + 2, n + 4, n)
    return (c[..., 0] | c[..., 1] << 4).reshape(*c.shape[:n], 8 * d)


def unpack(name, u, d):
    """The codes [..., 16 tokens, d] of a block's bytes."""
    n = u.dim() - 1
    lead = list(range(n))
    c = torch.stack([u & 15, u >> 4], -1).view(*u.shape[:n], d // 16, 8, 4, 2, 2, 2)  # w g c l t h
    if name == "k":
        return c.permute(*lead, n + 4, n + 1, n, n + 2, n + 5, n + 3).reshape(*u.shape[:n], B, d)
    return c.permute(*lead, n + 5, n + 2, n + 3, n, n + 4, n + 1).reshape(*u.shape[:n], B, d)


def parts(blocks, d):
    """Views of blocks [..., 16 d + 128]: key bytes, value bytes, float16 [..., 16, 4]."""
    sc = blocks[..., 16 * d:].view(torch.float16)
    return blocks[..., :8 * d], blocks[..., 8 * d:16 * d], sc.view(*sc.shape[:-1], B, 4)


# ---- inputs


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dev = "cuda"
    past, new = sizes(case)
    heads, d, typ = case["heads"], case["d"], DT[case["type"]]
    total = [p + n for p, n in zip(past, new)]
    st = dict(case=case, batch=case["batch"], heads=heads, d=d, start=torch.tensor(past, dtype=torch.int32, device=dev),
              length=torch.tensor(total, dtype=torch.int32, device=dev),
              cu=torch.tensor([0] + torch.tensor(new).cumsum(0).tolist(), dtype=torch.int32, device=dev),
              tokens=sum(new), max_new=max(new), max_len=max(total))
    # channels of unequal size, keys' around means of their own
    size = torch.exp(0.5 * torch.randn(2, heads, d, generator=g, device=dev))
    mean = 0.5 * torch.randn(heads, d, generator=g, device=dev)
    if case["op"] == "rotate":
        hq = heads * case["group"]
        rows = torch.randn(sum(new), hq + heads * (2 if case["fused"] else 1), d, generator=g, device=dev)
        rows[:, hq:hq + heads] = rows[:, hq:hq + heads] * size[0] + mean
        rows = rows.to(typ)
        st["Q"], st["K"] = rows[:, :hq], rows[:, hq:hq + heads]
        if not case["fused"]:
            st["Q"], st["K"] = st["Q"].contiguous(), st["K"].contiguous()
        return st
    page = st["page"] = case["page"]
    need = [-(-t // page) for t in total]
    cols, pages = max(need) + 1, sum(need) + 3
    order = torch.randperm(pages, generator=g, device=dev, dtype=torch.int64).to(torch.int32)
    table = st["table"] = torch.full((case["batch"], cols), -1, dtype=torch.int32, device=dev)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    blocks = st["blocks"] = torch.empty(pages, heads, page // B, 16 * d + 128, dtype=torch.uint8, device=dev)
    stretch = max(1, int(1e8) // (heads * page * d))
    for lo in range(0, pages, stretch):
        some = blocks[lo:lo + stretch]
        k, v, sc = parts(some, d)
        for t, (name, where) in enumerate((("k", k), ("v", v))):
            x = torch.randn(*some.shape[:3], B, d, generator=g, device=dev) * size[t][:, None, None]
            if t == 0:
                x += mean[:, None, None]
            low, high = x.aminmax(dim=-1)
            b = bits_down(low)
            s = ((high - b.float()) * (1.001 / 15)).half()
            where.copy_(pack(name, ((x - b.float()[..., None]) / s.float()[..., None]).round().clamp(0, 15).to(torch.uint8)))
            sc[..., 2 * t], sc[..., 2 * t + 1] = s, b
    if case["op"] == "write":
        wide = heads * (4 if case["fused"] else 0)
        rows = torch.randn(sum(new), wide + 2 * heads, d, generator=g, device=dev)
        rows[:, wide:wide + heads] = rows[:, wide:wide + heads] * size[0] + mean
        rows = rows.to(typ)
        st["K"], st["V"] = rows[:, wide:wide + heads], rows[:, wide + heads:]
        if not case["fused"]:
            st["K"], st["V"] = st["K"].contiguous(), st["V"].contiguous()
        # what the call wrote, from the first token of the block that each sequence's new tokens begin in
        first = [p - p % B for p in past]
        st["first"] = torch.tensor(first, dtype=torch.int32, device=dev)
        count = [p + n - f for p, n, f in zip(past, new, first)]
        st["back"] = torch.tensor([0] + torch.tensor(count).cumsum(0).tolist(), dtype=torch.int32, device=dev)
        st["back_tokens"], st["back_max"] = sum(count), max(count)
    elif case["op"] == "read":
        st.update(first=st["start"], back=st["cu"], back_tokens=st["tokens"], back_max=st["max_new"])
    else:
        st["Q"] = (1.5 * torch.randn(sum(new), heads * case["group"], d, generator=g, device=dev)).to(typ)
    return st


#: how positions are scaled for contexts longer than trained ones
SCALED = {"none": dict(), "linear": dict(factor=4.0), "base": dict(factor=8.0),
          "index": dict(factor=16.0, trained=4096.0, low=1.0, high=32.0), "turns": dict(factor=8.0, trained=8192.0, low=1.0, high=4.0)}
BASE = 500000.0


def run(st):
    if own:
        return run_own(st)
    case = st["case"]
    if case["op"] == "rotate":
        return plain_rotate(st)
    if case["op"] == "write":
        plain_write(st)
        return plain_read(st, case["type"])
    if case["op"] == "read":
        return plain_read(st, case["type"])
    return plain_attend(st)


def run_own(st):
    import paper_2608_14648_gb300 as skm

    case = st["case"]
    if case["op"] == "rotate":
        if "rotary" not in st:  # the frequencies, which a program keeps
            layout = skm.ROTARY_HALF if case["layout"] == "half" else skm.ROTARY_INTERLEAVED
            scaling = {"none": skm.ROTARY_NONE, "linear": skm.ROTARY_LINEAR, "base": skm.ROTARY_BASE, "index": skm.ROTARY_INDEX,
                       "turns": skm.ROTARY_TURNS}[case["scaling"]]
            st["rotary"] = skm.Rotary(case["dims"], base=BASE, layout=layout, scaling=scaling, **SCALED[case["scaling"]])
        Q, K = skm.skm_kv_rotate(st["rotary"], st["start"], st["cu"], (st["Q"], st["K"]), st["max_new"], transpose=case["back"])
        return {"q": Q, "k": K}
    cache = st.get("cache")
    if cache is None:  # the handle, and attention's workspace, that a program keeps
        cache = st["cache"] = skm.KVCache4(st["heads"], st["d"], st["page"], st["blocks"])
        st["dtype"] = {"bf16": skm.DTYPE_BF16, "f16": skm.DTYPE_F16, "f32": skm.DTYPE_F32}[case["type"]]
        if case["op"] == "attend":
            st["ws"] = skm.kv4_workspace(cache, st["batch"], case["heads"] * case["group"], st["tokens"], st["max_new"],
                                         st["max_len"], st["dtype"])
    if case["op"] == "attend":
        out, lse = skm.skm_kv4_attend(cache, st["table"], st["length"], st["cu"], st["Q"], st["max_new"], st["max_len"],
                                      causal=case["causal"], window=case["window"], want_lse=case["lse"], ws=st["ws"])
        return {"out": out, "lse": lse} if case["lse"] else {"out": out}
    if case["op"] == "write":
        skm.skm_kv4_write(cache, st["table"], st["start"], st["cu"], st["K"], st["V"], st["max_new"])
    K, V = skm.skm_kv4_read(cache, st["table"], st["first"], st["back"], st["back_tokens"], st["back_max"], st["dtype"])
    return {"k": K, "v": V}


# ---- the plain forms --------------------------------------------------------


def rows_of(first, cu, tokens):
    """For each of the tokens: its sequence and its position there."""
    n = (cu[1:] - cu[:-1]).to(torch.int64)
    seq = torch.repeat_interleave(torch.arange(n.numel(), device=cu.device), n, output_size=tokens)
    return seq, torch.arange(tokens, device=cu.device) - cu[:-1].to(torch.int64)[seq] + first.to(torch.int64)[seq]


def pairs(dims, layout, device):
    """The two dims of each pair."""
    i = torch.arange(dims // 2, device=device)
    return (i, i + dims // 2) if layout == "half" else (2 * i, 2 * i + 1)


def frequencies(case, device):
    """Radians a position of each pair in 64 bits, and the factor of the rotated dims."""
    dims, kind, p = case["dims"], case["scaling"], SCALED[case["scaling"]]
    i = torch.arange(dims // 2, dtype=torch.float64, device=device)
    base = BASE * p["factor"] ** (dims / (dims - 2)) if kind == "base" and dims > 2 else BASE
    f = base ** (-2 * i / dims)
    if kind == "linear":
        return f / p["factor"], 1.0
    if kind == "index":  # pairs up to one that turns `high` times over the trained length keep their frequency
        at = lambda turns: dims * math.log(p["trained"] / (2 * math.pi * turns)) / (2 * math.log(BASE))  # noqa: E731
        lo, hi = max(math.floor(at(p["high"])), 0), min(math.ceil(at(p["low"])), dims - 1)
        ramp = ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        return f * (1 - ramp) + f / p["factor"] * ramp, 0.1 * math.log(p["factor"]) + 1
    if kind == "turns":
        turns = f * p["trained"] / (2 * math.pi)
        keep = ((turns - p["low"]) / (p["high"] - p["low"])).clamp(0, 1)
        return f * keep + f / p["factor"] * (1 - keep), 1.0
    return f, 1.0


def plain_rotate(st):
    case = st["case"]
    _, pos = rows_of(st["start"], st["cu"], st["tokens"])
    f, gain = frequencies(case, pos.device)
    angle = pos.double()[:, None] * f  # in 64 bits: far positions turn thousands of times
    c, s = (gain * angle.cos()).float()[:, None], (gain * angle.sin()).float()[:, None]
    if case["back"]:
        s = -s
    a, b = pairs(case["dims"], case["layout"], pos.device)
    out = {}
    for name in "QK":
        x = st[name].float()
        y = x.clone()
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., a] * s + x[..., b] * c
        out[name.lower()] = y.to(st[name].dtype)
    return out


def plain_write(st):
    heads, d, page = st["heads"], st["d"], st["page"]
    seq, pos = rows_of(st["start"], st["cu"], st["tokens"])
    start, end = st["start"].to(torch.int64), (st["start"] + st["cu"][1:] - st["cu"][:-1]).to(torch.int64)
    # the blocks that new rows reach, and the rows of each
    low, high = start // B, (end + B - 1) // B
    which = torch.repeat_interleave(torch.arange(st["batch"], device=pos.device), high - low)
    skip = torch.cumsum(high - low, 0) - (high - low)
    blk = torch.arange(which.numel(), device=pos.device) - skip[which] + low[which]
    there = blk[:, None] * B + torch.arange(B, device=pos.device)
    fresh = ((there >= start[which][:, None]) & (there < end[which][:, None]))[:, None]  # [blocks, 1, 16]
    src = (st["cu"][:-1].to(torch.int64)[which][:, None] + there - start[which][:, None]).clamp(0, st["tokens"] - 1)
    pg, bi = st["table"][which, blk // (page // B)].to(torch.int64), blk % (page // B)
    held = st["blocks"][pg, :, bi]  # [blocks, heads, bytes]
    for t, (name, was, X) in enumerate(zip("kv", parts(held, d)[:2], (st["K"], st["V"]))):
        s, b, c = quantise(X)
        s, b, c = s[src].transpose(1, 2), b[src].transpose(1, 2), c[src].transpose(1, 2)
        was.copy_(pack(name, torch.where(fresh[..., None], c, unpack(name, was, d))))
        sc = parts(held, d)[2]
        sc[..., 2 * t] = torch.where(fresh, s, sc[..., 2 * t])
        sc[..., 2 * t + 1] = torch.where(fresh, b, sc[..., 2 * t + 1])
    st["blocks"][pg, :, bi] = held


def plain_values(st, seq, pos):
    """Keys and values at positions pos of sequences seq, each [tokens][heads][d] in 32 bits."""
    page, d = st["page"], st["d"]
    per = page // B
    blocks = st["blocks"].view(-1, st["heads"], per, 16 * d + 128)
    # block by block: whole blocks are unpacked once
    key = seq * (st["table"].shape[1] * per) + pos // B
    some, back = torch.unique_consecutive(key, return_inverse=True)
    at = some % (st["table"].shape[1] * per)
    held = blocks[st["table"][some // (st["table"].shape[1] * per), at // per].to(torch.int64), :, at % per]
    k, v, sc = parts(held, d)
    out = []
    for t, (name, u) in enumerate((("k", k), ("v", v))):
        x = unpack(name, u, d).float().mul_(sc[..., 2 * t, None].float()).add_(sc[..., 2 * t + 1, None].float())
        out.append(x[back, :, pos % B])
    return out


def plain_read(st, typ):
    seq, pos = rows_of(st["first"], st["back"], st["back_tokens"])
    K, V = plain_values(st, seq, pos)
    return {"k": K.to(DT[typ]), "v": V.to(DT[typ])}


def plain_attend(st):
    case = st["case"]
    heads, group, d, batch = st["heads"], case["group"], st["d"], st["batch"]
    dev = st["table"].device
    out = torch.empty(st["tokens"], heads * group, d, dtype=DT[case["type"]], device=dev)
    lse = torch.empty(st["tokens"], heads * group, device=dev)
    row, where = rows_of(torch.zeros_like(st["start"]), st["cu"], st["tokens"])
    n, length = st["cu"][1:] - st["cu"][:-1], st["length"]
    # sequences padded to the longest, positions past their end on the first one and masked; as many at a time as 2 GB hold
    most = max(1, int(5e8) // (st["max_len"] * heads * (d + group * st["max_new"])))
    for b0 in range(0, batch, most):
        nb = min(most, batch - b0)
        seq = torch.arange(b0, b0 + nb, device=dev).repeat_interleave(st["max_len"])
        pos = torch.arange(st["max_len"], device=dev).repeat(nb)
        pos = torch.where(pos < length.to(torch.int64)[seq], pos, torch.zeros_like(pos))
        K, V = (x.view(nb, -1, heads, d).transpose(1, 2) for x in plain_values(st, seq, pos))
        mine = (row >= b0) & (row < b0 + nb) if nb < batch else torch.ones_like(row, dtype=torch.bool)
        r, w = row[mine] - b0, where[mine]
        q = torch.zeros(nb, st["max_new"], heads, group, d, device=dev)
        q[r, w] = st["Q"][mine].float().view(-1, heads, group, d)
        q = q.permute(0, 2, 3, 1, 4).reshape(nb, heads, group * st["max_new"], d)
        S = torch.matmul(q, K.transpose(-1, -2)).mul_(1 / math.sqrt(d)).view(nb, heads, group, st["max_new"], -1)
        p = (length - n)[b0:b0 + nb, None] + torch.arange(st["max_new"], device=dev)
        j = torch.arange(st["max_len"], device=dev)
        see = (j < length[b0:b0 + nb, None, None]).expand(-1, st["max_new"], -1)
        if case["causal"]:
            see = see & (j <= p[:, :, None])
        if case["window"]:
            see = see & (j > p[:, :, None] - case["window"])
        S.masked_fill_(~see[:, None, None], -math.inf)
        m = S.amax(-1, keepdim=True)
        S.sub_(torch.where(m > -math.inf, m, torch.zeros_like(m))).exp_()
        l = S.sum(-1, keepdim=True)
        S.div_(torch.where(l > 0, l, torch.ones_like(l)))
        O = torch.matmul(S.view(nb, heads, group * st["max_new"], -1), V).view(nb, heads, group, st["max_new"], d)
        out[mine] = O.permute(0, 3, 1, 2, 4)[r, w].reshape(-1, heads * group, d).to(out.dtype)
        lse[mine] = (m + l.log())[..., 0].permute(0, 3, 1, 2)[r, w].reshape(-1, heads * group)
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}


# ---- the work of one pass ----------------------------------------------------


def work(case):
    past, new = sizes(case)
    heads, d, size = case["heads"], case["d"], SIZE[case["type"]]
    if case["op"] == "rotate":
        rows = sum(new) * heads * (case["group"] + 1)
        return {"bytes": 2 * rows * d * size, "flops": 3.0 * rows * case["dims"]}
    token = heads * (d + 8)  # a token's codes, scales and biases
    if case["op"] == "read":
        return {"bytes": sum(new) * (token + 2 * heads * d * size), "flops": 4.0 * sum(new) * heads * d}
    if case["op"] == "write":
        back = sum(n + p % B for p, n in zip(past, new))
        return {"bytes": sum(new) * (token + 2 * heads * d * size) + back * (token + 2 * heads * d * size),
                "flops": 8.0 * sum(new) * heads * d + 4.0 * back * heads * d}
    rows = heads * case["group"]
    seen = seen_pairs = 0
    for p, n in zip(past, new):
        if not case["causal"]:
            seen, seen_pairs = seen + p + n, seen_pairs + n * (p + n)
            continue
        w = case["window"] or p + n
        seen += p + n - max(0, p - w + 1)
        # position q sees min(q + 1, w) keys
        full = max(0, min(p + n, w) - p)  # the positions below w see all before them
        seen_pairs += full * p + full * (full + 1) // 2 + (n - full) * w
    return {"bytes": seen * token + sum(new) * rows * (2 * d * size + (4 if case["lse"] else 0)), "flops": 4.0 * d * seen_pairs * rows}


# ---- in 64 bits, from the definitions -----------------------------------------


def nibbles(d):
    """For each token of a block and dim: the byte of its key code, of its value code, and their halves (0 low)."""
    t, x = torch.arange(B, device="cuda")[:, None], torch.arange(d, device="cuda")[None]
    w, i = x // 16, x % 16
    key = ((w * 8 + t % 8) * 4 + i // 4) * 4 + i % 2 * 2 + t // 8, (i // 2 % 2).expand(B, d)
    value = ((w * 8 + i % 8) * 4 + t % 8 // 2) * 4 + t % 2 * 2 + i // 8, (t // 8).expand(B, d)
    return key, value


def sequence_values(st, t, b, lo, hi):
    """float64 [heads][hi - lo][d] of one sequence's keys (t = 0) or values (t = 1), lo a multiple of the block."""
    heads, d, per = st["heads"], st["d"], st["page"] // B
    pg = st["table"][b].tolist()
    ids = torch.tensor([pg[i // per] * per + i % per for i in range(lo // B, -(-hi // B))], device="cuda")
    pool = st["blocks"].transpose(1, 2).reshape(-1, heads, 16 * d + 128)[ids].transpose(0, 1)
    byte, half = nibbles(d)[t]
    codes = pool[:, :, 8 * d * t:8 * d * (t + 1)][:, :, byte] >> (4 * half).to(torch.uint8) & 15
    sc = pool[:, :, 16 * d:].contiguous().view(torch.float16).view(heads, -1, B, 4).double()
    val = sc[..., 2 * t + 1, None] + sc[..., 2 * t, None] * codes.double()
    return val.reshape(heads, -1, d)[:, :hi - lo]


def held_vector(x):
    """What a cache holds of vectors x, float64 [..., d]: the definition of bias, scale and codes."""
    def grid(y, towards):  # to a multiple of float16's step at y
        e = torch.frexp(y)[1].double() - 1
        step = torch.exp2(e.clamp(min=-14) - 10)
        return towards(y / step) * step

    x = x.clamp(-F16_MOST, F16_MOST)
    b = grid(x.amin(-1, keepdim=True), torch.floor)
    s = grid((x.amax(-1, keepdim=True) - b) / 15, torch.ceil)
    return torch.where(s > 0, b + s * torch.round((x - b) / torch.where(s > 0, s, torch.ones_like(s))), b)


def exact(case, seed):
    st = prepare(case, seed)
    past, new = sizes(case)
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    if case["op"] == "rotate":
        return exact_rotate(st, case, past, new)
    if case["op"] == "attend":
        return exact_attend(st, case, past, new, cu)
    got = {"k": [], "v": []}
    for b, (p, n) in enumerate(zip(past, new)):
        lo = p - p % B
        for t, name in enumerate("kv"):
            val = sequence_values(st, t, b, lo, p + n).transpose(0, 1)
            if case["op"] == "write":
                val = torch.cat([val[:p - lo], held_vector(st["KV"[t]][cu[b]:cu[b + 1]].double())])
            got[name].append(val if case["op"] == "write" else val[p - lo:])
    return {name: torch.cat(v) for name, v in got.items()}


def exact_rotate(st, case, past, new):
    dims, kind, p = case["dims"], case["scaling"], SCALED[case["scaling"]]
    turn = []  # radians a position
    for i in range(dims // 2):
        f = math.exp(-2.0 * i / dims * math.log(BASE))
        if kind == "linear":
            f /= p["factor"]
        elif kind == "base" and dims > 2:
            f *= math.exp(-2.0 * i / (dims - 2) * math.log(p["factor"]))
        elif kind == "index":
            first = max(0, math.floor(dims / 2 * math.log(p["trained"] / (2 * math.pi * p["high"]), BASE)))
            end = min(dims - 1, math.ceil(dims / 2 * math.log(p["trained"] / (2 * math.pi * p["low"]), BASE)))
            share = min(1.0, max(0.0, (i - first) / max(end - first, 0.001)))
            f *= 1 - share + share / p["factor"]
        elif kind == "turns":
            share = min(1.0, max(0.0, (p["trained"] * f / (2 * math.pi) - p["low"]) / (p["high"] - p["low"])))
            f *= share + (1 - share) / p["factor"]
        turn.append(f)
    at = torch.tensor([p0 + i for p0, n in zip(past, new) for i in range(n)], dtype=torch.float64, device="cuda")
    angle = torch.outer(at, torch.tensor(turn, dtype=torch.float64, device="cuda")) * (-1 if case["back"] else 1)
    gain = 1 + 0.1 * math.log(p["factor"]) if kind == "index" else 1.0
    by = torch.polar(torch.full_like(angle, gain), angle)[:, None]
    got = {}
    for name in "QK":
        x = st[name].double()
        if case["layout"] == "half":
            z = torch.complex(x[..., :dims // 2], x[..., dims // 2:dims]) * by
            y = torch.cat([z.real, z.imag], -1)
        else:
            y = torch.view_as_real(torch.view_as_complex(x[..., :dims].reshape(*x.shape[:2], -1, 2).contiguous()) * by).flatten(-2)
        got[name.lower()] = torch.cat([y, x[..., dims:]], -1)
    return got


def exact_attend(st, case, past, new, cu):
    heads, group, d = case["heads"], case["group"], case["d"]
    outs, lses = [], []
    for b, (p, n) in enumerate(zip(past, new)):
        L = p + n
        K, V = sequence_values(st, 0, b, 0, L), sequence_values(st, 1, b, 0, L)
        pos = torch.arange(p, L, device="cuda")[:, None]
        j = torch.arange(L, device="cuda")[None]
        hidden = torch.zeros(n, L, dtype=torch.bool, device="cuda")
        if case["causal"]:
            hidden |= j > pos
        if case["window"]:
            hidden |= j <= pos - case["window"]
        o = torch.empty(n, heads * group, d, dtype=torch.float64, device="cuda")
        e = torch.empty(n, heads * group, dtype=torch.float64, device="cuda")
        for h in range(heads * group):
            q = st["Q"][cu[b]:cu[b + 1], h].double()
            S = (q @ K[h // group].T / math.sqrt(d)).masked_fill_(hidden, -math.inf)
            e[:, h] = torch.logsumexp(S, -1)
            o[:, h] = torch.exp(S - e[:, h, None]) @ V[h // group]
        outs.append(o)
        lses.append(e)
    return {"out": torch.cat(outs), "lse": torch.cat(lses)} if case["lse"] else {"out": torch.cat(outs)}

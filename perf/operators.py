"""Cases of the 8-bit key/value cache: quantising keys and values as they are
written, reading them back, and attention over the cache (single tokens, a few
tokens, prompt chunks).

A cache is a pool of pages; a page holds `page` token positions of every head in
blocks of 16 tokens, one scale a block, head and tensor (key, value).  Codes are
uint8 = value / scale + 128:
  key block    [d / 16][16 tokens][16 dims]
  value block  [d][16 tokens], token t at byte 4 ((t % 8) / 2) + 2 (t / 8) + t % 2
"""
import math
import random

import torch

own = False

B = 16  # tokens of a block
#: the byte of each token of a value block
PLACE = [4 * ((t % 8) // 2) + 2 * (t // 8) + t % 2 for t in range(B)]
DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}


def listed():
    return [
        # a decode step's new token of 32 running sequences, written and its block read back: latency counts
        dict(name="append one token", op="write", type="bf16", batch=32, heads=8, d=128, page=64, past=2000, new=1, fused=True, even=False),
        # the prompts that one scheduling step admits, out of the rows of a fused projection
        dict(name="write prompts", op="write", type="bf16", batch=12, heads=8, d=128, page=64, past=0, new=2500, fused=True, even=False),
        # further pieces of prompts that end and begin inside a block, small heads
        dict(name="write odd pieces", op="write", type="f16", batch=5, heads=4, d=64, page=16, past=701, new=900, fused=False, even=False),
        # a short sequence's keys and values in 32 bits, as an index over its keys would take them
        dict(name="read one sequence", op="read", type="f32", batch=1, heads=2, d=96, page=32, past=37, new=257, even=True),
        # long sequences moved out of the cache in 16 bits
        dict(name="read long sequences", op="read", type="bf16", batch=4, heads=8, d=128, page=64, past=0, new=32768, even=False),
        # one user's next token on a short context: latency counts
        dict(name="decode one", op="attend", type="bf16", batch=1, heads=8, group=4, d=128, page=64, past=332, new=1, causal=True, window=0, lse=False, even=True),
        # a full server's decode step, sequences of all lengths
        dict(name="decode batch", op="attend", type="bf16", batch=64, heads=8, group=4, d=128, page=64, past=8191, new=1, causal=True, window=0, lse=False, even=False),
        # one very long document, merged with other parts by its log-sum-exp
        dict(name="decode long", op="attend", type="f16", batch=1, heads=8, group=8, d=128, page=128, past=131078, new=1, causal=True, window=0, lse=True, even=True),
        # five guessed tokens checked at once, wide heads, a sliding window
        dict(name="verify in a window", op="attend", type="bf16", batch=16, heads=2, group=8, d=256, page=32, past=5000, new=5, causal=True, window=1024, lse=False, even=False),
        # a chunk of two long prompts behind what the cache holds of them
        dict(name="prompt chunk", op="attend", type="bf16", batch=2, heads=8, group=4, d=128, page=64, past=6144, new=2048, causal=True, window=0, lse=False, even=False),
        # whole prompts of a small model with ungrouped heads
        dict(name="whole prompts", op="attend", type="f16", batch=4, heads=16, group=1, d=64, page=16, past=0, new=4096, causal=True, window=0, lse=True, even=False),
        # a small 32-bit model's decode step
        dict(name="decode in 32 bits", op="attend", type="f32", batch=8, heads=12, group=1, d=64, page=16, past=1000, new=1, causal=True, window=0, lse=True, even=False),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    d = rng.choice([64, 64, 80, 96, 128, 128, 128, 192, 256])
    page = rng.choice([16, 32, 64, 128])
    heads = rng.choice([1, 2, 3, 4, 8, 8, 16])
    op = rng.choice(["write", "read", "attend", "attend", "attend", "attend"])
    if op != "attend":
        case = dict(op=op, type=rng.choice(["bf16", "bf16", "f16", "f32"]), batch=log(1, 64), heads=heads, d=d, page=page,
                    past=rng.choice([0, log(1, 4000)]), new=log(1, 8000), even=rng.random() < 0.3)
        if op == "write":
            case["fused"] = rng.random() < 0.5
        while case["batch"] * case["new"] * heads * d > 30e6:
            case["new"] = max(1, case["new"] // 2)
        return case
    kind = rng.choice(["decode", "decode", "few", "prompt"])
    group = rng.choice([1, 2, 4, 4, 6, 7, 8, 16])
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


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dev = "cuda"
    heads, d, page, typ = case["heads"], case["d"], case["page"], DT[case["type"]]
    past, new = sizes(case)
    total = [p + n for p, n in zip(past, new)]
    need = [-(-t // page) for t in total]
    cols, pages = max(need) + 1, sum(need) + 3
    order = torch.randperm(pages, generator=g, device=dev, dtype=torch.int64).to(torch.int32)
    table = torch.full((case["batch"], cols), -1, dtype=torch.int32, device=dev)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    st = dict(case=case, table=table, batch=case["batch"], heads=heads, d=d, page=page, pages=pages,
              start=torch.tensor(past, dtype=torch.int32, device=dev), length=torch.tensor(total, dtype=torch.int32, device=dev),
              cu=torch.tensor([0] + torch.tensor(new).cumsum(0).tolist(), dtype=torch.int32, device=dev),
              tokens=sum(new), max_new=max(new), max_len=max(total))
    # channels of unequal size, as keys have them
    size = torch.exp(0.5 * torch.randn(2, heads, 1, 1, d, generator=g, device=dev))
    for t, name in enumerate("kv"):
        x = torch.randn(pages, heads, page // B, B, d, generator=g, device=dev) * size[t]
        s = x.abs().amax((-1, -2)) * (1.0 / 127)
        u = ((x / s[..., None, None]).round() + 128).to(torch.uint8)
        del x
        if name == "k":
            u = u.view(pages, heads, page // B, B, d // B, B).transpose(3, 4)
        else:
            back = torch.empty(B, dtype=torch.int64)
            back[torch.tensor(PLACE)] = torch.arange(B)
            u = u[:, :, :, back.to(dev)].transpose(3, 4)
        st[name] = u.reshape(pages, heads, page // B, B * d).contiguous()
        st["s" + name] = s
    st["scales"] = torch.stack([st.pop("sk"), st.pop("sv")], -1).contiguous()
    if case["op"] == "write":
        wide = heads * (4 if case["fused"] else 0)
        rows = torch.randn(sum(new), wide + 2 * heads, d, generator=g, device=dev)
        rows[:, wide:wide + heads] *= 1.2 * size[0, :, 0, 0]
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


def run(st):
    if own:
        return run_own(st)
    case = st["case"]
    if case["op"] == "write":
        plain_write(st)
        return plain_read(st, case["type"])
    if case["op"] == "read":
        return plain_read(st, case["type"])
    return plain_attend(st)


def run_own(st):
    import paper_2608_14648_gb300 as skm

    case = st["case"]
    cache = st.get("cache")
    if cache is None:  # the handle, and attention's workspace, that a program keeps
        cache = st["cache"] = skm.KVCache(st["heads"], st["d"], st["page"], st["k"], st["v"], st["scales"])
        st["dtype"] = {"bf16": skm.DTYPE_BF16, "f16": skm.DTYPE_F16, "f32": skm.DTYPE_F32}[case["type"]]
        if case["op"] == "attend":
            st["ws"] = skm.kv_workspace(cache, st["batch"], case["heads"] * case["group"], st["tokens"], st["max_new"],
                                        st["max_len"], st["dtype"])
    if case["op"] == "attend":
        out, lse = skm.skm_kv_attend(cache, st["table"], st["length"], st["cu"], st["Q"], st["max_new"], st["max_len"],
                                     causal=case["causal"], window=case["window"], want_lse=case["lse"], ws=st["ws"])
        return {"out": out, "lse": lse} if case["lse"] else {"out": out}
    if case["op"] == "write":
        skm.skm_kv_write(cache, st["table"], st["start"], st["cu"], st["K"], st["V"], st["max_new"])
    K, V = skm.skm_kv_read(cache, st["table"], st["first"], st["back"], st["back_tokens"], st["back_max"], st["dtype"])
    return {"k": K, "v": V}


# ---- the plain forms --------------------------------------------------------


def rows_of(first, cu, tokens):
    """For each of the tokens: its sequence and its position there."""
    n = (cu[1:] - cu[:-1]).to(torch.int64)
    seq = torch.repeat_interleave(torch.arange(n.numel(), device=cu.device), n, output_size=tokens)
    return seq, torch.arange(tokens, device=cu.device) - cu[:-1].to(torch.int64)[seq] + first.to(torch.int64)[seq]


def place(device):
    return torch.tensor(PLACE, device=device)


def codes_at(st, name, page, block):
    """Codes of blocks as [blocks][heads][16 tokens][d]."""
    u = st[name][page, :, block]
    if name == "k":
        return u.view(-1, st["heads"], st["d"] // B, B, B).transpose(2, 3).reshape(-1, st["heads"], B, st["d"])
    return u.view(-1, st["heads"], st["d"], B).transpose(2, 3)[:, :, place(u.device)]


def plain_write(st):
    heads, d, page = st["heads"], st["d"], st["page"]
    start, cu = st["start"].to(torch.int64), st["cu"].to(torch.int64)
    end = start + cu[1:] - cu[:-1]
    low, high = start // B, (end + B - 1) // B
    seq = torch.repeat_interleave(torch.arange(st["batch"], device=cu.device), high - low)
    skip = torch.cumsum(high - low, 0) - (high - low)
    blk = torch.arange(seq.numel(), device=cu.device) - skip[seq] + low[seq]
    pos = blk[:, None] * B + torch.arange(B, device=cu.device)
    old, fresh = pos < start[seq][:, None], (pos >= start[seq][:, None]) & (pos < end[seq][:, None])
    src = (cu[:-1][seq][:, None] + pos - start[seq][:, None]).clamp(0, st["tokens"] - 1)
    pg, bi = st["table"][seq, blk // (page // B)].to(torch.int64), blk % (page // B)
    fresh_, old_ = fresh[:, None, :, None], old[:, None, :, None]
    for t, (name, X) in enumerate((("k", st["K"]), ("v", st["V"]))):
        x = X[src].float().transpose(1, 2)
        fine = fresh_ & torch.isfinite(x)
        a = torch.where(fine, x.abs(), torch.zeros_like(x)).amax((-1, -2))
        s_old = torch.where(old.any(1)[:, None], st["scales"][pg, :, bi, t], torch.zeros_like(a))
        s = torch.maximum(s_old, a * (1.0 / 127))
        safe = torch.where(s > 0, s, torch.ones_like(s))[..., None, None]
        was = codes_at(st, name, pg, bi)
        c_old = ((was.float() - 128) * (s_old[..., None, None] / safe)).round() + 128
        c_new = torch.nan_to_num(x / safe, nan=0.0, posinf=127.0, neginf=-127.0).round().clamp(-127, 127)
        c_new = torch.where(s[..., None, None] > 0, c_new, torch.zeros_like(c_new)) + 128
        u = torch.where(fresh_, c_new, torch.where(old_, c_old, was.float())).to(torch.uint8)
        if name == "k":
            u = u.view(-1, heads, B, d // B, B).transpose(2, 3)
        else:
            u = u[:, :, torch.argsort(place(u.device))].transpose(2, 3)
        st[name][pg, :, bi] = u.reshape(-1, heads, B * d)
        st["scales"][pg, :, bi, t] = s


def plain_values(st, name, seq, pos):
    """Values of tokens at positions pos of sequences seq as [tokens][heads][d], 32 bits."""
    page = st["table"][seq, pos // st["page"]].to(torch.int64)
    block, tok = pos % st["page"] // B, pos % B
    heads, d = st["heads"], st["d"]
    if name == "k":
        u = st["k"].view(-1, heads, st["page"] // B, d // B, B, B)[page, :, block, :, tok].reshape(-1, heads, d)
    else:
        u = st["v"].view(-1, heads, st["page"] // B, d, B)[page, :, block, :, place(pos.device)[tok]]
    return (u.float() - 128) * st["scales"][page, :, block, 0 if name == "k" else 1][..., None]


def plain_read(st, typ):
    seq, pos = rows_of(st["first"], st["back"], st["back_tokens"])
    return {name: plain_values(st, name, seq, pos).to(DT[typ]) for name in "kv"}


def plain_attend(st):
    case = st["case"]
    heads, group, d, batch = st["heads"], case["group"], st["d"], st["batch"]
    dev = st["table"].device
    n, length = st["cu"][1:] - st["cu"][:-1], st["length"]
    # every sequence padded to the longest, positions past its end on some valid page and masked
    seq = torch.arange(batch, device=dev).repeat_interleave(st["max_len"])
    pos = torch.arange(st["max_len"], device=dev).repeat(batch)
    there = pos < length.to(torch.int64)[seq]
    pos_ = torch.where(there, pos, torch.zeros_like(pos))
    K, V = (plain_values(st, name, seq, pos_).view(batch, -1, heads, d).transpose(1, 2) for name in "kv")
    row, where = rows_of(torch.zeros_like(st["start"]), st["cu"], st["tokens"])
    q = torch.zeros(batch, st["max_new"], heads, group, d, device=dev)
    q[row, where] = st["Q"].float().view(-1, heads, group, d)
    q = q.permute(0, 2, 3, 1, 4).reshape(batch, heads, group * st["max_new"], d)
    S = torch.matmul(q, K.transpose(-1, -2)).mul_(1 / math.sqrt(d)).view(batch, heads, group, st["max_new"], -1)
    p = (length - n)[:, None] + torch.arange(st["max_new"], device=dev)
    j = torch.arange(st["max_len"], device=dev)
    see = (j < length[:, None, None]).expand(-1, st["max_new"], -1)
    if case["causal"]:
        see = see & (j <= p[:, :, None])
    if case["window"]:
        see = see & (j > p[:, :, None] - case["window"])
    S.masked_fill_(~see[:, None, None], -math.inf)
    m = S.amax(-1, keepdim=True)
    S.sub_(torch.where(m > -math.inf, m, torch.zeros_like(m))).exp_()
    l = S.sum(-1, keepdim=True)
    S.div_(torch.where(l > 0, l, torch.ones_like(l)))
    O = torch.matmul(S.view(batch, heads, group * st["max_new"], -1), V).view(batch, heads, group, st["max_new"], d)
    out = {"out": O.permute(0, 3, 1, 2, 4)[row, where].reshape(-1, heads * group, d).to(DT[case["type"]])}
    if case["lse"]:
        out["lse"] = (m + l.log())[..., 0].permute(0, 3, 1, 2)[row, where].reshape(-1, heads * group)
    return out


# ---- the work of one pass ----------------------------------------------------


def work(case):
    past, new = sizes(case)
    heads, d, size = case["heads"], case["d"], SIZE[case["type"]]
    token = 2 * heads * d + 2 * heads * 4 / B  # a token's codes and its part of the scales
    if case["op"] == "read":
        return {"bytes": sum(new) * (token + 2 * heads * d * size), "flops": 2.0 * sum(new) * heads * d}
    if case["op"] == "write":
        back = sum(n + p % B for p, n in zip(past, new))
        return {"bytes": sum(new) * (token + 2 * heads * d * size) + back * (token + 2 * heads * d * size),
                "flops": 6.0 * sum(new) * heads * d + 2.0 * back * heads * d}
    rows = heads * case["group"]
    seen = pairs = 0
    for p, n in zip(past, new):
        if not case["causal"]:
            seen, pairs = seen + p + n, pairs + n * (p + n)
            continue
        w = case["window"] or p + n
        seen += p + n - max(0, p - w + 1)
        # position q sees min(q + 1, w) keys
        full = max(0, min(p + n, w) - p)  # the positions below w see all before them
        pairs += full * p + full * (full + 1) // 2 + (n - full) * w
    return {"bytes": seen * token + sum(new) * rows * (2 * d * size + (4 if case["lse"] else 0)), "flops": 4.0 * d * pairs * rows}


# ---- in 64 bits, from the definitions -----------------------------------------


def token_codes(st, name, page, slot):
    """[heads][d] codes of the token at a slot of a page."""
    heads, d = st["heads"], st["d"]
    blk, t = slot // B, slot % B
    raw = st[name][page, :, blk]
    if name == "k":
        return raw.view(heads, d // B, B, B)[:, :, t].reshape(heads, d)
    return raw.view(heads, d, B)[:, :, PLACE[t]]


def sequence_values(st, name, b, lo, hi):
    """float64 [heads][hi - lo][d] of one sequence, lo a multiple of the block."""
    heads, d, page = st["heads"], st["d"], st["page"]
    per = page // B
    blocks = range(lo // B, -(-hi // B))
    pg = st["table"][b].tolist()
    ids = torch.tensor([pg[i // per] * per + i % per for i in blocks], device="cuda")
    pool = st[name].permute(0, 2, 1, 3).reshape(-1, heads, B * d)[ids]
    sc = st["scales"][..., 0 if name == "k" else 1].permute(0, 2, 1).reshape(-1, heads)[ids].double()
    if name == "k":
        val = pool.view(-1, heads, d // B, B, B).permute(0, 1, 3, 2, 4).reshape(-1, heads, B, d)
    else:
        val = torch.stack([pool.view(-1, heads, d, B)[..., PLACE[t]] for t in range(B)], 2)
    val = (val.double() - 128.0) * sc[:, :, None, None]
    return val.permute(1, 0, 2, 3).reshape(heads, -1, d)[:, lo - blocks[0] * B:hi - blocks[0] * B]


def exact(case, seed):
    st = prepare(case, seed)
    past, new = sizes(case)
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    if case["op"] == "attend":
        return exact_attend(st, case, past, new, cu)
    if case["op"] == "read":
        got = {}
        for name in "kv":
            got[name] = torch.cat([sequence_values(st, name, b, p - p % B, p + n)[:, p % B:].transpose(0, 1)
                                   for b, (p, n) in enumerate(zip(past, new))])
        return got
    got = {"k": [], "v": []}
    third = torch.tensor(1.0 / 127, dtype=torch.float32, device="cuda")
    for b, (p, n) in enumerate(zip(past, new)):
        lo, held = p - p % B, p % B
        full = -(-(p + n) // B) * B
        for t, name in enumerate("kv"):
            X = st["K" if name == "k" else "V"][cu[b]:cu[b + 1]].double()
            # the blocks as [blocks][16][heads][d], with what is new and what was there
            x = torch.zeros(full - lo, st["heads"], st["d"], dtype=torch.float64, device="cuda")
            x[held:held + n] = X
            x = x.view(-1, B, st["heads"], st["d"])
            s = (x.abs().amax((1, 3)).float() * third).double()  # a scale is held in 32 bits
            if held:
                pg, blk = int(st["table"][b, lo // case["page"]]), lo % case["page"] // B
                was = st["scales"][pg, :, blk, t].double()
                s[0] = torch.maximum(s[0], was)
            val = torch.round(x / s[:, None, :, None]).clamp(-127, 127) * s[:, None, :, None]
            val = val.reshape(-1, st["heads"], st["d"])
            for i in range(held):
                c = token_codes(st, name, pg, lo % case["page"] + i).double() - 128
                val[i] = torch.round(c * (was / s[0])[:, None]) * s[0][:, None]
            got[name].append(val[:held + n])
    return {name: torch.cat(v) for name, v in got.items()}


def exact_attend(st, case, past, new, cu):
    heads, group, d = case["heads"], case["group"], case["d"]
    outs, lses = [], []
    for b, (p, n) in enumerate(zip(past, new)):
        L = p + n
        K, V = sequence_values(st, "k", b, 0, L), sequence_values(st, "v", b, 0, L)
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

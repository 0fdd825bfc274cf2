"""The 4-bit key/value cache on the GPU against plain implementations.

Codes, scales and biases are compared for equality with their definition (numpy, 64 bits).
Attention is compared with the definition in 64 bits over the values that the cache
really holds, elementwise within

  u |ref| + (w + 2 e) A + n 2^-28 M,

u the rounding of the output type (2^-8 bf16, 2^-11 f16, 2^-24 f32), A = sum_j p_j (|b_j| + s_j (c_j + 16)) (codes less 8 and
values at code 8, or codes and biases, are summed apart: s |c - 8| + |b + 8 s| at most), M the largest |b| + 15 s; w the relative error of a weight
and of the sums that carry it (f16 weights: 2^-11 and fp32 sums that tensor cores may truncate, n 2^-23; the value scales'
approximate logarithm and reciprocal, 2^-20; f32: n + 16 roundings of 2^-24), e the error of a logit: fp32 products of d terms in
any order, (d + 16) 2^-23 scale sum |q| (|b| + s (c + 16)), plus 2^-22 |logit| for the base-2 form.  The last term covers weights that
underflow in f16: of half a block's tokens the weight is held divided by 16, so it is off by at most 2^-21 (half of f16's smallest
step, 2^-25, times 16), its code at most 15, and the row's largest weight times scale at least 2^7.  The kernel for many rows takes
values as f16 at worst: with `rounded`, 2^-11 of a value's size (2^-25 where it is subnormal) on top; and for bf16 outputs without lse keys
too: their logits are off by up to scale sum |q| (2^-11 |k| + 2^-25) more.  lse: e and
2^-22 of its size, and the sums' error w without the f16 weights' 2^-11 (sums are of the weights in fp32)."""
import math

import numpy as np
import pytest
import torch
from test_gpu_kv import ATTENDS, DT, WRITES, i32, make_table

pytestmark = pytest.mark.gpu

B = 16


def places(d):
    """For each token of a block and dim: the byte of its key code and of its value code, and whether it is the high half."""
    t, x = np.arange(B)[:, None], np.arange(d)[None]
    w, i = x // 16, x % 16
    key = 128 * w + 16 * (t % 8) + 4 * (i // 4) + 2 * (i % 2) + t // 8, np.broadcast_to(i // 2 % 2, (B, d))
    value = 8 * d + 128 * w + 16 * (i % 8) + 4 * (t // 2 % 4) + 2 * (t % 2) + i // 8, np.broadcast_to(t // 8, (B, d))
    return key, value


def vectors(x):
    """(scale, bias, codes) of vectors x [..., d] by the definition; float16, float16, int64."""
    x = x.astype(np.float64)
    fine = np.isfinite(x)
    lo = np.where(fine, x, np.inf).min(-1)
    hi = np.where(fine, x, -np.inf).max(-1)
    none = ~fine.any(-1)
    lo, hi = (np.where(none, 0.0, v).clip(-65504, 65504) for v in (lo, hi))
    down, up = np.float16(-np.inf), np.float16(np.inf)
    b = lo.astype(np.float16)
    b = np.where(b.astype(np.float64) > lo, np.nextafter(b, down), b)
    s = ((hi - b) / 15).astype(np.float16)
    enough = lambda s: b.astype(np.float64) + 15 * s.astype(np.float64) >= hi  # noqa: E731
    for _ in range(3):
        s = np.where(enough(s), s, np.nextafter(s, up))
    for _ in range(3):
        less = np.nextafter(s, down)
        s = np.where((s > 0) & enough(less), less, s)
    y = np.where(np.isnan(x), lo[..., None], np.clip(x, lo[..., None], hi[..., None]))
    step = np.where(s > 0, s, 1).astype(np.float64)[..., None]
    c = np.rint((y - b.astype(np.float64)[..., None]) / step)
    return s, b, np.where((s > 0)[..., None], c, 0).astype(np.int64)


class Held4:
    """What a cache holds, by the definition: codes [tensor][pages, heads, page, d], scales [pages, heads, page, 4]."""

    def __init__(self, c):
        self.page, self.heads, self.d, self.pages = c.page, c.heads, c.d, c.pages
        raw = c.blocks.cpu().numpy()
        self.code = []
        for byte, high in places(c.d):
            u = raw[..., byte] >> (4 * high).astype(np.uint8) & 15
            self.code.append(u.reshape(c.pages, c.heads, c.page, c.d).astype(np.int64))
        self.scale = raw[..., 16 * c.d:].copy().view(np.float16).reshape(c.pages, c.heads, c.page, 4)

    def write(self, table, start, cu, K, V):
        for b in range(table.shape[0]):
            for r in range(cu[b], cu[b + 1]):
                p = start[b] + r - cu[b]
                pg = int(table[b, p // self.page]) if p // self.page < table.shape[1] else -1
                if not 0 <= pg < self.pages:
                    continue
                for t, X in enumerate((K, V)):
                    s, bias, c = vectors(X[r].float().numpy())
                    self.code[t][pg, :, p % self.page] = c
                    self.scale[pg, :, p % self.page, 2 * t] = s
                    self.scale[pg, :, p % self.page, 2 * t + 1] = bias

    def values(self, t, table, b, lo, hi):
        """float64 values [hi - lo, heads, d] of keys (0) or values (1), zeros where the page is absent; |b| + s (c + 16); s; which are there."""
        val = np.zeros((hi - lo, self.heads, self.d))
        size, step = np.zeros_like(val), np.zeros((hi - lo, self.heads))
        there = np.zeros(hi - lo, bool)
        for p in range(lo // self.page, -(-hi // self.page)):
            pg = int(table[b, p]) if p < table.shape[1] else -1
            if not 0 <= pg < self.pages:
                continue
            a, z = max(lo, p * self.page), min(hi, (p + 1) * self.page)
            at, to = slice(a - p * self.page, z - p * self.page), slice(a - lo, z - lo)
            s, o = (self.scale[pg, :, at, 2 * t + i].astype(np.float64).T[..., None] for i in (0, 1))
            c = self.code[t][pg, :, at].transpose(1, 0, 2)
            val[to], size[to], step[to], there[to] = o + s * c, abs(o) + s * (c + 16), s[..., 0], True
        return (torch.from_numpy(x) for x in (val, size, step, there))

    def read(self, t, table, b, lo, hi):
        """As skm_kv4_read: b + s code rounded to fp32."""
        return next(self.values(t, table, b, lo, hi)).float()


def make_cache(heads, d, page, pages, seed=0):
    """A cache of random codes, scales and biases."""
    import paper_2608_14648_gb300 as skm

    c = skm.KVCache4(heads, d, page, pages=pages)
    g = torch.Generator().manual_seed(seed)
    c.blocks.copy_(torch.randint(0, 256, c.blocks.shape, generator=g, dtype=torch.int64).to(torch.uint8))
    sc = scales(c)
    draw = torch.rand(sc.shape, generator=g)
    sc[..., 0::2] = (0.05 + 0.3 * draw[..., 0::2]).to(torch.float16).cuda()
    sc[..., 1::2] = (-4 * draw[..., 1::2]).to(torch.float16).cuda()
    return c


def scales(c):
    """A view [pages, heads, page / 16, 16, 4] of a cache's scales and biases."""
    v = c.blocks.view(torch.float16)
    return v[..., 8 * c.d:].unflatten(-1, (16, 4))


def same(c, want):
    got = Held4(c)
    for t in range(2):
        assert np.array_equal(got.code[t], want.code[t])
    assert np.array_equal(got.scale.view(np.uint16), want.scale.view(np.uint16))


# ---- writing and reading back


def write_case(heads, d, page, typ, seqs, fused, seed=3, spoil=None):
    import paper_2608_14648_gb300 as skm

    cols = max(-(-(s + n) // page) for s, n in seqs) + 1
    pages = len(seqs) * cols + 2
    c = make_cache(heads, d, page, pages, seed)
    table = make_table(len(seqs), cols, pages, seed)
    start, cu = [s for s, _ in seqs], [0]
    for _, n in seqs:
        cu.append(cu[-1] + n)
    g = torch.Generator().manual_seed(seed + 1)
    rows = torch.randn(cu[-1], heads * 3, d, generator=g) * torch.exp(torch.randn(cu[-1], heads * 3, 1, generator=g))
    rows = (rows + 2 * torch.randn(cu[-1], heads * 3, 1, generator=g)).to(DT[typ])
    if spoil:
        spoil(rows)
    dev = rows.cuda()
    K, V = (dev[:, :heads], dev[:, 2 * heads:]) if fused else (dev[:, :heads].contiguous(), dev[:, 2 * heads:].contiguous())
    want = Held4(c)
    want.write(table, start, cu, rows[:, :heads], rows[:, 2 * heads:])
    most = max(n for _, n in seqs)
    skm.skm_kv4_write(c, table.cuda(), i32(start), i32(cu), K, V, most)
    torch.cuda.synchronize()
    return c, table, start, cu, want, most


@pytest.mark.parametrize("heads,d,page,typ,seqs", WRITES)
@pytest.mark.parametrize("fused", [False, True])
def test_write_and_read_back(cuda_ok, heads, d, page, typ, seqs, fused):
    import paper_2608_14648_gb300 as skm

    c, table, start, cu, want, most = write_case(heads, d, page, typ, seqs, fused)
    same(c, want)
    for dt, code in ((torch.float32, skm.DTYPE_F32), (torch.bfloat16, skm.DTYPE_BF16), (torch.float16, skm.DTYPE_F16)):
        got = skm.skm_kv4_read(c, table.cuda(), i32(start), i32(cu), cu[-1], most, code)
        for t in range(2):
            ref = torch.cat([want.read(t, table, b, s, s + n) for b, (s, n) in enumerate(seqs)])
            assert torch.equal(got[t].cpu(), ref.to(dt))


@pytest.mark.parametrize("heads,d,page,typ", [(8, 128, 64, "bf16"), (3, 96, 32, "f16"), (2, 256, 16, "f32"), (5, 16, 16, "bf16")])
def test_write_and_read_large_batches(cuda_ok, heads, d, page, typ):
    """More than 32 sequences: their blocks are placed in rows of the longest's, one or none reached by the others."""
    import paper_2608_14648_gb300 as skm

    seqs = [(i * 13 % 50, (i * 29 % 71) * (i % 5 > 0)) for i in range(45)] + [(15, 1), (16, 200), (31, 2)]
    c, table, start, cu, want, most = write_case(heads, d, page, typ, seqs, fused=True)
    same(c, want)
    got = skm.skm_kv4_read(c, table.cuda(), i32(start), i32(cu), cu[-1], most, skm.DTYPE_F32)
    for t in range(2):
        assert torch.equal(got[t].cpu(), torch.cat([want.read(t, table, b, s, s + n) for b, (s, n) in enumerate(seqs)]))


@pytest.mark.parametrize("typ", ["bf16", "f16", "f32"])
def test_values_read_back_are_within_half_a_scale(cuda_ok, typ):
    """... of what was written, and the scale within the bound that the header states."""
    import paper_2608_14648_gb300 as skm

    c = make_cache(2, 96, 16, 12, 1)
    table = make_table(1, 12, 12, 1).cuda()
    g = torch.Generator().manual_seed(2)
    x = torch.randn(190, 4, 96, generator=g) * 10.0 ** (6 * torch.rand(190, 4, 1, generator=g) - 4)
    x = (x + 3 * x[..., :1]).to(DT[typ])
    dev = x.cuda()
    skm.skm_kv4_write(c, table, i32([0]), i32([0, 190]), dev[:, :2], dev[:, 2:], 190)
    held, where = Held4(c), table.cpu()
    for t, X in ((0, x[:, :2].double()), (1, x[:, 2:].double())):
        val, _, s, _ = held.values(t, where, 0, 0, 190)
        assert ((val - X).abs().amax(-1) <= s / 2 * (1 + 2.0**-40)).all()
        lo, hi = X.amin(-1), X.amax(-1)
        assert (s <= (hi - lo + 2.0**-10 * lo.abs() + 2.0**-24) * (1 + 2.0**-10) / 15 + 2.0**-24).all()


def test_write_leaves_infinities_and_nan_out(cuda_ok):
    def spoil(rows):
        rows[0, 0, 3] = math.inf
        rows[1, 0, 5] = -math.inf
        rows[2, 4, 7] = math.nan
        rows[3:9, :, :] = 0
        rows[9, :, 1:] = math.nan  # one finite element
        rows[10] = math.inf  # none
        rows[20:36] = math.nan  # nor a whole block's

    for typ in ("bf16", "f16", "f32"):
        c, *_, want, _ = write_case(2, 64, 16, typ, [(0, 20), (0, 16), (3, 40)], True, spoil=spoil)
        same(c, want)


@pytest.mark.parametrize("typ", ["bf16", "f32"])
def test_write_of_values_at_the_ends_of_the_range(cuda_ok, typ):
    """Beyond f16: clipped; within its smallest step; around a mean far larger than their spread."""
    def spoil(rows):
        rows[:8] *= 1e6
        rows[8:12] *= 1e38
        rows[12:16] = 65504.0
        rows[16:24] *= 1e-9
        rows[24:30] *= 1e-42
        rows[30:40] = 1000 + rows[30:40] * 0.01
        rows[40:50] = -30000 + rows[40:50]

    for d in (64, 144):
        c, *_, want, _ = write_case(2, d, 16, typ, [(0, 50), (5, 10)], False, spoil=spoil)
        same(c, want)


@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
def test_write_rounds_as_in_exact_arithmetic(cuda_ok, typ):
    """Elements at and next to the middles of two codes: a few units in the last place to either side."""
    import paper_2608_14648_gb300 as skm

    g = torch.Generator().manual_seed(7)
    n, d = 960, 256
    c = make_cache(1, d, 16, n // 16)
    table = torch.arange(n // 16, dtype=torch.int32).view(1, -1)
    b = torch.randn(n, generator=g).half().float() * (torch.arange(n) % 3)  # a third around 0
    s = (0.001 + torch.rand(n, generator=g) * 2.0 ** torch.randint(-8, 4, (n,), generator=g)).half().float()
    s[:100] = 2.0 ** torch.randint(-8, 4, (100,), generator=g)  # exact middles
    x = b[:, None] + s[:, None] * (torch.randint(0, 15, (n, d), generator=g) + 0.5)
    if typ == "f32":
        x = (x.view(torch.int32) + torch.randint(-3, 4, x.shape, generator=g, dtype=torch.int32)).view(torch.float32)
    x[:, 0], x[:, 1] = b, b + 15 * s
    K = x.to(DT[typ]).view(n, 1, d)
    V = K.flip(2)
    want = Held4(c)
    want.write(table, [0], [0, n], K, V)
    skm.skm_kv4_write(c, table.cuda(), i32([0]), i32([0, n]), K.cuda(), V.cuda(), n)
    same(c, want)


def test_write_token_by_token_is_writing_at_once(cuda_ok):
    import paper_2608_14648_gb300 as skm

    x = torch.randn(40, 4, 80, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).cuda()
    one, all_ = make_cache(2, 80, 32, 5, 1), make_cache(2, 80, 32, 5, 1)
    table = make_table(1, 3, 5, 1).cuda()
    for t in range(40):
        skm.skm_kv4_write(one, table, i32([t + 3]), i32([0, 1]), x[t:t + 1, :2], x[t:t + 1, 2:], 1)
    skm.skm_kv4_write(all_, table, i32([3]), i32([0, 40]), x[:, :2], x[:, 2:], 40)
    assert torch.equal(one.blocks, all_.blocks)


def test_write_unaligned_rows(cuda_ok):
    import paper_2608_14648_gb300 as skm

    heads, d = 2, 48
    for typ in ("f16", "f32"):
        c = make_cache(heads, d, 16, 6, 4)
        table = make_table(1, 5, 6, 4)
        want = Held4(c)
        flat = torch.randn(1 + 33 * 101 * 3, generator=torch.Generator().manual_seed(5)).to(DT[typ])
        view = lambda x: (x[1:].as_strided((33, heads, d), (301, 101, 1)),  # noqa: E731
                          x[1:].as_strided((33, heads, d), (299, 53, 1)))
        want.write(table, [9], [0, 33], *view(flat))
        skm.skm_kv4_write(c, table.cuda(), i32([9]), i32([0, 33]), *view(flat.cuda()), 33)
        same(c, want)


def test_absent_pages_and_the_tables_end(cuda_ok):
    import paper_2608_14648_gb300 as skm

    c = make_cache(1, 32, 16, 4, 6)
    table = torch.tensor([[2, -1, 9, 0]], dtype=torch.int32)  # 9: not a page of the pool
    want = Held4(c)
    x = torch.randn(70, 2, 32, generator=torch.Generator().manual_seed(7)).to(torch.bfloat16)
    want.write(table, [3], [0, 70], x[:, :1], x[:, 1:])  # the table ends at 64
    dev = x.cuda()
    skm.skm_kv4_write(c, table.cuda(), i32([3]), i32([0, 70]), dev[:, :1], dev[:, 1:], 70)
    same(c, want)
    got = skm.skm_kv4_read(c, table.cuda(), i32([0]), i32([0, 80]), 80, 80, skm.DTYPE_F32)
    for t in range(2):
        assert torch.equal(got[t].cpu(), want.read(t, table, 0, 0, 80))


def test_read_one_of_the_two(cuda_ok):
    import paper_2608_14648_gb300 as skm

    c = make_cache(2, 64, 32, 4, 8)
    table = make_table(1, 4, 4, 8)
    out = torch.full((21, 2, 64), 7.0, device="cuda")
    skm.skm_kv4_read(c, table.cuda(), i32([5]), i32([0, 21]), 21, 21, skm.DTYPE_F32, out=(None, out))
    assert torch.equal(out.cpu(), Held4(c).read(1, table, 0, 5, 26))


def test_write_of_a_sequence_without_rows_touches_nothing(cuda_ok):
    # 40 sequences: the even ones have no rows, and table rows that name pages of the odd ones
    import paper_2608_14648_gb300 as skm

    g = torch.Generator().manual_seed(5)
    for _ in range(5):
        c = make_cache(2, 64, 16, 40)
        table = torch.arange(40, dtype=torch.int32).view(40, 1)
        table[0::2] = table[1::2]
        n = [b % 2 * 3 for b in range(40)]
        cu = [0] + torch.tensor(n).cumsum(0).tolist()
        start = [5 + b % 7 for b in range(40)]
        K, V = torch.randn(2, cu[-1], 2, 64, generator=g)
        want = Held4(c)
        want.write(table, start, cu, K, V)
        skm.skm_kv4_write(c, table.cuda(), i32(start), i32(cu), K.cuda(), V.cuda(), 3)
        same(c, want)


@pytest.mark.parametrize("start", [64, 80, 2**31 - 1, 2**31 - 40, -2**31])
def test_write_beyond_the_table(cuda_ok, start):
    # nothing at or past cols * page = 64; a negative position counts as 0
    import paper_2608_14648_gb300 as skm

    c = make_cache(1, 32, 32, 3)
    want = Held4(c)
    table = torch.tensor([[2, 0]], dtype=torch.int32)
    K, V = torch.randn(2, 100, 1, 32, generator=torch.Generator().manual_seed(6))
    if start < 0:
        want.write(table, [0], [0, 100], K, V)
    skm.skm_kv4_write(c, table.cuda(), i32([start]), i32([0, 100]), K.cuda(), V.cuda(), 100)
    same(c, want)


def test_write_and_read_no_rows(cuda_ok):
    import paper_2608_14648_gb300 as skm

    c = make_cache(2, 64, 16, 2, 1)
    table, pos, cu = i32([[0, 1]]), i32([20]), i32([0, 0])
    skm.skm_kv4_write(c, table, pos, cu, *torch.empty(2, 0, 2, 64, device="cuda"), 0)
    K, V = skm.skm_kv4_read(c, table, pos, cu, 0, 0)
    assert K.shape == V.shape == (0, 2, 64)


# ---- attention


def attend_ref(held, table, length, cu, Q, group, scale, causal, window, typ, rounded):
    """(out, lse, tolerance of out, tolerance of lse, tolerance of out with rounded keys) in 64 bits."""
    heads, d = held.heads, held.d
    T = Q.shape[0]
    out = torch.zeros(T, heads * group, d, dtype=torch.float64)
    lse = torch.full((T, heads * group), -math.inf, dtype=torch.float64)
    tol, ltol, ktol = torch.zeros_like(out), torch.zeros_like(lse), torch.zeros_like(out)
    u = {"bf16": 2.0**-8, "f16": 2.0**-11, "f32": 2.0**-24}[typ]
    for b in range(table.shape[0]):
        n, L = cu[b + 1] - cu[b], length[b]
        if n == 0 or L == 0:
            continue
        K, K_size, _, there = held.values(0, table, b, 0, L)
        V, V_size, V_step, _ = held.values(1, table, b, 0, L)
        p = torch.arange(L - n, L)[:, None]
        j = torch.arange(L)[None]
        see = there[None].expand(n, L).clone()
        if causal:
            see &= j <= p
        if window:
            see &= j > p - window
        any_ = see.any(1)
        for h in range(heads * group):
            q, kv = Q[cu[b]:cu[b + 1], h].double(), h // group
            S = (q @ K[:, kv].T * scale).masked_fill(~see, -math.inf)
            most = lambda k: (abs(scale) * (q.abs() @ k.T)).masked_fill(~see, 0).amax(1)  # noqa: E731
            big = S.abs().masked_fill(~see, 0).amax(1)
            e = (d + 16) * 2.0**-23 * most(K_size[:, kv]) + 2.0**-22 * big
            l = torch.logsumexp(S, 1)
            w = torch.where(any_[:, None], torch.exp(S - l[:, None]), torch.zeros((), dtype=torch.float64)).nan_to_num()
            o, A = w @ V[:, kv], w @ V_size[:, kv]
            sums = L * 2.0**-23 + (16 * 2.0**-24 if typ == "f32" else 2.0**-20)
            sl = slice(cu[b], cu[b + 1])
            out[sl, h], lse[sl, h] = o, l
            tol[sl, h] = (u * o.abs() + ((0.0 if typ == "f32" else 2.0**-11) + sums + 2 * e)[:, None] * A * 1.01
                          + L * 2.0**-28 * (V_size[:, kv].amax() + 15 * V_step[:, kv].amax()))
            if rounded:
                tol[sl, h] += 2.0**-11 * (w @ V[:, kv].abs()) + 2.0**-25
                # exp(2 e) - 1, as these logits are off by more
                ktol[sl, h] = tol[sl, h] + torch.expm1(2 * most(2.0**-11 * K[:, kv].abs() + 2.0**-25))[:, None] * A * 1.01
            ltol[sl, h] = e + sums + 2.0**-22 * l.abs().nan_to_num(posinf=0)
    return out, lse, tol, ltol, ktol


def check_attend(heads, group, d, page, typ, seqs, causal=True, window=0, absent=0.0, scale=None, seed=11, spread=1.0,
                 strided=False, max_len=None, max_tokens=None, spoil=None):
    """seqs: (tokens held before, query rows) of each sequence."""
    import paper_2608_14648_gb300 as skm

    length = [max(p + n, 0) for p, n in seqs]
    cols = max(-(-t // page) for t in length) + 1
    pages = len(seqs) * cols + 1
    c = make_cache(heads, d, page, pages, seed)
    table = make_table(len(seqs), cols, pages, seed)
    g = torch.Generator().manual_seed(seed + 1)
    if spoil:
        spoil(c)
    if absent:
        gone = torch.rand(table.shape, generator=g) < absent
        table = torch.where(gone, torch.full_like(table, -1), table)
    # what was never written: NaN scales and biases past each sequence's end
    held, sc = Held4(c), scales(c)
    for b, L in enumerate(length):
        for p in range(L, cols * page):
            pg = int(table[b, p // page])
            if pg >= 0:
                sc[pg, :, p % page // B, p % B] = math.nan
    cu = [0]
    for _, n in seqs:
        cu.append(cu[-1] + n)
    Q = (spread * torch.randn(cu[-1], heads * group, d, generator=g)).to(DT[typ])
    dev = Q.cuda()
    if strided:
        wide = torch.zeros(cu[-1], heads * group + 3, d + 5, dtype=Q.dtype, device="cuda")
        wide[:, 2: 2 + heads * group, 1: 1 + d] = dev
        dev = wide[:, 2: 2 + heads * group, 1: 1 + d]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got, lse = skm.skm_kv4_attend(c, table.cuda(), i32(length), i32(cu), dev, max_tokens or max(n for _, n in seqs),
                                  max(length) if max_len is None else max_len, scale=scale, causal=causal, window=window,
                                  want_lse=True, status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    rounded = typ != "f32" and (max_tokens or max(n for _, n in seqs)) * group > 32
    out, ref, tol, ltol, ktol = attend_ref(held, table, length, cu, Q, group, d**-0.5 if scale is None else scale, causal, window, typ, rounded)
    got, lse = got.cpu().double(), lse.cpu().double()
    assert torch.equal(torch.isneginf(lse), torch.isneginf(ref))
    fine = ~torch.isneginf(ref)
    assert torch.isfinite(got).all() and torch.isfinite(lse[fine]).all()
    assert (got[~fine] == 0).all()
    over = ((got - out).abs() - tol).amax() if got.numel() else 0.0
    assert over <= 0, f"out is off by {float((got - out).abs().max()):.3g}, over the bound by {float(over):.3g}"
    if fine.any():
        assert ((lse - ref).abs() - ltol)[fine].amax() <= 0
    if rounded and typ == "bf16":  # without log-sum-exps keys may be rounded as well
        alone, _ = skm.skm_kv4_attend(c, table.cuda(), i32(length), i32(cu), dev, max_tokens or max(n for _, n in seqs),
                                      max(length) if max_len is None else max_len, scale=scale, causal=causal, window=window, status=status)
        alone = alone.cpu().double()
        assert int(status) == 0 and torch.isfinite(alone).all() and (alone[~fine] == 0).all()
        assert ((alone - out).abs() - ktol).amax() <= 0
    return got


@pytest.mark.parametrize("heads,group,d,page,typ,seqs", ATTENDS)
@pytest.mark.parametrize("kind", ["causal", "all", "window"])
def test_attend(cuda_ok, heads, group, d, page, typ, seqs, kind):
    check_attend(heads, group, d, page, typ, seqs, causal=kind != "all", window=37 if kind == "window" else 0)


@pytest.mark.parametrize("typ,group,new", [("bf16", 4, 1), ("f32", 1, 1), ("f16", 8, 4), ("bf16", 4, 80)])
def test_attend_with_pages_gone(cuda_ok, typ, group, new):
    check_attend(2, group, 64, 16, typ, [(300, new), (40, new), (5, new)], absent=0.4)
    check_attend(2, group, 64, 16, typ, [(300, new), (40, new)], absent=1.0)


@pytest.mark.parametrize("typ", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 5, 100])
def test_attend_rows_that_see_nothing(cuda_ok, typ, new):
    """No tokens at all, and more rows than tokens (the first rows stand before position 0)."""
    check_attend(2, 2, 64, 16, typ, [(-new, new), (20, new), (-new + 1, new), (-(new // 2) - 1, new)])


@pytest.mark.parametrize("typ,group", [("bf16", 4), ("f16", 16), ("f32", 2)])
def test_attend_split_over_the_whole_gpu(cuda_ok, typ, group):
    """Few long sequences: units cut between warps and CTAs, next to short and empty ones."""
    check_attend(2, group, 64, 64, typ, [(9000, 1), (0, 1), (-1, 1), (17, 1), (5111, 1)])
    check_attend(1, group, 128, 32, typ, [(20011, 1)])


def test_attend_many_sequences(cuda_ok):
    """More sequences than one launch lines up."""
    check_attend(1, 2, 32, 16, "bf16", [(i * 37 % 90, i % 3) for i in range(1100)])


@pytest.mark.parametrize("d,new,typ", [(128, 20, "bf16"), (96, 32, "f16"), (256, 12, "bf16"), (192, 30, "f16")])
def test_attend_large_batches_of_many_rows(cuda_ok, d, new, typ):
    """1024 sequences take more shared memory beside a large tile than a CTA has: several launches."""
    check_attend(1, 1, d, 16, typ, [(i % 23, new - i % 3) for i in range(1024)])


@pytest.mark.parametrize("typ,new", [("bf16", 1), ("f16", 150), ("f32", 2)])
def test_attend_strides_and_alignment(cuda_ok, typ, new):
    check_attend(2, 3, 64, 16, typ, [(50, new), (0, new)], strided=True)


@pytest.mark.parametrize("typ,new", [("bf16", 1), ("bf16", 140), ("f16", 1), ("f32", 1)])
@pytest.mark.parametrize("scale", [-0.3, 0.0, 1.5])
def test_attend_scales(cuda_ok, typ, new, scale):
    check_attend(1, 4, 64, 16, typ, [(200, new)], scale=scale)


@pytest.mark.parametrize("typ,new", [("bf16", 1), ("bf16", 140), ("f16", 3), ("f32", 1)])
def test_attend_sharp_rows(cuda_ok, typ, new):
    """Logits of a few hundred: the reference moves and most weights vanish."""
    check_attend(1, 4, 64, 16, typ, [(700, new)], spread=60.0)


@pytest.mark.parametrize("typ,size,scale", [("bf16", 1e6, 1e-6), ("bf16", 1e-9, 1e8), ("bf16", 1e-38, 2e37), ("bf16", 3e37, 1e-38),
                                            ("bf16", 0.0, 1.0), ("f16", 1e-6, 1e5), ("f16", 1e4, 1e-4)])
def test_attend_queries_at_the_ends_of_the_range(cuda_ok, typ, size, scale):
    check_attend(1, 4, 64, 16, typ, [(90, 1), (50, 1)], spread=size, scale=scale)
    check_attend(1, 4, 64, 16, typ, [(90, 1), (50, 100)], spread=size, scale=scale)


@pytest.mark.parametrize("typ,new", [("bf16", 1), ("f16", 20), ("f16", 100), ("f32", 1)])
def test_attend_value_scales_far_apart(cuda_ok, typ, new):
    """Tokens of equal elements (scale 0), of the smallest scale, of large values: all have their weight."""
    def spoil(c):
        sc = scales(c)
        sc[:, :, :, 0::5, 2] = 0.0
        c.blocks[..., 8 * c.d:16 * c.d] &= 0xF0  # codes of tokens 0 .. 7 of a block are 0, those of scale 0 among them
        sc[:, :, :, 1::5, 2] = 2.0**-24
        sc[:, :, :, 2::5, 2] = 100.0
        sc[:, :, :, 8::5, 2] = 1e-3

    check_attend(2, 4, 64, 16, typ, [(300, new), (61, new)], spoil=spoil)


@pytest.mark.parametrize("typ,new", [("bf16", 1), ("f16", 100), ("f32", 1)])
def test_attend_values_around_a_far_mean(cuda_ok, typ, new):
    """Biases a thousand times the spread of a vector's elements."""
    def spoil(c):
        scales(c)[..., 3] = -300.0

    check_attend(2, 4, 64, 16, typ, [(300, new), (61, new)], spoil=spoil)


@pytest.mark.parametrize("new", [1, 100])
def test_attend_values_at_the_ends_of_f16(cuda_ok, new):
    """Vectors from -65504 to 65504, whose largest code stands for more than f16 holds."""
    def spoil(c):
        sc = scales(c)
        sc[:, :, :, 3::4, 1::2] = -65504.0
        sc[:, :, :, 3::4, 0::2] = 8736.0  # the smallest with -65504 + 15 s >= 65504
        c.blocks[..., :16 * c.d] |= c.blocks[..., :16 * c.d] << 1  # (many codes of 15)

    # the bound counts a value of up to 65536, taken as 65504: 2^-11 of it
    check_attend(2, 4, 64, 16, "bf16", [(300, new), (61, new)], spoil=spoil, scale=1e-6)


def test_attend_hints_may_be_larger(cuda_ok):
    check_attend(2, 4, 64, 16, "bf16", [(90, 1), (3, 1)], max_len=5000, max_tokens=4)
    check_attend(2, 4, 64, 16, "bf16", [(90, 20), (3, 7)], max_len=5000, max_tokens=900)


def test_attend_of_no_rows(cuda_ok):
    import paper_2608_14648_gb300 as skm

    c = make_cache(1, 64, 16, 2, 1)
    out, lse = skm.skm_kv4_attend(c, i32([[0, 1]]), i32([20]), i32([0, 0]),
                                  torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda"), 1, 20, want_lse=True)
    assert out.shape == (0, 2, 64) and lse.shape == (0, 2)


@pytest.mark.parametrize("typ,new", [("bf16", 1), ("f32", 1), ("f16", 200)])
def test_attend_twice_is_the_same_bit_for_bit(cuda_ok, typ, new):
    a = check_attend(2, 4, 128, 64, typ, [(3000, new), (10, new)], seed=5)
    b = check_attend(2, 4, 128, 64, typ, [(3000, new), (10, new)], seed=5)
    assert torch.equal(a, b)


def test_on_another_stream_and_in_a_graph(cuda_ok):
    import paper_2608_14648_gb300 as skm

    c = make_cache(2, 64, 16, 300, 9)
    table = make_table(1, 300, 300, 9).cuda()
    length, cu = i32([4000]), i32([0, 1])
    Q = torch.randn(1, 8, 64, device="cuda").to(torch.bfloat16)
    want, _ = skm.skm_kv4_attend(c, table, length, cu, Q, 1, 4000)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    got, _ = skm.skm_kv4_attend(c, table, length, cu, Q, 1, 4000, stream=st)
    st.synchronize()
    assert torch.equal(got, want)
    ws, out = skm.kv4_workspace(c, 1, 8, 1, 1, 4800), torch.empty_like(Q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        skm.skm_kv4_attend(c, table, length, cu, Q, 1, 4800, out=out, ws=ws)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    length.fill_(100)  # lengths are read on the device: the same graph serves the next step
    graph.replay()
    torch.cuda.synchronize()
    want, _ = skm.skm_kv4_attend(c, table, length, cu, Q, 1, 4800)
    assert torch.equal(out, want)


@pytest.mark.parametrize("heads,group,d,page,typ,seqs,causal,window", [
    (20, 1, 64, 16, "f16", [(0, 600), (300, 257), (17, 40)], True, 0),
    (20, 1, 64, 16, "bf16", [(0, 600), (300, 257), (17, 40)], True, 200),
    (10, 4, 128, 64, "bf16", [(100, 200), (0, 130), (500, 64), (900, 1)], True, 0),
    (16, 1, 256, 32, "bf16", [(0, 300), (200, 129), (1290, 33)], False, 0),
    (16, 1, 192, 32, "f16", [(0, 300), (200, 129), (1290, 33), (5, 60)], True, 0),
    (1, 1, 96, 16, "bf16", [(i * 7 % 100, 33 + i % 30) for i in range(300)], True, 0),
    (1, 2, 64, 16, "f16", [(i * 7 % 50, 1 + i % 20) for i in range(1100)], True, 0),
    (1, 2, 256, 64, "bf16", [(1500, 40)], True, 0), (2, 3, 192, 32, "f16", [(1400, 150), (0, 33), (70, 1)], True, 0),
    (1, 2, 256, 16, "f16", [(1600, 300), (3, 129)], True, 1350), (8, 16, 256, 64, "bf16", [(5, 40), (0, 17), (60, 3)], False, 0),
])
def test_attend_many_rows_in_several_waves(cuda_ok, heads, group, d, page, typ, seqs, causal, window):
    check_attend(heads, group, d, page, typ, seqs, causal, window)


@pytest.mark.parametrize("typ,group,new", [("bf16", 8, 1), ("f16", 5, 2), ("f32", 1, 1), ("f32", 2, 3)])
@pytest.mark.parametrize("d", [144, 192, 256])
def test_attend_wide_heads_split_over_the_whole_gpu(cuda_ok, typ, group, new, d):
    check_attend(2, group, d, 64, typ, [(6000, new), (0, new), (3111, new), (40, new)])
    check_attend(1, group, d, 16, typ, [(i * 11 % 70, new) for i in range(160)])


@pytest.mark.parametrize("typ", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("new", [1, 6, 100])
@pytest.mark.parametrize("what", [math.nan, math.inf])
def test_attend_rows_that_see_nothing_may_hold_anything(cuda_ok, typ, new, what):
    """Padded rows: all pages of a sequence absent, or no position left to see, whatever the queries are."""
    import paper_2608_14648_gb300 as skm

    c = make_cache(2, 64, 16, 40, 31)
    table = torch.full((4, 13), -1, dtype=torch.int32)
    table[0], table[2], table[3, 3:] = torch.arange(13), torch.arange(13, 26), torch.arange(26, 36)
    Q = torch.randn(4 * new, 4, 64, generator=torch.Generator().manual_seed(32)).to(DT[typ])
    clean = Q.clone()
    Q[new: 2 * new] = what  # no page
    Q[2 * new: 3 * new] = what  # no token
    Q[3 * new: 3 * new + new // 2] = what  # the first pages are absent, and these rows see no others
    args = table.cuda(), i32([200, 200, 0, 48 + new - new // 2]), i32([0, new, 2 * new, 3 * new, 4 * new])
    out, lse = skm.skm_kv4_attend(c, *args, Q.cuda(), new, 200, want_lse=True)
    want, want_lse = skm.skm_kv4_attend(c, *args, clean.cuda(), new, 200, want_lse=True)
    nothing = slice(new, 3 * new + new // 2)
    assert (out[nothing] == 0).all() and torch.isneginf(lse[nothing]).all()
    assert torch.isfinite(want).all() and torch.equal(out, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("typ", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("new", [1, 6, 100])
def test_attend_nan_in_a_query_stays_in_its_row(cuda_ok, typ, new):
    import paper_2608_14648_gb300 as skm

    c = make_cache(2, 64, 16, 40, 33)
    table = torch.arange(26, dtype=torch.int32).view(2, 13)
    table[1, 4] = -1  # an absent page among the others
    Q = torch.randn(2 * new, 4, 64, generator=torch.Generator().manual_seed(34)).to(DT[typ])
    args = table.cuda(), i32([200, 150]), i32([0, new, 2 * new])
    want, want_lse = skm.skm_kv4_attend(c, *args, Q.cuda(), new, 200, want_lse=True)
    hit = torch.zeros(2 * new, 4, dtype=torch.bool)
    for row, head, dim in ((0, 1, 63), (new, 0, 0), (2 * new - 1, 3, 17)):
        Q[row, head, dim] = math.nan
        hit[row, head] = True
    out, lse = skm.skm_kv4_attend(c, *args, Q.cuda(), new, 200, want_lse=True)
    hit = hit.cuda()
    assert torch.isnan(out[hit]).all() and torch.isnan(lse[hit]).all()
    assert torch.equal(out[~hit], want[~hit]) and torch.equal(lse[~hit], want_lse[~hit])


# heads, group, d, type, row counts of the sequences, tokens they hold at most
GIVES_UP = [
    (8, 4, 64, "bf16", [1] * 1000, 60), (8, 4, 128, "f16", [1] * 40, 700), (2, 8, 128, "bf16", [1, 1], 40000),
    (2, 1, 64, "f32", [1, 3, 2] * 300, 50), (2, 4, 64, "bf16", [1] * 3, 500),
]


@pytest.mark.parametrize("heads,group,d,typ,rows,most", GIVES_UP)
def test_attend_that_gives_up_says_so(cuda_ok, heads, group, d, typ, rows, most):
    """A wait that runs out (SKM_FAULT_WAIT, 1 ms): the status is set and every row is NaN or what it is without the fault."""
    import paper_2608_14648_gb300 as skm

    batch = len(rows)
    g = torch.Generator().manual_seed(21)
    length = [max(n, most - int(torch.randint(0, most // 2, (), generator=g))) for n in rows]
    cols = -(-max(length) // 16)
    c = make_cache(heads, d, 16, batch * cols, 22)
    table = make_table(batch, cols, batch * cols, 23).cuda()
    cu = [0] + torch.tensor(rows).cumsum(0).tolist()
    Q = torch.randn(cu[-1], heads * group, d, generator=g).to(DT[typ]).cuda()
    ws = skm.kv4_workspace(c, batch, heads * group, cu[-1], max(rows), max(length), {"bf16": 1, "f16": 2, "f32": 0}[typ])
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def call():
        ws.zero_()  # as a part: no weight, sums 0
        status.zero_()
        out = torch.full_like(Q, 77.0)
        out, lse = skm.skm_kv4_attend(c, table, i32(length), i32(cu), Q, max(rows), max(length), want_lse=True, out=out, ws=ws,
                                      status=status)
        return out, lse, int(status)

    want, want_lse, fine = call()
    assert fine == 0 and torch.isfinite(want).all()
    hit = 0
    for stuck in (0, 5, 16, 300, 1207):
        skm.skm_inject_fault(skm.FAULT_WAIT, stuck + 1)
        out, lse, gave_up = call()
        skm.skm_inject_fault(skm.FAULT_WAIT, 0)
        bad = torch.isnan(out).all(-1)
        assert (bad | (out == want).all(-1)).all() and (torch.isnan(lse) == bad).all()
        assert torch.equal(lse[~bad], want_lse[~bad])
        assert gave_up == int(bad.any())
        hit += gave_up
    assert hit >= 1
    out, lse, fine = call()  # nothing is left of it
    assert fine == 0 and torch.equal(out, want) and torch.equal(lse, want_lse)


def test_offsets_beyond_32_bits(cuda_ok):
    # a pool of 5 GB: its last pages against a small pool's, bit for bit
    import paper_2608_14648_gb300 as skm

    heads, d, page, pages, n = 8, 256, 64, 40000, 1500
    cols = -(-n // page)
    small, big = (skm.KVCache4(heads, d, page, pages=p) for p in (cols, pages))
    assert big.blocks.numel() > 1 << 32
    at = torch.arange(cols, dtype=torch.int32, device="cuda").view(1, cols)
    g = torch.Generator(device="cuda").manual_seed(8)
    K, V = torch.randn(2, n, heads, d, generator=g, device="cuda").to(torch.bfloat16)
    got = []
    for c, table in ((small, at), (big, at + (pages - cols))):
        skm.skm_kv4_write(c, table, i32([0]), i32([0, n]), K, V, n)
        res = list(skm.skm_kv4_read(c, table, i32([0]), i32([0, n]), n, n))
        for rows, typ in ((1, torch.bfloat16), (1, torch.float32), (300, torch.float16)):
            Q = torch.randn(rows, 2 * heads, d, generator=torch.Generator().manual_seed(9)).cuda().to(typ)
            res += skm.skm_kv4_attend(c, table, i32([n]), i32([0, rows]), Q, rows, n, want_lse=True)
        got.append(res)
    for x, y in zip(*got):
        assert torch.isfinite(x).all() and torch.equal(x, y)

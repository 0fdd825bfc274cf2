"""The 8-bit key/value cache on the GPU against plain implementations.

Codes and scales are compared for equality (their definition is fp32
arithmetic, done here on the CPU).  Attention is compared with the definition
in 64 bits over the codes that the cache really holds, elementwise within

  u |ref| + (w + 2 e) A + n 2^-30 max|v|,   A = sum_j p_j |v_j|,

u the rounding of the output type (2^-8 bf16, 2^-11 f16, 2^-24 f32), w the
relative error of a weight and of the sums that carry it (f16 weights: 2^-11
and fp32 sums that tensor cores may truncate, n 2^-23; f32: n + 16 roundings of
2^-24), e the error of a logit: fp32 products of d terms in any order, (d + 16)
2^-23 scale sum |q k|, plus 2^-22 |logit| for the base-2 form.  The last term covers
weights that underflow in f16 (2^-24 against a largest weight of at least
2^7; n of them).  lse: e and 2^-22 of its size, and the sums' error w without 2^-11."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

B = 16
DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
PLACE = [4 * ((t % 8) // 2) + 2 * (t // 8) + t % 2 for t in range(B)]


def logical(cache, name):
    """Codes as [pages, heads, page, d] on the CPU."""
    P, H, nb = cache.pages, cache.heads, cache.page // B
    u = getattr(cache, name).cpu()
    if name == "k":
        return u.view(P, H, nb, cache.d // B, B, B).permute(0, 1, 2, 4, 3, 5).reshape(P, H, cache.page, cache.d)
    return u.view(P, H, nb, cache.d, B)[..., PLACE].transpose(3, 4).reshape(P, H, cache.page, cache.d)


def make_cache(heads, d, page, pages, seed=0, fill=True):
    import paper_2608_14648_gb300 as skm

    c = skm.KVCache(heads, d, page, pages=pages)
    g = torch.Generator().manual_seed(seed)
    if fill:
        c.k.copy_(torch.randint(1, 256, c.k.shape, generator=g, dtype=torch.int64).to(torch.uint8))
        c.v.copy_(torch.randint(1, 256, c.v.shape, generator=g, dtype=torch.int64).to(torch.uint8))
        c.scales.copy_(0.004 + 0.02 * torch.rand(c.scales.shape, generator=g))
    return c


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def make_table(batch, cols, pages, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randperm(pages, generator=g)[: batch * cols].view(batch, cols).to(torch.int32)


class Held:
    """What a cache holds, by the definition, on the CPU."""

    def __init__(self, c):
        self.page, self.heads, self.d = c.page, c.heads, c.d
        self.code = {n: logical(c, n).to(torch.int64) for n in "kv"}
        self.scale = c.scales.cpu().clone()

    def write(self, table, start, cu, K, V):
        third = torch.tensor(1.0 / 127, dtype=torch.float32)
        for b in range(table.shape[0]):
            n = cu[b + 1] - cu[b]
            end = min(start[b] + n, table.shape[1] * self.page)
            for t0 in range(start[b] - start[b] % B, end, B):
                pg = int(table[b, t0 // self.page])
                if pg < 0 or pg >= self.scale.shape[0]:
                    continue
                slot = t0 % self.page
                lo, hi = max(t0, start[b]), min(t0 + B, end)
                for t, (name, X) in enumerate((("k", K), ("v", V))):
                    x = X[cu[b] + lo - start[b]: cu[b] + hi - start[b]].float().transpose(0, 1)
                    a = torch.where(torch.isfinite(x), x.abs(), torch.zeros(())).amax((1, 2))
                    old = self.scale[pg, :, slot // B, t] if t0 < start[b] else torch.zeros(self.heads)
                    s = torch.maximum(old, a * third)
                    held = self.code[name][pg, :, slot: slot + lo - t0]
                    if t0 < start[b]:
                        safe = torch.where(s > 0, s, torch.ones(()))
                        r = torch.where(old > 0, old / safe, torch.ones(()))
                        held[:] = torch.round((held - 128).float() * r[:, None, None]).to(torch.int64) + 128
                    q = x / s[:, None, None]
                    q = torch.where(torch.isnan(q), torch.zeros(()), q.round().clamp(-127, 127))
                    q = torch.where(s[:, None, None] > 0, q, torch.zeros(()))
                    self.code[name][pg, :, slot + lo - t0: slot + hi - t0] = q.to(torch.int64) + 128
                    self.scale[pg, :, slot // B, t] = s

    def values(self, name, table, b, lo, hi, dtype=torch.float64):
        """[hi - lo, heads, d]; zeros where the page is absent; and which are there."""
        out = torch.zeros(hi - lo, self.heads, self.d, dtype=dtype)
        there = torch.zeros(hi - lo, dtype=torch.bool)
        t = 0 if name == "k" else 1
        for p in range(lo // self.page, -(-hi // self.page)):
            pg = int(table[b, p]) if p < table.shape[1] else -1
            if pg < 0 or pg >= self.scale.shape[0]:
                continue
            a, z = max(lo, p * self.page), min(hi, (p + 1) * self.page)
            c = self.code[name][pg, :, a - p * self.page: z - p * self.page]
            s = self.scale[pg, :, :, t].repeat_interleave(B, 1)[:, a - p * self.page: z - p * self.page]
            out[a - lo: z - lo] = ((c - 128).to(dtype) * s.to(dtype)[:, :, None]).transpose(0, 1)
            there[a - lo: z - lo] = True
        return out, there


# ---- writing and reading back

WRITES = [
    # heads, d, page, type, (start, new) of each sequence
    (1, 16, 16, "bf16", [(0, 1)]),
    (2, 64, 16, "f16", [(0, 16), (5, 1), (15, 2), (16, 0), (31, 70)]),
    (3, 80, 32, "bf16", [(1, 15), (30, 3), (0, 100), (17, 17)]),
    (8, 128, 64, "bf16", [(63, 1), (64, 1), (0, 64), (100, 29)]),
    (2, 96, 48, "f32", [(7, 90), (47, 2)]),
    (1, 192, 16, "f32", [(3, 40)]),
    (2, 256, 128, "f16", [(120, 20), (0, 5)]),
]


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
    rows = rows.to(DT[typ])
    if spoil:
        spoil(rows)
    dev = rows.cuda()
    K, V = (dev[:, :heads], dev[:, 2 * heads:]) if fused else (dev[:, :heads].contiguous(), dev[:, 2 * heads:].contiguous())
    want = Held(c)
    want.write(table, start, cu, rows[:, :heads], rows[:, 2 * heads:])
    most = max(n for _, n in seqs)
    skm.skm_kv_write(c, table.cuda(), i32(start), i32(cu), K, V, most)
    torch.cuda.synchronize()
    return c, table, start, cu, want, most


def same(c, want):
    assert torch.equal(c.scales.cpu(), want.scale)
    for name in "kv":
        assert torch.equal(logical(c, name).to(torch.int64), want.code[name])


@pytest.mark.parametrize("heads,d,page,typ,seqs", WRITES)
@pytest.mark.parametrize("fused", [False, True])
def test_write_and_read_back(cuda_ok, heads, d, page, typ, seqs, fused):
    import paper_2608_14648_gb300 as skm

    c, table, start, cu, want, most = write_case(heads, d, page, typ, seqs, fused)
    same(c, want)
    for dt, code in ((torch.float32, skm.DTYPE_F32), (torch.bfloat16, skm.DTYPE_BF16), (torch.float16, skm.DTYPE_F16)):
        K, V = skm.skm_kv_read(c, table.cuda(), i32(start), i32(cu), cu[-1], most, code)
        for name, got in (("k", K), ("v", V)):
            ref = torch.cat([want.values(name, table, b, s, s + n, torch.float32)[0] for b, (s, n) in enumerate(seqs)])
            assert torch.equal(got.cpu(), ref.to(dt))


def test_write_leaves_infinities_and_nan_out(cuda_ok):
    def spoil(rows):
        rows[0, 0, 3] = math.inf
        rows[1, 0, 5] = -math.inf
        rows[2, 4, 7] = math.nan
        rows[3:9, :, :] = 0  # with the block's others
        rows[20:36] = math.nan  # a whole block without a finite value

    c, *_, want, _ = write_case(2, 64, 16, "bf16", [(0, 20), (0, 16)], True, spoil=spoil)
    same(c, want)


def test_write_of_zeros_and_tiny_values(cuda_ok):
    def spoil(rows):
        rows[:20] = 0
        rows[20:36] = 1e-42  # subnormal scale

    c, *_, want, _ = write_case(1, 32, 16, "f32", [(0, 20), (0, 16)], False, spoil=spoil)
    same(c, want)


def test_write_token_by_token_rescales_what_the_block_holds(cuda_ok):
    import paper_2608_14648_gb300 as skm

    c = make_cache(2, 64, 32, 5, 1)
    table = make_table(1, 3, 5, 1)
    want = Held(c)
    g = torch.Generator().manual_seed(2)
    for t in range(40):
        x = (torch.randn(1, 4, 64, generator=g) * (1 + t)).to(torch.bfloat16)
        want.write(table, [t], [0, 1], x[:, :2], x[:, 2:])
        dev = x.cuda()
        skm.skm_kv_write(c, table.cuda(), i32([t]), i32([0, 1]), dev[:, :2], dev[:, 2:], 1)
    same(c, want)


def test_write_unaligned_rows(cuda_ok):
    import paper_2608_14648_gb300 as skm

    heads, d = 2, 48
    c = make_cache(heads, d, 16, 6, 4)
    table = make_table(1, 5, 6, 4)
    want = Held(c)
    flat = torch.randn(1 + 33 * 101 * 3, generator=torch.Generator().manual_seed(5)).to(torch.float16)
    view = lambda x: (x[1:].as_strided((33, heads, d), (301, 101, 1)),  # noqa: E731
                      x[1:].as_strided((33, heads, d), (299, 53, 1)))
    K, V = view(flat)
    want.write(table, [9], [0, 33], K, V)
    dev = flat.cuda()
    skm.skm_kv_write(c, table.cuda(), i32([9]), i32([0, 33]), *view(dev), 33)
    same(c, want)


def test_absent_pages_and_the_tables_end(cuda_ok):
    import paper_2608_14648_gb300 as skm

    c = make_cache(1, 32, 16, 4, 6)
    table = torch.tensor([[2, -1, 9, 0]], dtype=torch.int32)  # 9: not a page of the pool
    want = Held(c)
    x = torch.randn(70, 2, 32, generator=torch.Generator().manual_seed(7)).to(torch.bfloat16)
    want.write(table, [3], [0, 70], x[:, :1], x[:, 1:])  # the table ends at 64
    dev = x.cuda()
    skm.skm_kv_write(c, table.cuda(), i32([3]), i32([0, 70]), dev[:, :1], dev[:, 1:], 70)
    same(c, want)
    K, V = skm.skm_kv_read(c, table.cuda(), i32([0]), i32([0, 80]), 80, 80, skm.DTYPE_F32)
    for name, got in (("k", K), ("v", V)):
        assert torch.equal(got.cpu(), want.values(name, table, 0, 0, 80, torch.float32)[0])


def test_read_one_of_the_two(cuda_ok):
    import paper_2608_14648_gb300 as skm

    c = make_cache(2, 64, 32, 4, 8)
    table = make_table(1, 4, 4, 8)
    held = Held(c)
    out = torch.full((21, 2, 64), 7.0, device="cuda")
    skm.skm_kv_read(c, table.cuda(), i32([5]), i32([0, 21]), 21, 21, skm.DTYPE_F32, out=(None, out))
    assert torch.equal(out.cpu(), held.values("v", table, 0, 5, 26, torch.float32)[0])


# ---- attention


def attend_ref(held, table, length, cu, Q, group, scale, causal, window, typ):
    """(out, lse, tolerance of out, tolerance of lse) in 64 bits."""
    heads, d = held.heads, held.d
    T = Q.shape[0]
    out = torch.zeros(T, heads * group, d, dtype=torch.float64)
    lse = torch.full((T, heads * group), -math.inf, dtype=torch.float64)
    tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
    for b in range(table.shape[0]):
        n, L = cu[b + 1] - cu[b], length[b]
        if n == 0 or L == 0:
            continue
        K, there = held.values("k", table, b, 0, L)
        V, _ = held.values("v", table, b, 0, L)
        p = torch.arange(L - n, L)[:, None]
        j = torch.arange(L)[None]
        see = there[None].expand(n, L).clone()
        if causal:
            see &= j <= p
        if window:
            see &= j > p - window
        any_ = see.any(1)
        for h in range(heads * group):
            q = Q[cu[b]:cu[b + 1], h].double()
            k, v = K[:, h // group], V[:, h // group]
            S = (q @ k.T * scale).masked_fill(~see, -math.inf)
            size = (abs(scale) * (q.abs() @ k.abs().T)).masked_fill(~see, 0).amax(1)
            big = S.abs().masked_fill(~see, 0).amax(1)
            e = (d + 16) * 2.0**-23 * size + 2.0**-22 * big
            l = torch.logsumexp(S, 1)
            w = torch.where(any_[:, None], torch.exp(S - l[:, None]), torch.zeros((), dtype=torch.float64)).nan_to_num()
            o, A = w @ v, w @ v.abs()
            sums = L * 2.0**-23 + 16 * 2.0**-24
            half = 2.0**-11 if typ != "f32" else 0.0
            u = {"bf16": 2.0**-8, "f16": 2.0**-11, "f32": 2.0**-24}[typ]
            sl = slice(cu[b], cu[b + 1])
            out[sl, h], lse[sl, h] = o, l
            tol[sl, h] = u * o.abs() + (half + sums + 2 * e)[:, None] * A * 1.01 + L * 2.0**-30 * v.abs().max()
            ltol[sl, h] = e + sums + 2.0**-22 * l.abs().nan_to_num(posinf=0)
    return out, lse, tol, ltol


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
    cu = [0]
    for _, n in seqs:
        cu.append(cu[-1] + n)
    Q = (spread * torch.randn(cu[-1], heads * group, d, generator=g)).to(DT[typ])
    dev = Q.cuda()
    if strided:
        wide = torch.zeros(cu[-1], heads * group + 3, d + 5, dtype=Q.dtype, device="cuda")
        wide[:, 2: 2 + heads * group, 1: 1 + d] = dev
        dev = wide[:, 2: 2 + heads * group, 1: 1 + d]
    sc = d**-0.5 if scale is None else scale
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got, lse = skm.skm_kv_attend(c, table.cuda(), i32(length), i32(cu), dev, max_tokens or max(n for _, n in seqs),
                                 max(length) if max_len is None else max_len, scale=scale, causal=causal, window=window,
                                 want_lse=True, status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    out, ref, tol, ltol = attend_ref(Held(c), table, length, cu, Q, group, sc, causal, window, typ)
    # with more rows than tokens the rows before the first position see nothing
    got, lse = got.cpu().double(), lse.cpu().double()
    assert torch.equal(torch.isneginf(lse), torch.isneginf(ref))
    fine = ~torch.isneginf(ref)
    assert torch.isfinite(got).all() and torch.isfinite(lse[fine]).all()
    assert (got[~fine] == 0).all()
    over = ((got - out).abs() - tol).amax() if got.numel() else 0.0
    assert over <= 0, f"out is off by {float((got - out).abs().max()):.3g}, over the bound by {float(over):.3g}"
    if fine.any():
        assert ((lse - ref).abs() - ltol)[fine].amax() <= 0
    return got


ATTENDS = [
    # heads, group, d, page, type, sequences
    (1, 1, 16, 16, "bf16", [(0, 1)]),
    (2, 4, 64, 16, "bf16", [(0, 1), (1, 1), (14, 1), (15, 1), (16, 1), (200, 1)]),
    (8, 4, 128, 64, "bf16", [(332, 1)]),
    (2, 8, 128, 32, "f16", [(1000, 1), (7, 1), (511, 1)]),
    (3, 1, 80, 32, "f16", [(31, 1), (63, 1), (64, 1), (65, 1)]),
    (1, 7, 96, 48, "bf16", [(100, 1), (47, 1)]),
    (2, 6, 192, 16, "bf16", [(77, 1), (300, 2)]),
    (2, 8, 256, 32, "f16", [(500, 5), (3, 5), (0, 5)]),
    (1, 16, 128, 128, "bf16", [(1500, 1), (90, 2)]),
    (1, 32, 64, 16, "f16", [(250, 1)]),
    (1, 40, 64, 16, "bf16", [(250, 3)]),
    (12, 1, 64, 16, "f32", [(100, 1), (0, 1), (33, 1)]),
    (2, 4, 128, 64, "f32", [(700, 3), (12, 1)]),
    (1, 3, 256, 16, "f32", [(60, 9)]),
    (4, 4, 128, 64, "bf16", [(0, 130), (300, 65), (17, 1), (5, 33)]),
    (3, 1, 64, 16, "f16", [(0, 300), (100, 129)]),
    (2, 2, 96, 32, "bf16", [(40, 200)]),
    (1, 5, 80, 16, "f16", [(1, 77), (64, 64)]),
    (1, 2, 256, 64, "bf16", [(10, 90)]),
    (2, 3, 192, 32, "bf16", [(70, 150), (0, 33)]),
    (1, 4, 256, 128, "f16", [(300, 260), (1, 7)]),
    (1, 2, 144, 16, "f16", [(20, 60)]),
    (1, 8, 16, 16, "bf16", [(60, 40), (0, 1)]),
]


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
    seqs = [(i * 37 % 90, i % 3) for i in range(1100)]
    check_attend(1, 2, 32, 16, "bf16", seqs)


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


def test_attend_bf16_queries_beyond_f16(cuda_ok):
    check_attend(1, 4, 64, 16, "bf16", [(90, 1), (50, 100)], spread=1e6, scale=1e-6)
    check_attend(1, 4, 64, 16, "bf16", [(90, 1), (50, 100)], spread=1e-9, scale=1e8)


@pytest.mark.parametrize("typ,new", [("bf16", 1), ("f16", 20), ("f16", 100), ("f32", 1)])
def test_attend_value_scales_far_apart(cuda_ok, typ, new):
    """Blocks of zeros, of tiny values and of large ones carry weight all the same."""
    def spoil(c):
        c.scales[0::5, :, :, 1] = 0.0
        c.v[0::5] = 128
        c.scales[1::5, :, :, 1] = 1e-35
        c.scales[2::5, :, :, 1] = 3e-20
        c.scales[3::5, :, :, 1] = 50.0

    check_attend(2, 4, 64, 16, typ, [(300, new), (61, new)], spoil=spoil)


def test_attend_hints_may_be_larger(cuda_ok):
    check_attend(2, 4, 64, 16, "bf16", [(90, 1), (3, 1)], max_len=5000, max_tokens=4)
    check_attend(2, 4, 64, 16, "bf16", [(90, 20), (3, 7)], max_len=5000, max_tokens=900)


def test_attend_of_no_rows(cuda_ok):
    import paper_2608_14648_gb300 as skm

    c = make_cache(1, 64, 16, 2, 1)
    out, lse = skm.skm_kv_attend(c, i32([[0, 1]]), i32([20]), i32([0, 0]),
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
    want, _ = skm.skm_kv_attend(c, table, length, cu, Q, 1, 4000)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    got, _ = skm.skm_kv_attend(c, table, length, cu, Q, 1, 4000, stream=st)
    st.synchronize()
    assert torch.equal(got, want)
    ws, out = skm.kv_workspace(c, 1, 8, 1, 1, 4800), torch.empty_like(Q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        skm.skm_kv_attend(c, table, length, cu, Q, 1, 4800, out=out, ws=ws)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    length.fill_(100)  # lengths are read on the device: the same graph serves the next step
    graph.replay()
    torch.cuda.synchronize()
    want, _ = skm.skm_kv_attend(c, table, length, cu, Q, 1, 4800)
    assert torch.equal(out, want)


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
        want = Held(c)
        odd = [cu[b] for b in range(1, 40, 2)] + [cu[-1]]
        want.write(table[1::2], start[1::2], odd, K, V)
        skm.skm_kv_write(c, table.cuda(), i32(start), i32(cu), K.cuda(), V.cuda(), 3)
        same(c, want)


@pytest.mark.parametrize("start", [64, 80, 2**31 - 1, 2**31 - 40, -2**31])
def test_write_beyond_the_table(cuda_ok, start):
    # nothing at or past cols * page = 64; a negative position counts as 0
    import paper_2608_14648_gb300 as skm

    c = make_cache(1, 32, 32, 3)
    want = Held(c)
    table = torch.tensor([[2, 0]], dtype=torch.int32)
    K, V = torch.randn(2, 100, 1, 32, generator=torch.Generator().manual_seed(6))
    if start < 0:
        want.write(table, [0], [0, 100], K, V)
    skm.skm_kv_write(c, table.cuda(), i32([start]), i32([0, 100]), K.cuda(), V.cuda(), 100)
    same(c, want)


@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
def test_write_rounds_like_a_division(cuda_ok, typ):
    # values at and next to the middles of two codes: a few units in the last place to either side
    import paper_2608_14648_gb300 as skm

    g = torch.Generator().manual_seed(7)
    blocks, d = 60, 256
    c = make_cache(1, d, 16, blocks)
    table = torch.arange(blocks, dtype=torch.int32).view(1, blocks)
    top = torch.exp(60 * torch.rand(blocks, 1, 1, generator=g) - 30)
    top[:6, 0, 0] = torch.tensor([1.0, 127.0, 126.99999, 254.0, 3.0, 0.7])
    if typ == "f16":
        top = top.clamp(1e-3, 6e4)
    s = top.to(DT[typ]).float() * torch.tensor(1.0 / 127)
    x = s * (torch.randint(-127, 127, (blocks, 16, d), generator=g) + 0.5)
    if typ == "f32":
        x = (x.view(torch.int32) + torch.randint(-3, 4, x.shape, generator=g, dtype=torch.int32)).view(torch.float32)
    x = torch.minimum(torch.maximum(x, -top), top)
    x[:, 0, 0] = top[:, 0, 0]
    K = x.to(DT[typ]).view(blocks * 16, 1, d)
    V = K.flip(2)
    want = Held(c)
    want.write(table, [0], [0, blocks * 16], K, V)
    skm.skm_kv_write(c, table.cuda(), i32([0]), i32([0, blocks * 16]), K.cuda(), V.cuda(), blocks * 16)
    same(c, want)


@pytest.mark.parametrize("heads,group,d,page,typ,seqs,window", [
    (1, 2, 256, 64, "bf16", [(1500, 40)], 0), (2, 3, 192, 32, "f16", [(1400, 150), (0, 33), (70, 1)], 0),
    (1, 2, 256, 16, "f16", [(1600, 300), (3, 129)], 1350), (8, 16, 256, 64, "bf16", [(5, 40), (0, 17), (60, 3)], 0),
])
@pytest.mark.parametrize("causal", [True, False])
def test_attend_wide_heads_many_rows(cuda_ok, heads, group, d, page, typ, seqs, window, causal):
    # long enough, or enough units, for d > 128 to go to the kernel for many rows
    check_attend(heads, group, d, page, typ, seqs, causal, window if causal else 0)


def test_offsets_beyond_32_bits(cuda_ok):
    # a pool of 5 GB of keys and as much of values: its last pages against a small pool's, bit for bit
    import paper_2608_14648_gb300 as skm

    heads, d, page, pages, n = 8, 256, 64, 40000, 1500
    cols = -(-n // page)
    small, big = (skm.KVCache(heads, d, page, pages=p) for p in (cols, pages))
    assert big.k.numel() > 1 << 32
    at = torch.arange(cols, dtype=torch.int32, device="cuda").view(1, cols)
    g = torch.Generator(device="cuda").manual_seed(8)
    K, V = torch.randn(2, n, heads, d, generator=g, device="cuda").to(torch.bfloat16)
    got = []
    for c, table in ((small, at), (big, at + (pages - cols))):
        skm.skm_kv_write(c, table, i32([0]), i32([0, n]), K, V, n)
        res = list(skm.skm_kv_read(c, table, i32([0]), i32([0, n]), n, n))
        for rows, typ in ((1, torch.bfloat16), (1, torch.float32), (300, torch.float16)):
            Q = torch.randn(rows, 2 * heads, d, generator=torch.Generator().manual_seed(9)).cuda().to(typ)
            res += skm.skm_kv_attend(c, table, i32([n]), i32([0, rows]), Q, rows, n, want_lse=True)
        got.append(res)
    for x, y in zip(*got):
        assert torch.isfinite(x).all() and torch.equal(x, y)

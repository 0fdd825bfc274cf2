"""The 4-bit key/value cache where weighted sums cancel, where its values end, where codes lie next to the middle of two,
where a wait runs out, and what the two operands of prompts' products hold."""
from fractions import Fraction

import pytest
import torch
from test_gpu_kv import DT, i32
from test_gpu_kv4 import Held4, make_cache, make_table, scales

pytestmark = pytest.mark.gpu


# ---- sums that cancel

@pytest.mark.parametrize("typ", ["bf16", "f16"])
def test_long_sums_keep_their_precision(cuda_ok, typ):
    """1024 sequences of a million tokens (which share pages), 55,000 a warp and unit.  Neighbouring tokens have one weight (of
    sixteen, as keys' first dims have codes 0..15) and codes 8 + i and 8 - i: a value's mean is b + 8 s = 2^-9 exactly, and a sum of
    codes around their middle is 0 after every block, where one of the codes themselves loses bits to every product that is
    added.  Bound: the output's rounding, the fp32 sums of weights and of biases (two tokens a block in a lane's own:
    n 2^-24 each), and the value scale's logarithm and reciprocal, 2^-20 of |b| + 16 s."""
    import paper_2608_14648_gb300 as skm

    page, cols, d, batch = 16384, 64, 16, 1024
    n = page * cols
    c = skm.KVCache4(1, d, page, pages=cols)
    g = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda lo, hi, *s: torch.randint(lo, hi, s, generator=g, dtype=torch.uint8, device="cuda")  # noqa: E731
    keys = c.blocks[..., :8 * d].view(-1, 8, 4, 2, 2)  # [block][token % 8][4 c][l][token / 8]
    keys.copy_(rand(0, 16, n // 16, 4, 1, 1, 2).repeat_interleave(2, 1) * 17)  # tokens 2 i and 2 i + 1 alike
    values = c.blocks[..., 8 * d:16 * d].view(-1, 8, 4, 2, 2)  # [block][g][token pair][token % 2][dim / 8], low and high half: token / 8
    low, high = rand(1, 16, n // 16, 8, 4, 2), rand(1, 16, n // 16, 8, 4, 2)
    values[:, :, :, 0], values[:, :, :, 1] = low | high << 4, (16 - low) | (16 - high) << 4
    sc = scales(c)
    sc[..., 0], sc[..., 1], sc[..., 2], sc[..., 3] = 0.11, 0.0, 0.125, -1 + 2.0**-9
    Q = torch.zeros(batch, 4, d, dtype=DT[typ], device="cuda")
    Q[..., 0] = torch.tensor([0.3, 1.0, -1.0, 2.0])
    table = torch.arange(cols, dtype=torch.int32, device="cuda").expand(batch, cols).contiguous()
    length, cu = torch.full((batch,), n, dtype=torch.int32, device="cuda"), torch.arange(batch + 1, dtype=torch.int32, device="cuda")
    out, _ = skm.skm_kv4_attend(c, table, length, cu, Q, 1, n, scale=1.0)
    u = {"bf16": 2.0**-8, "f16": 2.0**-11}[typ]
    adds = 2 * batch * n // (152 * 16) // 16
    tol = 2.0**-9 * (u + 2 * adds * 2.0**-24) + 2.0**-20 * 3
    assert (out.double() - 2.0**-9).abs().max() <= tol


@pytest.mark.parametrize("typ", ["bf16", "f16"])
def test_long_sums_of_any_codes_keep_their_precision(cuda_ok, typ):
    """As above with codes c and 15 - c of neighbouring tokens: a mean of b + 7.5 s = 2^-9, and sums of codes less 7.5 that are 0 after
    every block (of codes less 8, half a code a token).  Above, of codes less 7.5, half a code a token too: no sum may lose bits to
    every product that it takes."""
    import paper_2608_14648_gb300 as skm

    page, cols, d, batch = 16384, 64, 16, 1024
    n = page * cols
    c = skm.KVCache4(1, d, page, pages=cols)
    g = torch.Generator(device="cuda").manual_seed(4)
    rand = lambda lo, hi, *s: torch.randint(lo, hi, s, generator=g, dtype=torch.uint8, device="cuda")  # noqa: E731
    c.blocks[..., :8 * d].view(-1, 8, 4, 2, 2).copy_(rand(0, 16, n // 16, 4, 1, 1, 2).repeat_interleave(2, 1) * 17)
    values, two = c.blocks[..., 8 * d:16 * d].view(-1, 8, 4, 2, 2), rand(0, 256, n // 16, 8, 4, 2)
    values[:, :, :, 0], values[:, :, :, 1] = two, 255 - two
    sc = scales(c)
    sc[..., 0], sc[..., 1], sc[..., 2], sc[..., 3] = 0.11, 0.0, 0.125, -0.9375 + 2.0**-9
    Q = torch.zeros(batch, 4, d, dtype=DT[typ], device="cuda")
    Q[..., 0] = torch.tensor([0.3, 1.0, -1.0, 2.0])
    table = torch.arange(cols, dtype=torch.int32, device="cuda").expand(batch, cols).contiguous()
    length, cu = torch.full((batch,), n, dtype=torch.int32, device="cuda"), torch.arange(batch + 1, dtype=torch.int32, device="cuda")
    out, _ = skm.skm_kv4_attend(c, table, length, cu, Q, 1, n, scale=1.0)
    u = {"bf16": 2.0**-8, "f16": 2.0**-11}[typ]
    adds = 2 * batch * n // (152 * 16) // 16
    tol = 2.0**-9 * (u + 2 * adds * 2.0**-24) + 2.0**-20 * 3
    assert (out.double() - 2.0**-9).abs().max() <= tol


# ---- values at f16's ends

WIDE = 8736.0  # the smallest f16 s with -65504 + 15 s >= 65504: the largest code stands for 65536


@pytest.mark.parametrize("typ", ["f16", "f32"])
@pytest.mark.parametrize("back", ["f16", "bf16", "f32"])
def test_vectors_from_end_to_end_read_back(cuda_ok, typ, back):
    """Within half a scale of what was written and the type's rounding, in f16 too."""
    import paper_2608_14648_gb300 as skm

    x = (2 * torch.rand(20, 4, 48, generator=torch.Generator().manual_seed(1)) - 1) * 65504
    x[..., 5], x[..., 40] = -65504.0, 65504.0
    x = x.to(DT[typ])
    c, table, dev = make_cache(2, 48, 16, 2), i32([[1, 0]]), x.cuda()
    skm.skm_kv4_write(c, table, i32([3]), i32([0, 20]), dev[:, :2], dev[:, 2:], 20)
    got = skm.skm_kv4_read(c, table, i32([3]), i32([0, 20]), 20, 20, {"f32": 0, "bf16": 1, "f16": 2}[back])
    u = {"bf16": 2.0**-8, "f16": 2.0**-11, "f32": 2.0**-24}[back]
    for y, want in zip(got, (x[:, :2], x[:, 2:])):
        assert y.dtype == DT[back] and torch.isfinite(y).all()
        assert (y.cpu().double() - want.double()).abs().max() <= WIDE / 2 + u * 65536


@pytest.mark.parametrize("d", [64, 128, 192])
@pytest.mark.parametrize("batch,length,new", [(1, 300, 1), (1, 40000, 1), (40, 3000, 1), (3, 300, 5), (1, 400, 100), (1, 6000, 100)])
def test_attention_over_values_at_the_ends(cuda_ok, d, batch, length, new):
    """Means of 65536 and of -65504 in f16, in every way that a row's result is put together.  A mean is off by its weights'
    rounding and sums, 2^-11 + length 2^-23 of 65536, and f16's steps there are 32."""
    import paper_2608_14648_gb300 as skm

    cols = -(-length // 64)
    c = make_cache(1, d, 64, cols)
    c.blocks[..., 8 * d:16 * d] = 0
    sc = scales(c)
    sc[..., 2], sc[..., 3] = WIDE, -65504.0
    top = c.blocks[..., 8 * d:16 * d].unflatten(-1, (d // 16, 8, 16))  # codes of dims g and g + 8: the even g are 15
    top[..., 0::2, :] = 255
    table = torch.arange(cols, dtype=torch.int32, device="cuda").expand(batch, cols).contiguous()
    cu = i32([i * new for i in range(batch + 1)])
    Q = torch.randn(batch * new, 4, d, generator=torch.Generator().manual_seed(2)).to(torch.float16).cuda()
    out, _ = skm.skm_kv4_attend(c, table, i32([length] * batch), cu, Q, new, length, causal=False, scale=1e-3)
    want = torch.full((d,), -65504.0, dtype=torch.float64)
    want.view(d // 16, 2, 8)[..., 0::2] = 65504.0
    assert torch.isfinite(out).all()
    assert (out.cpu().double() - want).abs().max() <= (2.0**-11 + length * 2.0**-23) * 65536 + 32


# ---- codes at the middle of two

@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("slow", [False, True])
def test_codes_next_to_a_middle_are_exact(cuda_ok, typ, slow):
    """b = -(k + 1/2) s puts the middle of codes k and k + 1 at 0, where elements come as close to it as the type's smallest
    numbers: the code is that of exact rational arithmetic.  slow: an infinity among the elements, left out."""
    import paper_2608_14648_gb300 as skm

    near = [0.0, 1e-20, -1e-20, 1e-30, -1e-30, 1e-38, -1e-38, 1e-44, -1e-44, 3e-8, -3e-8, 6e-8, -6e-8, 1e-5, -1e-5]
    steps = [2.0, 0.5, 2.0**-10, 4096.0, 0.75, 1.25]
    rows, scale = [], []
    for s in steps:
        for k in range(15):
            b = -(k + 0.5) * s
            row = [b, b + 15 * s] + [v * max(s, 1.0) for v in near] + [b + 15 * s] * 15
            row[-1] = float("inf") if slow else b
            rows.append(row)
            scale.append((s, k))
    x = torch.tensor(rows, dtype=torch.float64).to(DT[typ])  # (ends are exact in all three types)
    n, d = x.shape
    c = make_cache(1, d, 16, -(-n // 16))
    table = torch.arange(-(-n // 16), dtype=torch.int32).view(1, -1)
    K = x.view(n, 1, d)
    V = K.flip(2)
    skm.skm_kv4_write(c, table.cuda(), i32([0]), i32([0, n]), K.cuda(), V.cuda(), n)
    held = Held4(c)
    for t, X in enumerate((K, V)):
        code, sc = (h.reshape(-1, h.shape[-1])[:n] for h in (held.code[t], held.scale))
        for r, (s, k) in enumerate(scale):
            assert sc[r, 2 * t] == s and sc[r, 2 * t + 1] == -(k + 0.5) * s
            exact = [15 if v == float("inf") else round((Fraction(v) + Fraction((k + 0.5) * s)) / Fraction(s)) for v in X[r, 0].tolist()]
            assert code[r].tolist() == exact, (s, k)


# ---- waits that run out

@pytest.mark.parametrize("heads,group,d,typ,lse,rows,most", [
    (8, 4, 64, "bf16", False, [100, 70, 90], 500), (4, 2, 128, "f16", True, [300, 40], 900), (2, 4, 128, "bf16", False, [64], 20000),
    (2, 1, 192, "bf16", True, [130, 40, 35], 700), (1, 2, 256, "f16", False, [50], 9000), (1, 1, 64, "f16", True, [33] * 1100, 90),
])
def test_many_rows_that_give_up_say_so(cuda_ok, heads, group, d, typ, lse, rows, most):
    """A tile of keys that never counts as arrived (SKM_FAULT_WAIT, 1 ms), the first of a CTA or, with products in flight, the second:
    the status is set, and every row is NaN or what it is without the fault."""
    import paper_2608_14648_gb300 as skm

    batch = len(rows)
    g = torch.Generator().manual_seed(21)
    length = [max(n, most - int(torch.randint(0, most // 2, (), generator=g))) for n in rows]
    cols = -(-max(length) // 16)
    c = make_cache(heads, d, 16, batch * cols, 22)
    table = make_table(batch, cols, batch * cols, 23).cuda()
    cu = [0] + torch.tensor(rows).cumsum(0).tolist()
    Q = torch.randn(cu[-1], heads * group, d, generator=g).to(DT[typ]).cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def call():
        status.zero_()
        out, l = skm.skm_kv4_attend(c, table, i32(length), i32(cu), Q, max(rows), max(length), want_lse=lse, out=torch.full_like(Q, 77.0), status=status)
        return out, l, int(status)

    want, want_lse, fine = call()
    assert fine == 0 and torch.isfinite(want).all()
    hits = set()
    for stuck in (0, 1, 2, 7, 20, 45, 46):
        skm.skm_inject_fault(skm.FAULT_WAIT, stuck + 1)
        out, l, gave_up = call()
        skm.skm_inject_fault(skm.FAULT_WAIT, 0)
        bad = torch.isnan(out).all(-1)
        assert (bad | (out == want).all(-1)).all()
        if lse:
            assert (torch.isnan(l) == bad).all() and torch.equal(l[~bad], want_lse[~bad])
        assert gave_up == int(bad.any())
        if gave_up:
            hits.add(stuck % 2)
    assert hits == {0, 1}
    out, l, fine = call()  # nothing is left of it
    assert fine == 0 and torch.equal(out, want) and (l is None or torch.equal(l, want_lse))


@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("typ,lse", [("f16", False), ("f16", True), ("bf16", True)])
def test_prompts_have_their_values_exactly(cuda_ok, d, typ, lse):
    """Up to 128 dims: s (c - 8) as the sum of two f16.  Equal weights, three codes of 15 for seven of 5 and b = -8 s: the mean is
    0, and what one f16 would leave of 7 s and of 3 s does not cancel.  Exact otherwise but for sums that tensor cores may truncate:
    of n / 16 blocks and two operands, 17 terms each within 2^-23 of a partial sum, 70 s a weight at most."""
    import paper_2608_14648_gb300 as skm

    n, rows = 640, 48
    s = torch.tensor(0.2998).half().double()
    tol = float(2 / 16 * 17 * 2.0**-23 * 70 * s)
    left = lambda k: float((k * s).half().double() - k * s)  # noqa: E731
    assert abs(3 * left(7) + 7 * left(-3)) / 10 > 3 * tol  # one operand would be seen
    c = make_cache(1, d, 64, n // 64)
    code = torch.where(torch.arange(n) % 10 < 3, 15, 5).to(torch.uint8).view(n // 16, 16)
    two = (code[:, :8] | code[:, 8:] << 4).view(n // 64, 1, 4, 1, 1, 4, 2, 1)  # [page][head][block][16 dims][g][token pair][token % 2][dim / 8]
    c.blocks[..., 8 * d:16 * d].unflatten(-1, (d // 16, 8, 4, 2, 2)).copy_(two.cuda())
    sc = scales(c)
    sc[..., 2], sc[..., 3] = float(s), float(-8 * s)
    Q = torch.zeros(rows, 1, d, dtype=DT[typ], device="cuda")
    table = torch.arange(n // 64, dtype=torch.int32, device="cuda").view(1, -1)
    assert Held4(c).code[1].reshape(-1, d)[:20].T.tolist() == [code.flatten()[:20].tolist()] * d
    out, _ = skm.skm_kv4_attend(c, table, i32([n]), i32([0, rows]), Q, rows, n, causal=False, want_lse=lse)
    assert out.double().abs().max() <= tol + 2.0**-25


@pytest.mark.parametrize("d", [144, 192, 256])
@pytest.mark.parametrize("typ,lse", [("f16", False), ("f16", True), ("bf16", True)])
def test_prompts_of_wide_heads_have_their_weights_in_two_parts(cuda_ok, d, typ, lse):
    """Above 128 dims: weights as the sum of two f16.  Tokens of equal elements (f16 numbers) and three weights, whose sums
    cancel; bound: logits to 2^-20 (key and bias around 8 apart before they meet), 2^x to 2^-22, weights to 2^-22, and as above."""
    import paper_2608_14648_gb300 as skm

    n, rows, size = 768, 48, 0.55
    # the keys' first dim has codes 0, 1, 2: logits 0, size, 2 size
    x = torch.tensor([0.0, size, 2 * size], dtype=torch.float64).to(DT["f32"]).double()
    p = torch.exp(x - x[2])
    v = torch.tensor([1.0, 0, 0], dtype=torch.float64)
    v[1] = (-v[0] * p[0] / p[1]).half()
    v[2] = (-(v[0] * p[0] + v[1] * p[1]) / p[2]).half()
    ref, A = float((p * v).sum() / p.sum()), float((p * v.abs()).sum() / p.sum())
    tol = 2.0**-18 * A + 2 / 16 * 17 * 2.0**-23 + abs(ref) * 2.0**-8 + 2.0**-25
    one = float(((128 * p).half().double() * v).sum() / (128 * p.sum()))
    assert abs(one - ref) > 3 * tol  # weights in one f16 would be seen
    c = make_cache(1, d, 64, n // 64)
    c.blocks[..., :16 * d] = 0
    kind = (torch.arange(n) % 3).view(n // 16, 16)
    keys = c.blocks[..., :8 * d].view(n // 16, d // 16, 8, 4, 2, 2)
    keys[:, 0, :, 0, 0, 0], keys[:, 0, :, 0, 0, 1] = kind[:, :8].to(torch.uint8).cuda(), kind[:, 8:].to(torch.uint8).cuda()
    sc = scales(c).view(n // 16, 16, 4)
    sc[..., 0], sc[..., 1], sc[..., 2], sc[..., 3] = 1.0, 0.0, 0.0, v[kind].half().cuda()
    Q = torch.zeros(rows, 1, d, dtype=DT[typ], device="cuda")
    Q[..., 0] = 1.0
    table = torch.arange(n // 64, dtype=torch.int32, device="cuda").view(1, -1)
    out, _ = skm.skm_kv4_attend(c, table, i32([n]), i32([0, rows]), Q, rows, n, causal=False, want_lse=lse, scale=size)
    assert (out.double() - ref).abs().max() <= tol


@pytest.mark.parametrize("d", [16, 64, 96, 128, 144, 256])
@pytest.mark.parametrize("n,group,rows", [(1920, 1, 48), (9600, 1, 100), (1440, 2, 40), (3840, 16, 17)])
def test_f16_prompts_have_their_weights_in_two_f16(cuda_ok, d, n, group, rows):
    """Values +- s of codes 9 and 7 (b = -8 s) whose sums under three weights cancel.  Bound: logits to 2^-20 and 2^x to 2^-22, weights to
    2^-21, in all 2^-18 of sum p |v|, and sums on tensor cores as above."""
    import paper_2608_14648_gb300 as skm

    size = 0.55
    x = torch.tensor([0.0, size, 2 * size], dtype=torch.float64).float().double()
    p = torch.exp(x - x[2])
    v = torch.tensor([1.0, 0, 0], dtype=torch.float64)
    v[1] = (-v[0] * p[0] / p[1]).half()
    v[2] = (-(v[0] * p[0] + v[1] * p[1]) / p[2]).half()
    ref, A = float((p * v).sum() / p.sum()), float((p * v.abs()).sum() / p.sum())
    tol = 2.0**-18 * A + 2 / 16 * 17 * 2.0**-23 + abs(ref) * 2.0**-11 + 2.0**-25
    one = float(((128 * p).half().double() * v).sum() / (128 * p.sum()))
    assert abs(one - ref) > 3 * tol  # weights in one f16 would be seen
    c = make_cache(1, d, 16, n // 16)
    c.blocks[..., :8 * d] = 0
    kind = (torch.arange(n) % 3).view(n // 16, 16)
    keys = c.blocks[..., :8 * d].view(n // 16, d // 16, 8, 4, 2, 2)
    keys[:, 0, :, 0, 0, 0], keys[:, 0, :, 0, 0, 1] = kind[:, :8].to(torch.uint8).cuda(), kind[:, 8:].to(torch.uint8).cuda()
    code = torch.where(v > 0, 9, 7)[kind].to(torch.uint8)
    two = (code[:, :8] | code[:, 8:] << 4).view(n // 16, 1, 1, 4, 2, 1).cuda()  # [block][16 dims][g][token pair][token % 2][dim / 8]
    c.blocks[..., 8 * d:16 * d].view(n // 16, d // 16, 8, 4, 2, 2).copy_(two)
    sc, s = scales(c).view(n // 16, 16, 4), v.abs()[kind].half().cuda()
    sc[..., 0], sc[..., 1], sc[..., 2], sc[..., 3] = 1.0, 0.0, s, -8 * s
    Q = torch.zeros(rows, group, d, dtype=torch.float16, device="cuda")
    Q[..., 0] = 1.0
    table = torch.arange(n // 16, dtype=torch.int32, device="cuda").view(1, -1)
    out, _ = skm.skm_kv4_attend(c, table, i32([n]), i32([0, rows]), Q, rows, n, causal=False, scale=size)
    assert (out.double() - ref).abs().max() <= tol


@pytest.mark.parametrize("d", [16, 64, 96, 128, 144, 256])
@pytest.mark.parametrize("n,group,rows", [(768, 1, 1), (768, 4, 3), (3840, 8, 1), (48, 1, 1), (768, 8, 4), (48000, 4, 2)])
def test_f16_rows_have_their_weights_in_two_f16(cuda_ok, d, n, group, rows):
    """As above for few rows, whose weights carry the value's scale: the scales' logarithms and reciprocals are good to 2^-22 more,
    b / s + 7.5 to 2^-23 of 7.5, which is within 2^-18 of sum p |v| still."""
    import paper_2608_14648_gb300 as skm

    size = 0.55
    x = torch.tensor([0.0, size, 2 * size], dtype=torch.float64).float().double()
    p = torch.exp(x - x[2])
    v = torch.tensor([1.0, 0, 0], dtype=torch.float64)
    v[1] = (-v[0] * p[0] / p[1]).half()
    v[2] = (-(v[0] * p[0] + v[1] * p[1]) / p[2]).half()
    ref, A = float((p * v).sum() / p.sum()), float((p * v.abs()).sum() / p.sum())
    tol = 2.0**-18 * A + 2 / 16 * 17 * 2.0**-23 + abs(ref) * 2.0**-11 + 2.0**-25
    w = p * v.abs()
    one = (w * 128 / w.max()).half().double() * w.max() / 128  # the largest is 2^7
    assert abs(float((one * v.sign()).sum() / p.sum()) - ref) > 3 * tol  # weights in one f16 would be seen
    c = make_cache(1, d, 16, n // 16)
    c.blocks[..., :8 * d] = 0
    kind = (torch.arange(n) % 3).view(n // 16, 16)
    keys = c.blocks[..., :8 * d].view(n // 16, d // 16, 8, 4, 2, 2)
    keys[:, 0, :, 0, 0, 0], keys[:, 0, :, 0, 0, 1] = kind[:, :8].to(torch.uint8).cuda(), kind[:, 8:].to(torch.uint8).cuda()
    code = torch.where(v > 0, 9, 7)[kind].to(torch.uint8)
    two = (code[:, :8] | code[:, 8:] << 4).view(n // 16, 1, 1, 4, 2, 1).cuda()  # [block][16 dims][g][token pair][token % 2][dim / 8]
    c.blocks[..., 8 * d:16 * d].view(n // 16, d // 16, 8, 4, 2, 2).copy_(two)
    sc, s = scales(c).view(n // 16, 16, 4), v.abs()[kind].half().cuda()
    sc[..., 0], sc[..., 1], sc[..., 2], sc[..., 3] = 1.0, 0.0, s, -8 * s
    Q = torch.zeros(rows, group, d, dtype=torch.float16, device="cuda")
    Q[..., 0] = 1.0
    table = torch.arange(n // 16, dtype=torch.int32, device="cuda").view(1, -1)
    out, _ = skm.skm_kv4_attend(c, table, i32([n]), i32([0, rows]), Q, rows, n, causal=False, scale=size)
    assert (out.double() - ref).abs().max() <= tol

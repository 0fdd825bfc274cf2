"""Rotary positions on the GPU against the definition in 64 bits: elementwise within

  u max(|ref|, least) + (2^-22 + 2^-24) gain (|x1| + |x2|),

u the rounding of the type (2^-8 bf16, 2^-11 f16, 2^-24 f32), least the type's smallest normal number (below 2^-14 f16's
step stays 2^-24, so a rounding is off by up to 2^-25 = 2^-11 2^-14 however small the value); the angle is off by at most 2^-24 up to position 2^26 and in the
reduced argument's rounding to fp32, sincospi's results by 2^-23 each, and three fp32 roundings of 2^-24 follow."""
import math

import pytest
import torch
from test_gpu_kv import DT, i32

pytestmark = pytest.mark.gpu

U = {"bf16": 2.0**-8, "f16": 2.0**-11, "f32": 2.0**-24}


def turned(x, pos, dims, layout, f, gain, back):
    """x [tokens, heads, d] in 64 bits at positions pos, and the bound's (|x1| + |x2|) beside it."""
    y, size = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64)
    angle = (torch.tensor(pos, dtype=torch.float64)[:, None] * f) * (-1 if back else 1)
    c, s = (gain * angle.cos())[:, None], (gain * angle.sin())[:, None]
    i = torch.arange(dims // 2)
    a, b = (i, i + dims // 2) if layout == 0 else (2 * i, 2 * i + 1)
    x1, x2 = x.double()[..., a], x.double()[..., b]
    y[..., a], y[..., b] = x1 * c - x2 * s, x1 * s + x2 * c
    size[..., a] = size[..., b] = abs(gain) * (x1.abs() + x2.abs())
    return y, size


def rows_at(seqs):
    """Positions of all rows, and cu."""
    cu, pos = [0], []
    for p, n in seqs:
        pos += range(p, p + n)
        cu.append(cu[-1] + n)
    return pos, cu


def near(got, x, pos, dims, layout, f, gain=1.0, back=False, typ="f32"):
    ref, size = turned(x, pos, dims, layout, f, gain, back)
    err = (got.cpu().double() - ref).abs() - (U[typ] * ref.abs().clamp(min=torch.finfo(DT[typ]).tiny) + (2.0**-22 + 2.0**-24) * size)
    assert err.amax() <= 0, float(err.amax())
    assert torch.equal(got[..., dims:].cpu(), x[..., dims:])


def plain_f(dims, base=10000.0):
    return base ** (-2 * torch.arange(dims // 2, dtype=torch.float64) / dims)


CASES = [
    # heads of the two tensors, d, dims, type, (position, rows) of each sequence
    (1, 1, 16, 16, "bf16", [(0, 1)]),
    (32, 8, 128, 128, "bf16", [(i * 97, 1) for i in range(64)]),
    (8, 2, 64, 64, "f16", [(0, 100), (31, 0), (5000, 37), (1000000, 3)]),
    (4, 4, 128, 64, "f32", [(7, 300), (65000, 1)]),
    (3, 1, 80, 40, "bf16", [(0, 50)]),
    (5, 2, 66, 22, "f16", [(11, 33), (0, 1)]),
    (2, 1, 30, 30, "f32", [(3, 17)]),
    (2, 2, 7, 6, "bf16", [(100, 9)]),
    (1, 1, 1024, 1024, "f32", [(2**26 - 3, 3)]),
    (12, 12, 256, 2, "bf16", [(5, 40)]),
    (8, 1, 96, 96, "f16", [(i * 13, i % 4) for i in range(300)]),
    (2, 2, 128, 128, "bf16", [(0, 5000)]),
]


@pytest.mark.parametrize("hq,hk,d,dims,typ,seqs", CASES)
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("back", [False, True])
def test_rotate(cuda_ok, hq, hk, d, dims, typ, seqs, layout, back):
    import paper_2608_14648_gb300 as skm

    pos, cu = rows_at(seqs)
    rows = torch.randn(len(pos), hq + hk + 1, d, generator=torch.Generator().manual_seed(1)).to(DT[typ])
    rot = skm.Rotary(dims, layout=layout)
    dev = rows.cuda()
    most = max(n for _, n in seqs)
    args = i32([p for p, _ in seqs]), i32(cu)
    parts = dev[:, :hq], dev[:, hq + 1:]  # as slices of a projection
    got = skm.skm_kv_rotate(rot, *args, parts, most, transpose=back)
    for y, x in zip(got, (rows[:, :hq], rows[:, hq + 1:])):
        assert y.dtype == x.dtype and y.shape == x.shape
        near(y, x, pos, dims, layout, plain_f(dims), back=back, typ=typ)
    one = skm.skm_kv_rotate(rot, *args, parts[1], most, transpose=back)  # a tensor by itself
    assert torch.equal(one, got[1])
    skm.skm_kv_rotate(rot, *args, parts, most, out=parts, transpose=back)  # in place
    assert torch.equal(dev[:, :hq], got[0]) and torch.equal(dev[:, hq + 1:], got[1])
    assert torch.equal(dev[:, hq], rows[:, hq].cuda())


@pytest.mark.parametrize("typ", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("layout", [0, 1])
def test_rotate_any_strides(cuda_ok, typ, layout):
    import paper_2608_14648_gb300 as skm

    flat = torch.randn(40000, generator=torch.Generator().manual_seed(2)).to(DT[typ])
    view = lambda t: t[3:].as_strided((33, 3, 64), (1001, 101, 1))  # noqa: E731
    x, out = view(flat.cuda()), view(torch.zeros(40000, dtype=DT[typ], device="cuda"))
    skm.skm_kv_rotate(skm.Rotary(48, layout=layout), i32([9]), i32([0, 33]), x, 33, out=out)
    near(out, view(flat), list(range(9, 42)), 48, layout, plain_f(48), typ=typ)
    same = x[:1].expand(33, 3, 64)  # one row at many positions
    near(skm.skm_kv_rotate(skm.Rotary(48, layout=layout), i32([9]), i32([0, 33]), same, 33), same.cpu(), list(range(9, 42)), 48, layout,
         plain_f(48), typ=typ)


def test_rows_of_no_sequence_are_left_alone(cuda_ok):
    """Before the first, behind the last, beyond max_tokens; sequences beyond the tensor's end are cut there."""
    import paper_2608_14648_gb300 as skm

    x = torch.randn(50, 2, 32, generator=torch.Generator().manual_seed(3))
    for cu, most, inside in (([4, 20, 30], 100, [(4, 20), (20, 30)]), ([0, 20, 30], 6, [(0, 6), (20, 26)]), ([40, 45, 90], 100, [(40, 45), (45, 50)]),
                             ([0, 0, 0], 5, []), ([60, 70, 80], 5, [])):
        out = torch.full_like(x, 7.0).cuda()
        skm.skm_kv_rotate(skm.Rotary(32), i32([5, 900]), i32(cu), x.cuda(), most, out=out)
        want = torch.full_like(x, 7.0).double()
        for (lo, hi), p in zip(inside, (5, 900)):
            want[lo:hi] = turned(x[lo:hi], list(range(p, p + hi - lo)), 32, 0, plain_f(32), 1.0, False)[0]
        assert torch.allclose(out.cpu().double(), want, rtol=0, atol=1e-5)
        left = torch.ones(50, dtype=torch.bool)
        for lo, hi in inside:
            left[lo:hi] = False
        assert (out.cpu()[left] == 7).all()
    for n in (0, 5):
        empty = torch.empty(n, 2, 32, device="cuda")
        assert skm.skm_kv_rotate(skm.Rotary(32), i32([5]), i32([0, 0]), empty, 0).shape == (n, 2, 32)


def scaled_f(kind, dims, base, factor, trained, low, high):
    f, i = plain_f(dims, base), torch.arange(dims // 2, dtype=torch.float64)
    if kind == "linear":
        return f / factor, 1.0
    if kind == "base":
        return plain_f(dims, base * factor ** (dims / (dims - 2)) if dims > 2 else base), 1.0
    if kind == "index":
        n = lambda t: dims * math.log(trained / (2 * math.pi * t)) / (2 * math.log(base))  # noqa: E731
        first, end = max(math.floor(n(high)), 0), min(math.ceil(n(low)), dims - 1)
        w = ((i - first) / max(end - first, 0.001)).clamp(0, 1)
        return f * (1 - w) + f / factor * w, 0.1 * math.log(factor) + 1 if factor > 1 else 1.0
    w = ((f * trained / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
    return f * w + f / factor * (1 - w), 1.0


@pytest.mark.parametrize("kind", ["linear", "base", "index", "turns"])
@pytest.mark.parametrize("dims,base,factor,trained,low,high", [(128, 10000.0, 16.0, 4096.0, 1.0, 32.0), (64, 500000.0, 8.0, 8192.0, 1.0, 4.0),
                                                              (2, 10000.0, 3.0, 100.0, 0.5, 2.0), (96, 1e6, 0.5, 32.0, 1.0, 40.0)])
def test_scaled_contexts(cuda_ok, kind, dims, base, factor, trained, low, high):
    import paper_2608_14648_gb300 as skm

    scaling = {"linear": skm.ROTARY_LINEAR, "base": skm.ROTARY_BASE, "index": skm.ROTARY_INDEX, "turns": skm.ROTARY_TURNS}[kind]
    rot = skm.Rotary(dims, base=base, scaling=scaling, factor=factor, trained=trained, low=low, high=high)
    f, gain = scaled_f(kind, dims, base, factor, trained, low, high)
    assert rot.gain == pytest.approx(gain, rel=1e-7)
    pos = list(range(10)) + list(range(100000, 100020))
    x = torch.randn(30, 2, dims, generator=torch.Generator().manual_seed(4))
    got = skm.skm_kv_rotate(rot, i32([0, 100000]), i32([0, 10, 30]), x.cuda(), 20)
    near(got, x, pos, dims, 0, f, gain)


@pytest.mark.parametrize("layout", [0, 1])
def test_the_transposed_call_is_the_gradient(cuda_ok, layout):
    """<R x, g> = <x, R' g>, and R' g by differences of <R x, g> (linear: any step gives it)."""
    import paper_2608_14648_gb300 as skm

    rot = skm.Rotary(20, layout=layout, scaling=skm.ROTARY_INDEX, factor=4.0, trained=64.0)
    gen = torch.Generator().manual_seed(5)
    x, g = torch.randn(2, 40, 2, 24, generator=gen).cuda()
    args = i32([3, 500]), i32([0, 15, 40])
    loss = lambda x: (skm.skm_kv_rotate(rot, *args, x, 25).double() * g.double()).sum()  # noqa: E731
    grad = skm.skm_kv_rotate(rot, *args, g, 25, transpose=True).double()
    # each of 40 * 2 * 24 products is off by a few fp32 roundings
    bound = 2.0**-21 * rot.gain * float((x.double().abs() * g.double().abs()).sum() + x.double().norm() * g.double().norm())
    assert abs(float(loss(x) - (x.double() * grad).sum())) <= bound
    for row, head, dim in ((0, 0, 0), (7, 1, 11), (20, 0, 19), (39, 1, 23), (14, 1, 10)):
        up, down = x.clone(), x.clone()
        up[row, head, dim] += 1.0
        down[row, head, dim] -= 1.0
        assert abs(float(loss(up) - loss(down)) / 2 - float(grad[row, head, dim])) <= 2 * bound


def test_in_a_graph_and_on_another_stream(cuda_ok):
    import paper_2608_14648_gb300 as skm

    rot = skm.Rotary(64)
    x = torch.randn(6, 4, 64, device="cuda").to(torch.bfloat16)
    start, cu = i32([5, 100]), i32([0, 2, 6])
    want = skm.skm_kv_rotate(rot, start, cu, x, 4)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    got = skm.skm_kv_rotate(rot, start, cu, x, 4, stream=st)
    st.synchronize()
    assert torch.equal(got, want)
    out = torch.empty_like(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        skm.skm_kv_rotate(rot, start, cu, x, 4, out=out)
    start.add_(1000)  # positions are read on the device
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, skm.skm_kv_rotate(rot, start, cu, x, 4))


def test_negative_positions_turn_back(cuda_ok):
    import paper_2608_14648_gb300 as skm

    x = torch.randn(9, 1, 32, generator=torch.Generator().manual_seed(6))
    got = skm.skm_kv_rotate(skm.Rotary(32), i32([-4]), i32([0, 9]), x.cuda(), 9)
    near(got, x, list(range(-4, 5)), 32, 0, plain_f(32))


def test_infinities_and_nan_stay_in_their_pairs(cuda_ok):
    import paper_2608_14648_gb300 as skm

    x = torch.randn(3, 2, 32, device="cuda")
    want = skm.skm_kv_rotate(skm.Rotary(32), i32([7]), i32([0, 3]), x, 3)
    x[1, 0, 5], x[2, 1, 20] = math.nan, math.inf
    got = skm.skm_kv_rotate(skm.Rotary(32), i32([7]), i32([0, 3]), x, 3)
    hit = torch.zeros(3, 2, 32, dtype=torch.bool, device="cuda")
    hit[1, 0, [5, 21]] = hit[2, 1, [4, 20]] = True
    assert torch.equal(got[~hit], want[~hit]) and not torch.isfinite(got[hit]).any()

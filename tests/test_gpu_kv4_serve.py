"""Rotary positions, the 4-bit cache and its attention as a server runs them: in chunks and
token by token, in graphs, on several streams; and the serving example on them.

Rotated rows are compared with the formula in 64 bits, the cache with its definition on the rows that
entered it (equality), attention with its definition over what the cache holds, each within the bounds
of tests/test_gpu_kv4.py and tests/test_gpu_rotary.py."""
import os
import sys

import pytest
import torch
from test_gpu_kv import DT, i32, make_table
from test_gpu_kv4 import Held4, attend_ref, make_cache, same
from test_gpu_rotary import near, plain_f, rows_at

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def check_step(c, held, table, start, new, rows, turned, out, group, dims, layout, typ, lse=None):
    """One step: rows [tokens, heads_q + 2 heads, d] before the rotation, turned (q, k), out of the attention."""
    heads, hq = c.heads, c.heads * group
    cu = [sum(new[:b]) for b in range(len(new) + 1)]
    pos, _ = rows_at(list(zip(start, new)))
    T, rows = cu[-1], rows.cpu()
    for got, x in zip(turned, (rows[:T, :hq], rows[:T, hq:hq + heads])):
        near(got[:T], x, pos, dims, layout, plain_f(dims), typ=typ)
    held.write(table, start, cu, turned[1][:T].cpu(), rows[:T, hq + heads:])
    same(c, held)
    length = [p + n for p, n in zip(start, new)]
    rounded = typ != "f32" and max(new) * group > 32
    want, ref, tol, ltol, ktol = attend_ref(held, table, length, cu, turned[0][:T].cpu(), group, c.d**-0.5, True, 0, typ, rounded)
    if rounded and typ == "bf16" and lse is None:
        tol = ktol
    assert ((out[:T].cpu().double() - want).abs() - tol).amax() <= 0
    if lse is not None:
        assert ((lse[:T].cpu().double() - ref).abs() - ltol).amax() <= 0


@pytest.mark.parametrize("typ,heads,group,d,dims,layout,page", [
    ("bf16", 2, 4, 64, 64, 0, 32), ("f16", 1, 8, 128, 64, 1, 16), ("f32", 2, 1, 48, 24, 0, 16), ("bf16", 1, 2, 192, 192, 1, 48)])
def test_chunks_and_tokens(cuda_ok, typ, heads, group, d, dims, layout, page):
    import paper_2608_14648_gb300 as skm

    lengths, chunk, steps = [70, 1, 131], 50, 20  # tokens that end blocks, pages and chunks anywhere
    batch, hq = len(lengths), heads * group
    cols = -(-(max(lengths) + steps + 1) // page)
    table = make_table(batch, cols, batch * cols + 1, 4)
    c = make_cache(heads, d, page, batch * cols + 1, 5)
    held, rot, dev = Held4(c), skm.Rotary(dims, layout=layout), table.cuda()
    ws = skm.kv4_workspace(c, batch, hq, batch * chunk, chunk, max(lengths) + steps + 1, dtype={"bf16": skm.DTYPE_BF16, "f16": skm.DTYPE_F16, "f32": skm.DTYPE_F32}[typ])
    g = torch.Generator().manual_seed(6)
    draw = lambda n: torch.randn(n, hq + 2 * heads, d, generator=g).to(DT[typ])  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    done = [0] * batch
    while done != lengths:
        new = [min(chunk, n - p) for p, n in zip(done, lengths)]
        rows = draw(sum(new)).cuda()
        start, cu = i32(done), i32([sum(new[:b]) for b in range(batch + 1)])
        length = start + cu.diff()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            q, k, v = rows.split([hq, heads, heads], dim=1)
            turned = skm.skm_kv_rotate(rot, start, cu, (q, k), chunk)
            skm.skm_kv4_write(c, dev, start, cu, turned[1], v, chunk)
            out, lse = skm.skm_kv4_attend(c, dev, length, cu, turned[0], max(new), max(lengths), want_lse=max(new) % 2 == 1, ws=ws)
        torch.cuda.synchronize()
        check_step(c, held, table, done, new, rows, turned, out, group, dims, layout, typ, lse)
        done = [p + n for p, n in zip(done, new)]

    # a token of each sequence but the last, whose slot is padding: its row of `rows` belongs to no sequence
    rows, start = draw(batch).cuda(), i32(done)
    cu, length = i32(list(range(batch)) + [batch - 1]), torch.empty(batch, dtype=torch.int32, device="cuda")
    turned = tuple(torch.full((batch, n, d), 7.0, dtype=DT[typ], device="cuda") for n in (hq, heads))
    out = torch.full((batch, hq, d), 9.0, dtype=DT[typ], device="cuda")

    def step():
        torch.add(start, cu.diff(), out=length)
        skm.skm_kv_rotate(rot, start, cu, (rows[:, :hq], rows[:, hq:hq + heads]), 1, out=turned)
        skm.skm_kv4_write(c, dev, start, cu, turned[1], rows[:, hq + heads:], 1)
        skm.skm_kv4_attend(c, dev, length, cu, turned[0], 1, cols * page, out=out, ws=ws)
        start.copy_(length)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    new = [1] * (batch - 1) + [0]
    for _ in range(steps):
        rows.copy_(draw(batch))
        graph.replay()
        torch.cuda.synchronize()
        check_step(c, held, table, done, new, rows, turned, out, group, dims, layout, typ)
        for t in turned:
            assert (t[batch - 1:] == 7).all()
        assert (out[batch - 1:] == 9).all()
        done = [p + n for p, n in zip(done, new)]
    assert start.tolist() == done


@pytest.mark.parametrize("typ", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("new", [1, 60])
def test_two_graphs_may_share_a_workspace(cuda_ok, typ, new):
    import paper_2608_14648_gb300 as skm

    calls = []
    c = make_cache(2, 64, 16, 1300, 7)
    ws = skm.kv4_workspace(c, 2, 8, 2 * new, new, 10000, dtype={"bf16": skm.DTYPE_BF16, "f16": skm.DTYPE_F16, "f32": skm.DTYPE_F32}[typ])
    g = torch.Generator(device="cuda").manual_seed(8)
    for seed, length in ((1, [9000, 3]), (2, [4000, 8888])):
        Q = torch.randn(2 * new, 8, 64, generator=g, device="cuda").to(DT[typ])
        args = c, make_table(2, 625, 1300, seed).cuda(), i32([max(n, new) for n in length]), i32([0, new, 2 * new]), Q, new, 10000
        want = skm.skm_kv4_attend(*args, want_lse=True)[0]
        torch.cuda.synchronize()
        out, graph = torch.empty_like(Q), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            skm.skm_kv4_attend(*args, want_lse=True, out=out, ws=ws)
        calls.append((graph, out, want, args))  # (a graph reads its arguments' tensors: they have to live)
    for _ in range(3):
        for graph, out, *_ in calls:
            out.zero_()
            graph.replay()
        torch.cuda.synchronize()
        for _, out, want, _ in calls:
            assert torch.equal(out, want)


def test_calls_on_two_streams_at_once(cuda_ok):
    import paper_2608_14648_gb300 as skm

    heads, d, page, n, batch = 4, 128, 64, 1500, 2
    cols = -(-n // page)
    g = torch.Generator(device="cuda").manual_seed(9)
    rot, cu = skm.Rotary(d), i32([0, n, 2 * n])
    zero, length = i32([0] * batch), i32([n] * batch)
    table = make_table(batch, cols, batch * cols, 10).cuda()
    inputs = [torch.randn(2 * n, 5 * heads, d, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)]
    caches = [make_cache(heads, d, page, batch * cols, 11) for _ in range(2)]

    def job(rows, c, ws):
        q, k, v = rows.split([3 * heads, heads, heads], dim=1)
        q, k = skm.skm_kv_rotate(rot, zero, cu, (q, k), n)
        skm.skm_kv4_write(c, table, zero, cu, k, v, n)
        one = i32([0, 1, 2])
        return (*skm.skm_kv4_attend(c, table, length, cu, q, n, n, want_lse=True, ws=ws),
                *skm.skm_kv4_attend(c, table, length, one, q[:2], 1, n, want_lse=True, ws=ws),
                *skm.skm_kv4_read(c, table, zero, cu, 2 * n, n))

    spaces = [skm.kv4_workspace(c, batch, 3 * heads, 2 * n, n, n) for c in caches]
    want = [[t.clone() for t in job(rows, c, ws)] for rows, c, ws in zip(inputs, caches, spaces)]
    for c in caches:
        c.blocks.fill_(255)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for st, rows, c, ws in zip(streams, inputs, caches, spaces):
        with torch.cuda.stream(st):
            got.append(job(rows, c, ws))
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_sequences_may_share_pages(cuda_ok):
    # one prompt's pages read by several sequences, the same page twice in a table too
    import paper_2608_14648_gb300 as skm

    heads, group, d, page, n = 2, 4, 64, 16, 40
    c = make_cache(heads, d, page, 9, 12)
    held = Held4(c)
    table = torch.tensor([[0, 1, 2, 3], [0, 1, 2, 4], [0, 1, 5, 5]], dtype=torch.int32)
    length = [60, 50, 64]
    Q = torch.randn(3 * n, heads * group, d, generator=torch.Generator().manual_seed(13)).to(torch.bfloat16)
    for m in (1, n):
        cu = [0, m, 2 * m, 3 * m]
        got, lse = skm.skm_kv4_attend(c, table.cuda(), i32(length), i32(cu), Q[:3 * m].cuda(), m, 64, want_lse=True)
        want, ref, tol, ltol, _ = attend_ref(held, table, length, cu, Q[:3 * m], group, d**-0.5, True, 0, "bf16", m * group > 32)
        assert ((got.cpu().double() - want).abs() - tol).amax() <= 0
        assert ((lse.cpu().double() - ref).abs() - ltol).amax() <= 0


@pytest.mark.parametrize("bits,rotary", [(4, False), (4, True), (8, True)])
@pytest.mark.parametrize("batch,prompt,chunk,steps", [(3, 200, 64, 8), (1, 1, 64, 20), (2, 2500, 1000, 3)])
def test_serving_example(cuda_ok, bits, rotary, batch, prompt, chunk, steps):
    import kv_serve

    r = kv_serve.run(batch, prompt, chunk, steps, bits=bits, rotary=rotary)
    assert r["length"] == [max(1, prompt * (b + 1) // batch) + steps for b in range(batch)]
    # 8 bits: as without positions.  4 bits: of 64 normal values the range is 4.7, a step 0.31, an error 0.09 of a value's
    # size; logits of size 1 move the weights as much: 0.13 of what attention adds to the state, twice that for what the
    # generated states carry on, half as much again for luck
    assert r["error"] < (0.1 if bits == 8 else 0.4)
    keys = r["keys"].double()
    assert tuple(keys.shape) == (r["length"][-1], 2, 64) and torch.isfinite(keys).all()
    for h, (C, assign, wcss) in enumerate(r["fits"]):
        d2 = ((keys[:, h] - C.double()[assign.long()]) ** 2).sum()
        assert wcss == pytest.approx(float(d2), rel=1e-4)


def test_capturing_the_4_bit_step_leaves_the_caches_as_they_were(cuda_ok):
    import kv_serve

    lengths = [20, 33, 41]
    server = kv_serve.Server(3, 60, bits=4, rotary=True)
    g = torch.Generator(device="cuda").manual_seed(5)
    server.prompts([torch.randn(n, 256, generator=g, device="cuda").to(torch.bfloat16) for n in lengths], 16)
    was = [lay.cache.blocks.clone() for lay in server.layers]
    server.capture()
    torch.cuda.synchronize()
    assert server.start.tolist() == lengths
    assert all(torch.equal(lay.cache.blocks, w) for lay, w in zip(server.layers, was))

"""The 8-bit key/value cache where sizes, values or events are out of the
ordinary; the bounds are those of test_gpu_kv.py."""
import math

import pytest
import test_gpu_kv
import torch
from test_gpu_kv import DT, check_attend, i32, make_cache, make_table, same, write_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,new,typ", [(128, 20, "bf16"), (96, 32, "f16"), (256, 12, "bf16"), (192, 30, "f16")])
def test_attend_large_batches_of_many_rows(cuda_ok, d, new, typ):
    """1024 sequences take more shared memory beside a large tile than a CTA has: several launches."""
    check_attend(1, 1, d, 16, typ, [(i % 23, new - i % 3) for i in range(1024)])


# heads, group, d, type, row counts of the sequences, tokens they hold at most
GIVES_UP = [
    (8, 4, 64, "bf16", [1] * 1000, 60),      # a warp's stretch holds several units, a CTA's some fifty
    (8, 4, 128, "f16", [1] * 40, 700),       # units of several warps
    (2, 8, 128, "bf16", [1, 1], 40000),      # units of several CTAs
    (2, 1, 64, "f32", [1, 3, 2] * 300, 50),
    (2, 4, 64, "bf16", [1] * 3, 500),        # one CTA a unit
]


@pytest.mark.parametrize("heads,group,d,typ,rows,most", GIVES_UP)
def test_attend_that_gives_up_says_so(cuda_ok, heads, group, d, typ, rows, most):
    """A wait that runs out (an armed SKM_FAULT_WAIT: a warp's first keys never count as arrived, the wait for them ends
    after 1 ms): the status is set and every row is NaN or what it is without the fault, whatever the workspace held."""
    import paper_2608_14648_gb300 as skm

    batch = len(rows)
    g = torch.Generator().manual_seed(21)
    length = [max(n, most - int(torch.randint(0, most // 2, (), generator=g))) for n in rows]
    cols = -(-max(length) // 16)
    c = make_cache(heads, d, 16, batch * cols, 22)
    table = make_table(batch, cols, batch * cols, 23).cuda()
    cu = [0] + torch.tensor(rows).cumsum(0).tolist()
    Q = torch.randn(cu[-1], heads * group, d, generator=g).to(DT[typ]).cuda()
    ws = skm.kv_workspace(c, batch, heads * group, cu[-1], max(rows), max(length), {"bf16": 1, "f16": 2, "f32": 0}[typ])
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def call():
        ws.zero_()  # as a part: no weight, sums 0
        status.zero_()
        out = torch.full_like(Q, 77.0)
        out, lse = skm.skm_kv_attend(c, table, i32(length), i32(cu), Q, max(rows), max(length), want_lse=True, out=out, ws=ws,
                                     status=status)
        return out, lse, int(status)

    want, want_lse, fine = call()
    assert fine == 0 and torch.isfinite(want).all()
    hit = 0
    for stuck in (0, 1, 5, 15, 16, 40, 300, 1000, 1207, 2431):
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
    out, lse = skm.skm_kv_attend(c, *args, Q.cuda(), new, 200, want_lse=True)
    want, want_lse = skm.skm_kv_attend(c, *args, clean.cuda(), new, 200, want_lse=True)
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
    want, want_lse = skm.skm_kv_attend(c, *args, Q.cuda(), new, 200, want_lse=True)
    hit = torch.zeros(2 * new, 4, dtype=torch.bool)
    for row, head, dim in ((0, 1, 63), (new, 0, 0), (2 * new - 1, 3, 17)):
        Q[row, head, dim] = math.nan
        hit[row, head] = True
    out, lse = skm.skm_kv_attend(c, *args, Q.cuda(), new, 200, want_lse=True)
    hit = hit.cuda()
    assert torch.isnan(out[hit]).all() and torch.isnan(lse[hit]).all()
    assert torch.equal(out[~hit], want[~hit]) and torch.equal(lse[~hit], want_lse[~hit])


@pytest.mark.parametrize("new", [1, 8, 100])
@pytest.mark.parametrize("large", [2.0**14, 2.0**20, -1.9921875 * 2.0**21])
def test_attend_bf16_queries_of_unequal_elements(cuda_ok, monkeypatch, new, large):
    """An element far above the others, on a dim where all keys are 0: the logits are the others'.  Elements of 2^-32 of the
    row's largest and more take part exactly, so the bound for exact queries holds."""
    def spoil(c):
        c.k.view(c.pages, c.heads, -1, c.d // 16, 16, 16)[..., 0, :, 0] = 128

    draw = torch.randn

    def randn(*size, **kw):
        x = draw(*size, **kw)
        x = torch.where(x.abs() < 2.0**-10, torch.full_like(x, 2.0**-10), x)
        x[..., 0] = large
        return x

    monkeypatch.setattr(torch, "randn", randn)
    check_attend(1, 4, 64, 16, "bf16", [(90, new), (50, new)], spoil=spoil)


@pytest.mark.parametrize("new", [1, 100])
@pytest.mark.parametrize("size,scale", [(1e-38, 2e37), (1e-39, 2e38), (3e37, 1e-38), (5e37, 1e-38), (0.0, 1.0)])
def test_attend_bf16_queries_at_the_ends_of_the_range(cuda_ok, new, size, scale):
    """Rows of subnormal elements, rows whose largest one is near the largest bf16, rows of zeros."""
    check_attend(1, 4, 64, 16, "bf16", [(90, new), (50, new)], spread=size, scale=scale)


def test_write_and_read_no_rows(cuda_ok):
    import paper_2608_14648_gb300 as skm

    c = make_cache(2, 64, 16, 2, 1)
    table, pos, cu = i32([[0, 1]]), i32([20]), i32([0, 0])
    skm.skm_kv_write(c, table, pos, cu, *torch.empty(2, 0, 2, 64, device="cuda"), 0)
    K, V = skm.skm_kv_read(c, table, pos, cu, 0, 0)
    assert K.shape == V.shape == (0, 2, 64)


@pytest.mark.parametrize("heads,group,d,page,typ,seqs,causal,window", [
    (20, 1, 64, 16, "f16", [(0, 600), (300, 257), (17, 40)], True, 0),      # 180 units of 9 row tiles, ranked by their lengths
    (20, 1, 64, 16, "bf16", [(0, 600), (300, 257), (17, 40)], True, 200),
    (10, 4, 128, 64, "bf16", [(100, 200), (0, 130), (500, 64), (900, 1)], True, 0),  # 160, d = 128
    (16, 1, 256, 32, "bf16", [(0, 300), (200, 129), (1290, 33)], False, 0),  # 144 of 128 rows
    (16, 1, 192, 32, "f16", [(0, 300), (200, 129), (1290, 33), (5, 60)], True, 0),
    (1, 1, 96, 16, "bf16", [(i * 7 % 100, 33 + i % 30) for i in range(300)], True, 0),  # 300 row tiles: too many to rank
    (1, 2, 64, 16, "f16", [(i * 7 % 50, 1 + i % 20) for i in range(1100)], True, 0),  # two launches
])
def test_attend_many_rows_in_several_waves(cuda_ok, heads, group, d, page, typ, seqs, causal, window):
    check_attend(heads, group, d, page, typ, seqs, causal, window)


def test_attend_a_prompt_among_single_tokens(cuda_ok):
    check_attend(4, 4, 128, 64, "bf16", [(300, 1), (700, 300), (40, 1), (1500, 1), (0, 1)] + [(90 * i, 1) for i in range(30)])


@pytest.mark.parametrize("typ,group,new", [("bf16", 8, 1), ("f16", 5, 2), ("f32", 1, 1), ("f32", 2, 3)])
@pytest.mark.parametrize("d", [144, 192, 256])
def test_attend_wide_heads_split_over_the_whole_gpu(cuda_ok, typ, group, new, d):
    """d > 128 in shared stretches: units cut between warps and CTAs, whose sums a lane joins in two vectors."""
    check_attend(2, group, d, 64, typ, [(6000, new), (0, new), (3111, new), (40, new)])
    check_attend(1, group, d, 16, typ, [(i * 11 % 70, new) for i in range(160)])


class HeldRows(test_gpu_kv.Held):
    """Held, for sequences of a call that have no rows."""

    def write(self, table, start, cu, K, V):
        for b, at in enumerate(start):
            rows = slice(cu[b], cu[b + 1])
            if cu[b + 1] > cu[b]:
                super().write(table[b: b + 1], [at], [0, cu[b + 1] - cu[b]], K[rows], V[rows])


@pytest.mark.parametrize("heads,d,page,typ", [(8, 128, 64, "bf16"), (3, 96, 32, "f16"), (2, 256, 16, "f32"), (5, 16, 16, "bf16")])
def test_write_and_read_large_batches(cuda_ok, monkeypatch, heads, d, page, typ):
    """More than 32 sequences: their blocks are placed in rows of the longest's, one or none reached by the others."""
    import paper_2608_14648_gb300 as skm

    monkeypatch.setattr(test_gpu_kv, "Held", HeldRows)
    seqs = [(i * 13 % 50, (i * 29 % 71) * (i % 5 > 0)) for i in range(45)] + [(15, 1), (16, 200), (31, 2)]
    c, table, start, cu, want, most = write_case(heads, d, page, typ, seqs, fused=True)
    same(c, want)
    for dt, code in ((torch.float32, skm.DTYPE_F32), (torch.bfloat16, skm.DTYPE_BF16), (torch.float16, skm.DTYPE_F16)):
        got = skm.skm_kv_read(c, table.cuda(), i32(start), i32(cu), cu[-1], most, code)
        for name, x in zip("kv", got):
            ref = torch.cat([want.values(name, table, b, s, s + n, torch.float32)[0] for b, (s, n) in enumerate(seqs)])
            assert torch.equal(x.cpu(), ref.to(dt))


@pytest.mark.parametrize("grow", [1.0, 1.02, 1.5])
def test_values_of_a_block_that_grows(cuda_ok, grow):
    """Single tokens, each up to `grow` times larger: a value read back is within half a step of every scale that it was rounded
    at, the block's at its own write and each larger one since, and so within (g + 1) / 2 steps of the last one after
    g growths.  (A scale and a ratio are rounded to fp32, a code of up to 127 by 127 2^-23 of a step in all each time.)"""
    import paper_2608_14648_gb300 as skm

    heads, d, n = 2, 64, 48
    c = make_cache(heads, d, 16, 4, 41)
    table = make_table(1, 4, 4, 41).cuda()
    g = torch.Generator().manual_seed(42)
    x = torch.randn(n, 2 * heads, d, generator=g) * grow ** (torch.arange(n) % 16)[:, None, None]
    dev = x.cuda()
    bound = torch.zeros(n, 2, heads, dtype=torch.float64)
    growths = torch.zeros(n, 2, heads)
    scale = torch.zeros(2, heads, dtype=torch.float64)
    for t in range(n):
        skm.skm_kv_write(c, table, i32([t]), i32([0, 1]), dev[t: t + 1, :heads], dev[t: t + 1, heads:], 1)
        was, scale = scale, c.scales[int(table[0, t // 16]), :, 0].T.cpu().double()
        step = (0.5 + 127 * 2.0**-23) * scale
        bound[t] = step
        if t % 16:
            grew = scale > was
            bound[t - t % 16: t] += torch.where(grew, step, torch.zeros(()))
            growths[t - t % 16: t] += grew
    got = torch.stack(skm.skm_kv_read(c, table, i32([0]), i32([0, n]), n, n, skm.DTYPE_F32), 1).cpu().double()
    off = (got - x.view(n, 2, heads, d).double()).abs().amax(-1)
    assert (off <= bound).all()
    last = torch.stack([c.scales[int(p), :, 0].T for p in table[0, :3]]).cpu().double().repeat_interleave(16, 0)
    assert (off <= (growths + 1) * (0.5 + 127 * 2.0**-23) * last).all()
    assert growths.max() >= 2


@pytest.mark.parametrize("typ,new", [("bf16", 1), ("bf16", 20), ("bf16", 100), ("f32", 1)])
def test_attend_value_scales_to_the_limit(cuda_ok, typ, new):
    """Value scales of 2^29 next to blocks of zeros (counted as 2^-80), 2^109 apart: both have their full weights."""
    def spoil(c):
        c.scales[0::3, :, :, 1] = 0.0
        c.v[0::3] = 128
        c.scales[1::3, :, :, 1] = 2.0**29

    check_attend(2, 4, 64, 16, typ, [(300, new), (61, new)], spoil=spoil)

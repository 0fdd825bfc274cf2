"""The 8-bit key/value cache where sizes, values or events are out of the
ordinary; the bounds are those of test_gpu_kv.py."""
import pytest
import torch
from test_gpu_kv import DT, check_attend, i32, make_cache, make_table

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

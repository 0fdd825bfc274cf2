"""The 4-bit key/value cache where weighted sums cancel."""
import pytest
import torch
from test_gpu_kv import DT
from test_gpu_kv4 import scales

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

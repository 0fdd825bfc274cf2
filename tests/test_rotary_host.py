"""Rotary positions: what the host decides (no GPU: the device pointers are fake and never dereferenced)."""
import itertools
from decimal import Decimal, localcontext

import pytest
import torch
from test_kv4_abi import part, rotate, rotary, turns
from test_kv_abi import FAKE, INVALID, UNSUPPORTED, OnDevice, seqs, skm  # noqa: F401


# ---- outputs whose rows share elements

@pytest.mark.parametrize("y_token,y_head", [(256, 63), (63, 4096), (255, 64), (64, 65), (128, 64), (-256, 32), (96, 64), (64 * 2, 64 * 3), (1, 1)])
@pytest.mark.parametrize("sign", [1, -1])
def test_outputs_that_overlap_are_refused(skm, y_token, y_head, sign):  # noqa: F811
    # 4 heads of 64 dims, 10 tokens
    s = seqs(skm, tokens=10, max_tokens=10)
    assert rotate(skm, s=s, rows=[part(skm, y_token=sign * y_token, y_head=y_head)]) == INVALID
    assert b"overlap" in skm.lib().skm_last_error()
    assert rotate(skm, s=s, rows=[part(skm), part(skm, x=5 * FAKE, y=7 * FAKE, y_token=y_token, y_head=sign * y_head)]) == INVALID
    # in place too
    assert rotate(skm, s=s, rows=[part(skm, y=FAKE, x_token=y_token, x_head=y_head, y_token=y_token, y_head=y_head)]) == INVALID


def reaches_launch(skm, s, rows, d=64):  # noqa: F811
    """Whether only the last check, of tokens x heads, refuses the call."""
    return rotate(skm, s=s, rows=rows, d=d) == UNSUPPORTED


def test_outputs_that_do_not_overlap_pass(skm):  # noqa: F811
    # every pair of small strides against the definition: the elements of all rows, counted
    tokens, heads, d = 5, 4, 3
    s, r = seqs(skm, tokens=tokens, max_tokens=tokens), rotary(skm, dims=2)
    for y_token, y_head in itertools.product(range(-16, 17), repeat=2):
        at = [t * y_token + h * y_head + i for t in range(tokens) for h in range(heads) for i in range(d)]
        y = part(skm, y_token=y_token, y_head=y_head, heads=heads)
        got = rotate(skm, s=s, r=r, rows=[y, part(skm, x=None)], d=d)  # the second tensor is refused in any case
        assert got == INVALID
        assert (b"overlap" in skm.lib().skm_last_error()) == (len(set(at)) < len(at)), (y_token, y_head)


def test_limits_of_sizes(skm):  # noqa: F811
    assert rotate(skm, rows=[part(skm, heads=65537)]) == INVALID
    wide = dict(x_token=1 << 30, y_token=1 << 30, heads=65536)
    assert reaches_launch(skm, seqs(skm, tokens=7630, max_tokens=1), [part(skm, **wide)])
    for token in (1 << 62, -(1 << 62)):  # no stride is too large for the check
        assert reaches_launch(skm, seqs(skm, tokens=7630, max_tokens=1), [part(skm, **(wide | dict(y_token=token)))])
    assert not rotate(skm, s=seqs(skm, tokens=0), rows=[part(skm, y_token=1)])  # nothing to do


# ---- rows that require a gradient

class Library:
    """Stands in for the library, whose calls it counts."""

    def __init__(self):
        self.calls = 0

    def __getattr__(self, name):
        def call(*args):
            self.calls += 1
            return 0
        return call


@pytest.mark.parametrize("which", ["x", "y", "out"])
def test_rows_that_require_a_gradient_are_refused(skm, monkeypatch, which):  # noqa: F811
    library = Library()
    monkeypatch.setattr(skm, "lib", lambda: library)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    rot = skm.Rotary.__new__(skm.Rotary)
    rot.index, rot.addrs = 0, (0, 0)
    on = lambda t: OnDevice(t, 0)  # noqa: E731
    ints = lambda *v: on(torch.tensor(v, dtype=torch.int32))  # noqa: E731
    tensor = {n: torch.zeros(3, 2, 64, requires_grad=n == which) for n in ("x", "y", "out")}
    x, y, out = (on(tensor[n]) for n in ("x", "y", "out"))
    args = ints(0), ints(0, 3), (x, y), 3
    with pytest.raises(ValueError, match="history"):
        skm.skm_kv_rotate(rot, *args, out=(out, x))
    assert library.calls == 0
    with torch.no_grad():
        skm.skm_kv_rotate(rot, *args, out=(out, x))
    with torch.inference_mode():
        skm.skm_kv_rotate(rot, *args, out=(out, x))
    assert library.calls == 2


# ---- frequencies

PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899862803482534211707")


@pytest.mark.parametrize("dims,base", [(2, 10000.0), (64, 10000.0), (128, 500000.0), (80, 1e7), (1024, 1.5)])
@pytest.mark.parametrize("kind,factor", [("none", 1.0), ("linear", 8.0), ("linear", 0.3), ("base", 8.0), ("base", 0.7)])
def test_frequencies_to_their_bound(skm, dims, base, kind, factor):  # noqa: F811
    """Against 40 digits.  Half a unit of 2^-64, and of the frequency: the exponent's rounding, |ln f| 2^-53, pow 2^-52, the
    divisions by factor and 2 pi and its constant 2^-53 each; a scaled base of relative error (|ln factor| dims / (dims - 2) + 3)
    2^-53 moves f by 2 i / dims of that."""
    scaling = {"none": skm.ROTARY_NONE, "linear": skm.ROTARY_LINEAR, "base": skm.ROTARY_BASE}[kind]
    rc, got, gain = turns(skm, dims=dims, base=base, scaling=scaling, factor=factor)
    assert rc == 0 and gain == 1.0
    with localcontext() as ctx:
        ctx.prec = 40
        lnb, lnfactor = Decimal(base).ln(), Decimal(factor).ln()
        if kind == "base" and dims > 2:
            lnb += lnfactor * dims / (dims - 2)
        eps, worst = Decimal(2) ** -53, Decimal(0)
        for i, t in enumerate(got):
            lnf = -lnb * 2 * i / dims
            f = lnf.exp() / (Decimal(factor) if kind == "linear" else 1)
            turn = f / (2 * PI)
            off = abs((Decimal(t) / 2**64 - turn + Decimal(1) / 2) % 1 - Decimal(1) / 2)  # (of a circle)
            bound = Decimal(2) ** -65 + turn * eps * (abs(lnf) + 6)
            if kind == "base":
                bound += turn * eps * Decimal(2 * i) / dims * (abs(lnfactor) * dims / max(dims - 2, 1) + 3)
            assert off <= bound, (i, off / bound)
            worst = max(worst, off * 2 * PI * 2**26)
        if kind == "none" or (kind == "linear" and factor >= 1):
            assert worst <= Decimal(2) ** -24  # the angle at position 2^26


def test_slow_frequencies_are_not_good_to_their_last_bits(skm):  # noqa: F811
    # what the units leave of them: a relative bound would not hold
    rc, got, _ = turns(skm, dims=80, base=1e7)
    with localcontext() as ctx:
        ctx.prec = 40
        turn = (-Decimal(1e7).ln() * 78 / 80).exp() / (2 * PI)
        assert Decimal(2) ** -50 < abs(Decimal(got[39]) / 2**64 / turn - 1) <= Decimal(2) ** -65 / turn + Decimal(2) ** -48

"""Refusals of the 4-bit cache's and of the rotary positions' entry points, before any launch (no
GPU: the device pointers are fake and never dereferenced), and the frequencies, which are computed on the host."""
import ctypes
import math

import pytest
import torch
from test_kv_abi import FAKE, INVALID, NO_MEMORY, UNSUPPORTED, OnDevice, attn, seqs, skm  # noqa: F401


def cache(skm, heads=2, d=64, page=32, pages=10, blocks=FAKE):  # noqa: F811
    return skm.KVCache4Ref(heads, d, page, pages, blocks)


def call(skm, what, c, s, a=None, dtype=1, K=FAKE, V=FAKE, ws=FAKE, ws_bytes=1 << 40):  # noqa: F811
    L = skm.lib()
    ref = None if c is None else ctypes.byref(c)
    if what == "write":
        return L.skm_kv4_write(ref, ctypes.byref(s), dtype, K, 256, 64, V, 256, 64, None)
    if what == "read":
        return L.skm_kv4_read(ref, ctypes.byref(s), dtype, K, V, None)
    return L.skm_kv4_attend(ref, ctypes.byref(s), ctypes.byref(a or attn(skm)), ws, ws_bytes, None)


@pytest.mark.parametrize("what", ["write", "read", "attend"])
@pytest.mark.parametrize("change,code", [
    (dict(heads=0), INVALID), (dict(heads=-1), INVALID), (dict(pages=0), INVALID), (dict(d=0), INVALID),
    (dict(page=0), INVALID), (dict(d=72), UNSUPPORTED), (dict(d=272), UNSUPPORTED), (dict(page=24), UNSUPPORTED),
    (dict(heads=1 << 16, pages=1 << 15), UNSUPPORTED), (dict(blocks=None), INVALID), (dict(blocks=FAKE + 8), INVALID),
])
def test_caches_are_checked(skm, what, change, code):  # noqa: F811
    assert call(skm, what, cache(skm, **change), seqs(skm)) == code
    assert skm.lib().skm_last_error()
    assert call(skm, what, None, seqs(skm)) == INVALID


@pytest.mark.parametrize("what", ["write", "read", "attend"])
@pytest.mark.parametrize("change,code", [
    (dict(batch=0), INVALID), (dict(cols=0), INVALID), (dict(tokens=-1), INVALID), (dict(max_tokens=-1), INVALID),
    (dict(table=None), INVALID), (dict(pos=None), INVALID), (dict(cu=None), INVALID),
    (dict(tokens=1 << 30), UNSUPPORTED), (dict(cols=1 << 25), UNSUPPORTED),
])
def test_sequences_are_checked(skm, what, change, code):  # noqa: F811
    assert call(skm, what, cache(skm), seqs(skm, **change)) == code


def test_tensors_are_checked(skm):  # noqa: F811
    c, s = cache(skm), seqs(skm)
    assert call(skm, "write", c, s, dtype=3) == INVALID and call(skm, "read", c, s, dtype=-1) == INVALID
    assert call(skm, "write", c, s, K=None) == INVALID and call(skm, "write", c, s, V=FAKE + 1) == INVALID
    assert call(skm, "read", c, s, K=None, V=None) == INVALID and call(skm, "read", c, s, K=FAKE + 8) == INVALID
    many = seqs(skm, batch=1 << 20, tokens=1 << 29, max_tokens=1 << 29)
    assert call(skm, "write", c, many) == UNSUPPORTED and call(skm, "read", c, many) == UNSUPPORTED


@pytest.mark.parametrize("change", [
    dict(heads_q=0), dict(heads_q=3), dict(dtype=7), dict(window=-1), dict(window=5, causal=0), dict(scale=float("nan")),
    dict(scale=float("inf")), dict(Q=None), dict(out=None), dict(out=FAKE + 8), dict(Q=FAKE + 1), dict(lse=FAKE + 2),
    dict(status=FAKE + 1),
])
def test_attention_is_checked(skm, change):  # noqa: F811
    assert call(skm, "attend", cache(skm), seqs(skm), attn(skm, **change)) == INVALID


def test_attention_refuses_sizes_and_workspaces(skm):  # noqa: F811
    c, long = cache(skm, pages=100000), seqs(skm, cols=100000, max_len=3000000)
    assert call(skm, "attend", c, seqs(skm, max_len=-1)) == INVALID
    assert call(skm, "attend", c, seqs(skm, tokens=1 << 29, max_tokens=1 << 29), attn(skm, heads_q=64)) == UNSUPPORTED
    a = attn(skm)
    size = skm.lib().skm_kv4_attend_workspace_size
    need = size(ctypes.byref(c), ctypes.byref(long), ctypes.byref(a))
    assert 0 < need <= 26 << 20
    assert call(skm, "attend", c, long, a, ws=None) == INVALID
    assert call(skm, "attend", c, long, a, ws=FAKE + 16) == INVALID
    assert call(skm, "attend", c, long, a, ws_bytes=need - 1) == NO_MEMORY
    bad = attn(skm, heads_q=5)
    assert size(ctypes.byref(c), ctypes.byref(long), ctypes.byref(bad)) == ctypes.c_size_t(-1).value


def test_nothing_to_do_is_fine_without_tensors(skm):  # noqa: F811
    c, s = cache(skm), seqs(skm, tokens=0)
    assert call(skm, "write", c, s, K=None, V=None) == 0
    assert call(skm, "read", c, s, K=None, V=None) == 0
    assert call(skm, "attend", c, s, attn(skm, Q=None, out=None), ws=None, ws_bytes=0) == 0


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_a_workspace_serves_smaller_calls(skm, d, dtype):  # noqa: F811
    # each call is stopped by an injected refusal, whose message says what it needs
    c = cache(skm, d=d, pages=100000)
    need_of = skm.lib().skm_kv4_attend_workspace_size
    for group, batch, most, length in [(1, 1, 1, 5000), (1, 40, 3, 700), (8, 3, 2, 90000), (4, 9, 60, 640), (2, 7, 900, 20000),
                                       (1, 200, 3, 300), (1, 60, 9, 1024), (3, 30, 6, 1100)]:
        sizes = dict(cols=100000, tokens=batch * most)
        a = attn(skm, heads_q=2 * group, dtype=dtype)
        need = need_of(ctypes.byref(c), ctypes.byref(seqs(skm, batch=batch, max_tokens=most, max_len=length, **sizes)), ctypes.byref(a))
        for b in {1, 2, batch // 2, batch - 1, batch} & set(range(1, batch + 1)):
            for m in {1, 2, 4, 8, 16, 17, 33, most // 2, most} & set(range(1, most + 1)):
                for n in {1, 600, 641, 2048, 2049, length // 2, length} & set(range(length + 1)):
                    for window in (0, 50, 2500):
                        smaller = seqs(skm, batch=b, max_tokens=m, max_len=n, **sizes)
                        skm.skm_inject_fault(skm.FAULT_WORKSPACE, 1)
                        rc = call(skm, "attend", c, smaller, attn(skm, heads_q=2 * group, dtype=dtype, window=window))
                        skm.skm_inject_fault(skm.FAULT_WORKSPACE, 0)
                        text = skm.lib().skm_last_error().decode()
                        assert rc == NO_MEMORY and int(text.split(",")[1].split()[0]) <= need, (b, m, n, window, text, need)


def test_binding_checks_its_tensors(skm):  # noqa: F811
    c = skm.KVCache4(2, 64, 32, pages=4, device="cpu")
    assert c.blocks.shape == (4, 2, 2, 1152)
    for bad in (c.blocks[:, :1], c.blocks.view(torch.int8), c.blocks[..., :1024], c.blocks.transpose(1, 2)):
        with pytest.raises(ValueError):
            skm.KVCache4(2, 64, 32, bad)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    table, pos, cu = i32(0, 1).view(1, 2), i32(0), i32(0, 3)
    K = torch.zeros(3, 2, 64)
    for bad in (dict(), dict(table=table.long()), dict(start=i32(0, 1)), dict(cu=i32(0)), dict(K=K[:, :1]), dict(K=K.double()),
                dict(V=K[:2]), dict(V=K.half()), dict(K=torch.zeros(3, 64, 2).transpose(1, 2))):
        kw = dict(table=table, start=pos, cu=cu, K=K, V=K, max_tokens=3) | bad
        with pytest.raises(ValueError):  # (the first: the cache is not on a GPU)
            skm.skm_kv4_write(c, **kw)
    with pytest.raises(ValueError):
        skm.skm_kv4_attend(c, table, pos, cu, torch.zeros(3, 4, 32), 3, 10)
    with pytest.raises(ValueError):
        skm.skm_kv4_attend(c, table, pos, cu, K, 3, 10, out=K.half())


# ---- rotary positions


def turns(skm, **change):  # noqa: F811
    kw = dict(dims=8, scaling=0, base=10000.0, factor=2.0, trained=64.0, low=1.0, high=4.0) | change
    out, gain = (ctypes.c_uint64 * 512)(), ctypes.c_float()
    rc = skm.lib().skm_rotary_turns(ctypes.byref(skm.RotaryConfig(*kw.values())), out, ctypes.byref(gain))
    return rc, list(out)[: kw["dims"] // 2], gain.value


@pytest.mark.parametrize("dims,base", [(2, 10000.0), (64, 10000.0), (128, 500000.0), (1024, 1.5)])
def test_frequencies(skm, dims, base):  # noqa: F811
    rc, got, gain = turns(skm, dims=dims, base=base)
    assert rc == 0 and gain == 1.0
    for i, t in enumerate(got):
        f = base ** (-2 * i / dims)
        assert t / 2**64 == pytest.approx(f / (2 * math.pi), rel=2.0**-49)


@pytest.mark.parametrize("change", [
    dict(dims=0), dict(dims=7), dict(dims=-2), dict(dims=1026), dict(scaling=-1), dict(scaling=5), dict(base=1.0), dict(base=0.5),
    dict(base=math.inf), dict(base=math.nan), dict(scaling=1, factor=0.0), dict(scaling=1, factor=-2.0), dict(scaling=2, factor=math.inf),
    dict(scaling=2, factor=1e-9), dict(scaling=2, factor=1e300, dims=4), dict(scaling=3, trained=0.0), dict(scaling=3, low=0.0),
    dict(scaling=4, low=4.0), dict(scaling=4, high=math.inf), dict(scaling=4, trained=math.nan),
])
def test_frequencies_are_checked(skm, change):  # noqa: F811
    assert turns(skm, **change)[0] == INVALID
    assert skm.lib().skm_last_error()
    with pytest.raises(skm.SkmError):
        names = ("dims", "base", "scaling", "factor", "trained", "low", "high")
        kw = dict(dims=8, scaling=0, base=10000.0, factor=2.0, trained=64.0, low=1.0, high=4.0) | change
        skm.skm_rotary_turns(**{k: kw[k] for k in names})


def rotate(skm, s=None, r=None, d=64, dtype=1, rows=None, count=None):  # noqa: F811
    rows = rows if rows is not None else [part(skm)]
    arr = (skm.RotaryRows * max(len(rows), 1))(*rows)
    return skm.lib().skm_kv_rotate(ctypes.byref(s or seqs(skm, table=None, cols=0)), ctypes.byref(r or rotary(skm)), d, dtype, arr,
                                   len(rows) if count is None else count, None)


def rotary(skm, dims=64, layout=0, transpose=0, gain=1.0, turns=FAKE):  # noqa: F811
    return skm.RotaryRef(dims, layout, transpose, gain, turns)


def part(skm, x=FAKE, y=2 * FAKE, x_token=256, x_head=64, y_token=256, y_head=64, heads=4):  # noqa: F811
    return skm.RotaryRows(x, y, x_token, x_head, y_token, y_head, heads, 0)


def test_rotation_is_checked(skm):  # noqa: F811
    for change, code in ((dict(batch=0), INVALID), (dict(tokens=-1), INVALID), (dict(max_tokens=-1), INVALID), (dict(pos=None), INVALID),
                         (dict(cu=None), INVALID), (dict(tokens=1 << 30), UNSUPPORTED), (dict(batch=1 << 30), UNSUPPORTED)):
        assert rotate(skm, s=seqs(skm, **change)) == code
    for change in (dict(dims=0), dict(dims=3), dict(dims=66), dict(layout=2), dict(gain=math.nan), dict(gain=math.inf),
                   dict(turns=None), dict(turns=FAKE + 4)):
        assert rotate(skm, r=rotary(skm, **change)) == INVALID
    for change in (dict(heads=0), dict(heads=1 << 17), dict(x=None), dict(y=None), dict(x=FAKE + 1), dict(y=FAKE + 1),
                   dict(y=FAKE, y_token=512), dict(y=FAKE, y_head=32)):
        assert rotate(skm, rows=[part(skm, **change)]) == INVALID
        assert rotate(skm, rows=[part(skm), part(skm, **change)]) == INVALID
    # rows that would be written twice: no stride, the other tensor's
    for change in (dict(y_token=0), dict(y_head=0)):
        assert rotate(skm, rows=[part(skm, **change)]) == INVALID
    for other in (dict(x=3 * FAKE), dict(x=2 * FAKE, y=3 * FAKE), dict(x=3 * FAKE, y=FAKE)):
        assert rotate(skm, rows=[part(skm), part(skm, **other)]) == INVALID
    assert rotate(skm, d=0) == INVALID and rotate(skm, d=1025) == INVALID and rotate(skm, dtype=3) == INVALID
    assert rotate(skm, count=0) == INVALID and rotate(skm, rows=[part(skm)] * 3) == INVALID
    assert rotate(skm, s=seqs(skm, tokens=1 << 29, max_tokens=1)) == UNSUPPORTED
    L = skm.lib()
    assert L.skm_kv_rotate(None, ctypes.byref(rotary(skm)), 64, 1, ctypes.byref(part(skm)), 1, None) == INVALID
    assert L.skm_kv_rotate(ctypes.byref(seqs(skm)), None, 64, 1, ctypes.byref(part(skm)), 1, None) == INVALID
    assert L.skm_kv_rotate(ctypes.byref(seqs(skm)), ctypes.byref(rotary(skm)), 64, 1, None, 1, None) == INVALID
    # nothing to do is fine without tensors
    for change in (dict(tokens=0), dict(max_tokens=0)):
        assert rotate(skm, s=seqs(skm, **change), rows=[part(skm, x=None, y=None)]) == 0


def test_rotation_binding_checks_its_tensors(skm, monkeypatch):  # noqa: F811
    rot = skm.Rotary(64, device="cpu")
    x = torch.zeros(3, 2, 64)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError, match="not on a GPU"):
        skm.skm_kv_rotate(rot, i32(0), i32(0, 3), x, 3)
    calls = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: calls.append(name) or 0

    monkeypatch.setattr(skm, "lib", Library)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0, raising=False)
    rot.index = 1
    on = lambda t: OnDevice(t, 1)  # noqa: E731
    good = dict(start=on(i32(0)), cu=on(i32(0, 3)), rows=(on(x), on(x)), max_tokens=3, out=(on(x), on(x)))
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    with pytest.raises(ValueError, match="cuda:1.*cuda:0"):
        skm.skm_kv_rotate(rot, **good)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1, raising=False)
    skm.skm_kv_rotate(rot, **good)
    assert calls == ["skm_kv_rotate"]
    for bad in (dict(rows=(on(x), on(x[:2]))), dict(rows=(on(x), on(x.half()))), dict(rows=(on(x), on(x[..., :32]))), dict(rows=()),
                dict(rows=(on(x.double()), on(x.double()))), dict(rows=(on(x), on(torch.zeros(3, 64, 2).transpose(1, 2)))),
                dict(rows=(on(x), x)), dict(out=(on(x),)), dict(out=(on(x), on(x[:, :1]))), dict(start=on(i32(0).long())),
                dict(start=on(i32(0).view(1, 1))), dict(cu=on(i32(0)))):
        with pytest.raises(ValueError):
            skm.skm_kv_rotate(rot, **(good | bad))
    assert len(calls) == 1

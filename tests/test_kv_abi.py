"""Refusals of the key/value cache's entry points, before any launch (no GPU:
the device pointers are fake and never dereferenced)."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def skm():
    from paper_2608_14648_gb300 import build as b

    b.build()
    import paper_2608_14648_gb300 as skm

    return skm


FAKE = 0x1000


def cache(skm, heads=2, d=64, page=32, pages=10, k=FAKE, v=FAKE, scales=FAKE):
    return skm.KVCacheRef(heads, d, page, pages, k, v, scales)


def seqs(skm, batch=3, cols=4, table=FAKE, pos=FAKE, cu=FAKE, tokens=5, max_tokens=2, max_len=100):
    return skm.KVSeqs(batch, cols, table, pos, cu, tokens, max_tokens, max_len)


def attn(skm, heads_q=4, dtype=1, causal=1, window=0, scale=0.1, Q=FAKE, out=FAKE, lse=None, status=None):
    return skm.KVAttn(heads_q, dtype, causal, window, scale, 0, Q, 256, 64, out, lse, status)


def call(skm, what, c, s, a=None, dtype=1, K=FAKE, V=FAKE, ws=FAKE, ws_bytes=1 << 40):
    L = skm.lib()
    if what == "write":
        return L.skm_kv_write(ctypes.byref(c), ctypes.byref(s), dtype, K, 256, 64, V, 256, 64, None)
    if what == "read":
        return L.skm_kv_read(ctypes.byref(c), ctypes.byref(s), dtype, K, V, None)
    return L.skm_kv_attend(ctypes.byref(c), ctypes.byref(s), ctypes.byref(a or attn(skm)), ws, ws_bytes, None)


INVALID, UNSUPPORTED, NO_MEMORY = 1, 2, 4


@pytest.mark.parametrize("what", ["write", "read", "attend"])
@pytest.mark.parametrize("change,code", [
    (dict(heads=0), INVALID), (dict(heads=-1), INVALID), (dict(pages=0), INVALID), (dict(d=0), INVALID),
    (dict(page=0), INVALID), (dict(d=72), UNSUPPORTED), (dict(d=272), UNSUPPORTED), (dict(page=24), UNSUPPORTED),
    (dict(heads=1 << 16, pages=1 << 15), UNSUPPORTED), (dict(k=None), INVALID), (dict(v=None), INVALID),
    (dict(scales=None), INVALID), (dict(k=FAKE + 8), INVALID), (dict(v=FAKE + 1), INVALID), (dict(scales=FAKE + 4), INVALID),
])
def test_caches_are_checked(skm, what, change, code):
    assert call(skm, what, cache(skm, **change), seqs(skm)) == code
    assert skm.lib().skm_last_error()


@pytest.mark.parametrize("what", ["write", "read", "attend"])
@pytest.mark.parametrize("change,code", [
    (dict(batch=0), INVALID), (dict(cols=0), INVALID), (dict(tokens=-1), INVALID), (dict(max_tokens=-1), INVALID),
    (dict(table=None), INVALID), (dict(pos=None), INVALID), (dict(cu=None), INVALID),
    (dict(tokens=1 << 30), UNSUPPORTED), (dict(cols=1 << 25), UNSUPPORTED),
])
def test_sequences_are_checked(skm, what, change, code):
    assert call(skm, what, cache(skm), seqs(skm, **change)) == code


def test_tensors_are_checked(skm):
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
def test_attention_is_checked(skm, change):
    assert call(skm, "attend", cache(skm), seqs(skm), attn(skm, **change)) == INVALID


def test_attention_refuses_sizes_and_workspaces(skm):
    c, long = cache(skm, pages=100000), seqs(skm, cols=100000, max_len=3000000)
    assert call(skm, "attend", c, seqs(skm, max_len=-1)) == INVALID
    assert call(skm, "attend", c, seqs(skm, tokens=1 << 29, max_tokens=1 << 29), attn(skm, heads_q=64)) == UNSUPPORTED
    a = attn(skm)
    need = skm.lib().skm_kv_attend_workspace_size(ctypes.byref(c), ctypes.byref(long), ctypes.byref(a))
    assert 0 < need < 1 << 30
    assert call(skm, "attend", c, long, a, ws=None) == INVALID
    assert call(skm, "attend", c, long, a, ws=FAKE + 16) == INVALID
    assert call(skm, "attend", c, long, a, ws_bytes=need - 1) == NO_MEMORY
    bad = attn(skm, heads_q=5)
    assert skm.lib().skm_kv_attend_workspace_size(ctypes.byref(c), ctypes.byref(long), ctypes.byref(bad)) == ctypes.c_size_t(-1).value


def test_nothing_to_do_is_fine_without_tensors(skm):
    c, s = cache(skm), seqs(skm, tokens=0)
    assert call(skm, "write", c, s, K=None, V=None) == 0
    assert call(skm, "read", c, s) == 0
    assert call(skm, "attend", c, s, attn(skm, Q=None, out=None), ws=None, ws_bytes=0) == 0


def test_binding_checks_its_tensors(skm):
    c = skm.KVCache(2, 64, 32, pages=4, device="cpu")
    assert c.k.shape == (4, 2, 2, 1024) and c.scales.shape == (4, 2, 2, 2)
    with pytest.raises(ValueError):
        skm.KVCache(2, 64, 32, c.k, c.v, c.scales.double())
    with pytest.raises(ValueError):
        skm.KVCache(3, 64, 32, c.k, c.v, c.scales)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    table, pos, cu = i32(0, 1).view(1, 2), i32(0), i32(0, 3)
    K = torch.zeros(3, 2, 64)
    for bad in (dict(table=table.long()), dict(start=i32(0, 1)), dict(cu=i32(0)), dict(K=K[:, :1]), dict(K=K.double()),
                dict(V=K[:2]), dict(V=K.half()), dict(K=torch.zeros(3, 64, 2).transpose(1, 2))):
        kw = dict(table=table, start=pos, cu=cu, K=K, V=K, max_tokens=3) | bad
        with pytest.raises(ValueError):
            skm.skm_kv_write(c, **kw)
    with pytest.raises(ValueError):
        skm.skm_kv_attend(c, table, pos, cu, torch.zeros(3, 4, 32), 3, 10)
    with pytest.raises(ValueError):
        skm.skm_kv_attend(c, table, pos, cu, K, 3, 10, out=K.half())


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_a_workspace_serves_smaller_calls(skm, d, dtype):
    # each call is stopped by an injected refusal, whose message says what it needs
    c = cache(skm, d=d, pages=100000)
    need_of = skm.lib().skm_kv_attend_workspace_size
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


class OnDevice:
    """What the binding asks of a tensor, on a device that need not exist."""

    def __init__(self, t, index):
        self.t, self.index = t, index

    def get_device(self):
        return self.index

    def __getattr__(self, name):
        return getattr(self.t, name)


def test_binding_refuses_another_current_device(skm, monkeypatch):
    # a launch goes to the current device: with the cache on another one its pointers would be foreign there
    calls = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: calls.append(name) or 0

    monkeypatch.setattr(skm, "lib", Library)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0, raising=False)
    c = skm.KVCache(2, 64, 32, pages=4, device="cpu")
    c.index = 1
    on = lambda t: OnDevice(t, 1)  # noqa: E731
    i32 = lambda *x: on(torch.tensor(x, dtype=torch.int32))  # noqa: E731
    table, pos, cu = on(torch.tensor([[0, 1]], dtype=torch.int32)), i32(0), i32(0, 3)
    rows = lambda heads: on(torch.zeros(3, heads, 64))  # noqa: E731
    ops = [lambda: skm.skm_kv_write(c, table, pos, cu, rows(2), rows(2), 3),
           lambda: skm.skm_kv_read(c, table, pos, cu, 3, 3, skm.DTYPE_F32, out=(rows(2), None)),
           lambda: skm.skm_kv_attend(c, table, pos, cu, rows(4), 3, 10, out=rows(4), ws=rows(4))]
    for current, made in ((0, 0), (1, 3)):
        monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current, raising=False)
        for op in ops:
            if current == 1:
                op()
            else:
                with pytest.raises(ValueError, match="cuda:1.*cuda:0"):
                    op()
        assert len(calls) == made


def test_reading_no_rows_is_fine_without_tensors(skm):
    # (an empty tensor has no address)
    for change in (dict(tokens=0), dict(max_tokens=0)):
        assert call(skm, "read", cache(skm), seqs(skm, **change), K=None, V=None) == 0

"""4-bit key/value cache and head norms: what is decided on the host.  No
compute call is made: every call below fails validation or has nothing to do."""
import ctypes
import math

import pytest

from paper_2607_29221_gb300 import build as B
from paper_2607_29221_gb300 import mosaic as M

FAKE = 1 << 40   # never dereferenced
OK, ARG, SHAPE, ALIGN, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3, 4, 6


@pytest.fixture(scope="module")
def lib():
    B.build()
    return M.lib()


def cache(**over):
    d = dict(type=M.KV_Q4, kv_heads=8, head_dim=128, page_size=16, pages=100, seqs=4, table_cols=20, ld_table=20,
             page_stride=8 * 16 * 80, head_stride=16 * 80, slot_stride=80, k=FAKE, v=FAKE, table=FAKE,
             position=FAKE, weight=FAKE)
    d.update(over)
    return M.mosaic_kv_cache(**d)


def attention(lib, c, **over):
    d = dict(q=FAKE, ldq=8192, heads=64, lens=FAKE, max_len=300, first=None, scale=0.1, decay=1.0, out=FAKE,
             ldo=8192, ws=FAKE, ws_bytes=1 << 40)
    d.update(over)
    return lib.mosaic_kv_attention(ctypes.byref(c), *d.values(), None)


def append(lib, c, **over):
    d = dict(qkv=FAKE, ldx=10240, l=4, heads=64, seq=FAKE, slot=FAKE, index=FAKE, rope=None,
             norm=M.mosaic_head_norm(1e-6, None, None), q=FAKE, ldq=8192)
    d.update(over)
    for name in ("rope", "norm"):
        if d[name] is not None:
            d[name] = ctypes.byref(d[name])
    return lib.mosaic_kv_append_norm(None if c is None else ctypes.byref(c), *d.values(), None)


def rows(lib, c, **over):
    d = dict(seq=FAKE, slot=FAKE, l=4, k=FAKE, v=FAKE, ld_token=1024, ld_head=128)
    d.update(over)
    return lib.mosaic_kv_rows(None if c is None else ctypes.byref(c), *d.values(), None)


@pytest.mark.parametrize("over,status", [
    (dict(head_dim=8), SHAPE), (dict(head_dim=80), SHAPE), (dict(head_dim=144), SHAPE), (dict(head_dim=288), SHAPE),
    (dict(k=FAKE + 8), ALIGN), (dict(slot_stride=88), ALIGN), (dict(head_stride=1288), ALIGN),
    (dict(page_stride=10248), ALIGN), (dict(type=3), ARG), (dict(type=5), ARG), (dict(v=None), ARG)])
def test_every_call_refuses_a_bad_cache(lib, over, status):
    c = cache(**over)
    r = ctypes.byref(c)
    assert attention(lib, c) == append(lib, c) == append(lib, c, norm=None) == rows(lib, c) == status
    assert lib.mosaic_kv_attention_workspace(r, 64, 300) == lib.mosaic_kv_evict_workspace(r, 300, 100) == 0


@pytest.mark.parametrize("over,status", [
    (dict(l=-1), SHAPE), (dict(heads=0), SHAPE), (dict(ldx=10239), SHAPE), (dict(ldq=8191), SHAPE),
    (dict(qkv=None), ARG), (dict(q=None), ARG), (dict(seq=None), ARG), (dict(slot=None), ARG), (dict(index=None), ARG),
    (dict(norm=M.mosaic_head_norm(-1e-6, None, None)), ARG), (dict(norm=M.mosaic_head_norm(math.nan, None, None)), ARG),
    (dict(l=0), OK)])
def test_append_with_norms_refuses(lib, over, status):
    for c in (cache(), cache(type=M.KV_BF16, slot_stride=128, head_stride=2048, page_stride=16384)):
        assert append(lib, c, **over) == status
    assert append(lib, None) == rows(lib, None) == ARG


@pytest.mark.parametrize("over,status", [
    (dict(l=-1), SHAPE), (dict(ld_token=127), SHAPE), (dict(ld_head=120), SHAPE), (dict(l=1 << 50), SHAPE),
    (dict(seq=None), ARG), (dict(slot=None), ARG), (dict(k=None), ARG), (dict(v=None), ARG),
    (dict(k=FAKE + 8), ALIGN), (dict(v=FAKE + 2), ALIGN), (dict(ld_token=1028), ALIGN), (dict(ld_head=132), ALIGN),
    (dict(l=0), OK)])
def test_rows_refuses(lib, over, status):
    assert rows(lib, cache(), **over) == status


def test_workspaces_follow_the_arguments(lib):
    c = cache()
    r = ctypes.byref(c)
    need = lib.mosaic_kv_attention_workspace(r, 64, 4000)
    assert need > 0 and lib.mosaic_kv_attention_workspace(r, 60, 4000) == 0
    assert attention(lib, c, max_len=4000, ws_bytes=need - 1) == WORKSPACE
    assert attention(lib, c, heads=8 * 65, ldq=1 << 20, ldo=1 << 20) == UNSUPPORTED
    assert lib.mosaic_kv_evict_workspace(r, 300, 100) > 0


def test_row_bytes(lib):
    """Codes (half a byte a channel), step and base (4 bytes for 32 channels), to 16 bytes."""
    for d in range(0, 300):
        want = -(-(d // 2 + d // 8) // 16) * 16 if d % 32 == 0 and 32 <= d <= 256 else 0
        assert M.mosaic_kv_row_bytes(M.KV_Q4, d) == want
        assert M.mosaic_kv_row_bytes(M.KV_F32, d) == (4 * d if d % 8 == 0 and 8 <= d <= 256 else 0)
    assert M.mosaic_kv_row_bytes(M.KV_BF16, 128) == M.mosaic_kv_row_bytes(M.KV_F16, 128) == 256
    assert M.mosaic_kv_row_bytes(3, 128) == M.mosaic_kv_row_bytes(-1, 128) == 0


def test_python_handles_refuse(lib):
    torch = pytest.importorskip("torch")
    from paper_2607_29221_gb300 import kvcache as KV
    assert KV.row_bytes(128) == 80
    for d in (0, 16, 80, 288):
        with pytest.raises(ValueError, match="multiple of 32"):
            KV.row_bytes(d)
    gain = torch.ones(64)
    n = KV.HeadNorm(64, 1e-5, gain)
    assert n.on(64, -1) is not None                       # host tensors report device -1
    with pytest.raises(ValueError, match="head_dim"):
        n.on(128, -1)
    with pytest.raises(ValueError, match="another device"):
        n.on(64, 0)
    for bad in (dict(eps=-1.0), dict(eps=math.nan), dict(q_gain=torch.ones(63)), dict(k_gain=torch.ones(64).double()),
                dict(q_gain=torch.ones(128)[::2]), dict(k_gain=torch.ones(64, 1))):
        with pytest.raises(ValueError):
            KV.HeadNorm(64, **bad)
    with pytest.raises(ValueError):                       # host tensors
        x = torch.zeros(2, 1, 4, 80, dtype=torch.uint8)
        KV.PagedCache(x, x, torch.zeros(1, 2, dtype=torch.int32))


def test_calls_refuse_while_another_device_is_current(lib, monkeypatch):
    """Host tensors and a library whose calls only count stand in."""
    torch = pytest.importorskip("torch")
    from paper_2607_29221_gb300 import kvcache as KV
    calls = []

    class Lib:
        def __getattr__(self, name):
            return lambda *a: calls.append(name) or 0
    monkeypatch.setattr(M, "_stream", lambda s: 0)
    monkeypatch.setattr(M, "lib", lambda: Lib())
    c = object.__new__(KV.PagedCache)
    c.head_dim, c.kv_heads, c.seqs, c.device, c._ref, c._index = 32, 1, 2, torch.device("cpu"), None, -1
    c._calls, c.k = [lambda *a: calls.append("other") or 0] * 3, torch.zeros(1, dtype=torch.uint8)
    ints, norm = torch.zeros(2, dtype=torch.int32), KV.HeadNorm(32)
    for run, name in ((lambda: c.append(torch.zeros(2, 96), 1, ints, ints, ints, norm=norm), "mosaic_kv_append_norm"),
                      (lambda: c.rows(ints, ints), "mosaic_kv_rows")):
        calls.clear()
        monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
        run()
        assert calls == [name]
        monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
        with pytest.raises(ValueError, match="not the current one"):
            run()
        assert calls == [name]

"""Key/value cache: what is decided on the host (validation, workspace sizes,
rotary frequencies, the page account).  No compute call is made: every call
below fails validation or has nothing to do."""
import ctypes
import math
from fractions import Fraction

import numpy as np
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
    d = dict(type=M.KV_BF16, kv_heads=8, head_dim=128, page_size=16, pages=100, seqs=4, table_cols=20, ld_table=20,
             page_stride=8 * 16 * 128, head_stride=16 * 128, slot_stride=128, k=FAKE, v=FAKE, table=FAKE,
             position=FAKE, weight=FAKE)
    d.update(over)
    return M.mosaic_kv_cache(**d)


BAD_CACHES = [
    (dict(type=3), ARG), (dict(type=-1), ARG), (dict(k=None), ARG), (dict(v=None), ARG), (dict(table=None), ARG),
    (dict(kv_heads=0), SHAPE), (dict(head_dim=0), SHAPE), (dict(head_dim=12), SHAPE), (dict(head_dim=264), SHAPE),
    (dict(page_size=0), SHAPE), (dict(page_size=65537), SHAPE), (dict(pages=0), SHAPE), (dict(seqs=-1), SHAPE),
    (dict(table_cols=0), SHAPE), (dict(ld_table=19), SHAPE),
    (dict(table_cols=1 << 28, ld_table=1 << 28), SHAPE),
    (dict(page_stride=-128), SHAPE), (dict(k=FAKE + 2), ALIGN), (dict(v=FAKE + 8), ALIGN),
    (dict(slot_stride=132), ALIGN), (dict(head_stride=1028), ALIGN), (dict(type=M.KV_F32, page_stride=1022), ALIGN),
]


def attention(lib, c, **over):
    d = dict(q=FAKE, ldq=8192, heads=64, lens=FAKE, max_len=300, first=None, scale=0.1, decay=1.0, out=FAKE,
             ldo=8192, ws=FAKE, ws_bytes=1 << 40)
    d.update(over)
    return lib.mosaic_kv_attention(None if c is None else ctypes.byref(c), *d.values(), None)


def append(lib, c, **over):
    d = dict(qkv=FAKE, ldx=10240, l=4, heads=64, seq=FAKE, slot=FAKE, index=FAKE, rope=None, q=FAKE, ldq=8192)
    d.update(over)
    if d["rope"] is not None:
        d["rope"] = ctypes.byref(d["rope"])
    return lib.mosaic_kv_append(None if c is None else ctypes.byref(c), *d.values(), None)


def evict(lib, c, **over):
    d = dict(lens=FAKE, max_len=300, keep=100, recent_from=None, new_lens=FAKE, ws=FAKE, ws_bytes=1 << 40)
    d.update(over)
    return lib.mosaic_kv_evict(None if c is None else ctypes.byref(c), *d.values(), None)


@pytest.mark.parametrize("over,status", BAD_CACHES)
def test_every_call_refuses_a_bad_cache(lib, over, status):
    c = cache(**over)
    assert attention(lib, c) == append(lib, c) == evict(lib, c) == status
    assert lib.mosaic_kv_attention_workspace(ctypes.byref(c), 64, 300) == 0
    assert lib.mosaic_kv_evict_workspace(ctypes.byref(c), 300, 100) == 0


def test_no_cache_is_an_argument_error(lib):
    assert attention(lib, None) == append(lib, None) == evict(lib, None) == ARG


@pytest.mark.parametrize("over,status", [
    (dict(heads=0), SHAPE), (dict(heads=60), SHAPE), (dict(ldq=8191), SHAPE), (dict(ldo=8191), SHAPE),
    (dict(max_len=-1), SHAPE), (dict(max_len=1 << 30), SHAPE), (dict(heads=8 * 65, ldq=1 << 20, ldo=1 << 20), UNSUPPORTED),
    (dict(scale=math.inf), ARG), (dict(scale=math.nan), ARG), (dict(decay=math.nan), ARG), (dict(q=None), ARG),
    (dict(out=None), ARG), (dict(lens=None), ARG), (dict(ws=None), ARG), (dict(ws=FAKE + 8), ALIGN),
    (dict(ws_bytes=100), WORKSPACE)])
def test_attention_refuses(lib, over, status):
    assert attention(lib, cache(), **over) == status


def test_attention_needs_positions_for_a_lower_bound(lib):
    assert attention(lib, cache(position=None), first=FAKE) == ARG
    assert attention(lib, cache(seqs=0)) == OK


@pytest.mark.parametrize("over,status", [
    (dict(l=-1), SHAPE), (dict(heads=0), SHAPE), (dict(ldx=10239), SHAPE), (dict(ldq=8191), SHAPE),
    (dict(qkv=None), ARG), (dict(q=None), ARG), (dict(seq=None), ARG), (dict(slot=None), ARG),
    (dict(index=None), ARG), (dict(l=0), OK)])
def test_append_refuses(lib, over, status):
    assert append(lib, cache(), **over) == status


@pytest.mark.parametrize("over,status", [
    (dict(rot_dim=136), SHAPE), (dict(rot_dim=12), SHAPE), (dict(rot_dim=-8), SHAPE), (dict(ldp=3), SHAPE),
    (dict(axes=0), ARG), (dict(axes=5), ARG), (dict(interleaved=2), ARG), (dict(turns=None), ARG),
    (dict(pos=None), ARG)])
def test_append_refuses_a_bad_rope(lib, over, status):
    d = dict(rot_dim=128, interleaved=0, axes=1, turns=FAKE, axis=None, pos=FAKE, ldp=4)
    d.update(over)
    assert append(lib, cache(), rope=M.mosaic_rope(**d)) == status


@pytest.mark.parametrize("over,status", [
    (dict(keep=0), SHAPE), (dict(max_len=-1), SHAPE), (dict(lens=None), ARG), (dict(new_lens=None), ARG),
    (dict(ws=None), ARG), (dict(ws=FAKE + 2), ALIGN), (dict(ws_bytes=64), WORKSPACE)])
def test_evict_refuses(lib, over, status):
    assert evict(lib, cache(), **over) == status


def test_evict_needs_weights_and_positions(lib):
    assert evict(lib, cache(weight=None)) == ARG
    assert evict(lib, cache(position=None), recent_from=FAKE) == ARG
    assert evict(lib, cache(seqs=0)) == OK


def test_workspaces_follow_the_arguments(lib):
    c = cache()
    r = ctypes.byref(c)
    assert lib.mosaic_kv_attention_workspace(r, 64, 300) > 0
    assert lib.mosaic_kv_attention_workspace(r, 60, 300) == lib.mosaic_kv_attention_workspace(r, 64, -1) == 0
    assert lib.mosaic_kv_evict_workspace(r, 300, 0) == 0
    bare = cache(weight=None)
    assert lib.mosaic_kv_attention_workspace(ctypes.byref(bare), 64, 300) < lib.mosaic_kv_attention_workspace(r, 64, 300)


@pytest.mark.parametrize("rot,base", [(2, 10000.0), (64, 10000.0), (128, 500000.0), (256, 1.5)])
def test_rope_turns(lib, rot, base):
    """Against rationals: the frequency is pow()'s double (1 ulp), pi to 60 digits, so the rounding to 2^-64 turns
    is off by the double's 2^-52 relative and half a unit."""
    pi = Fraction(314159265358979323846264338327950288419716939937510582097494, 10 ** 59)
    got = M.mosaic_rope_turns(rot, base)
    for j, t in enumerate(got):
        want = Fraction(base ** (-2.0 * j / rot)) / (2 * pi) * 2 ** 64
        assert abs(int(t) - want) <= want / 2 ** 51 + 1


@pytest.mark.parametrize("rot,base,status", [(0, 1e4, SHAPE), (3, 1e4, SHAPE), (258, 1e4, SHAPE), (64, 1.0, ARG),
                                             (64, math.inf, ARG), (64, math.nan, ARG)])
def test_rope_turns_refuses(lib, rot, base, status):
    buf = np.zeros(200, np.uint64)
    assert lib.mosaic_rope_turns(rot, base, buf.ctypes.data_as(ctypes.c_void_p)) == status
    assert lib.mosaic_rope_turns(64, 1e4, None) == ARG


def test_python_handles_refuse(lib):
    torch = pytest.importorskip("torch")
    from paper_2607_29221_gb300 import kvcache as KV
    with pytest.raises(ValueError):
        KV.Rope(12, device="cpu")
    with pytest.raises(ValueError):
        KV.Rope(64, sections=[10, 10], device="cpu")
    rope = KV.Rope(64, sections=[8, 12, 12], device="cpu")
    assert rope.axis.tolist() == [0] * 8 + [1] * 12 + [2] * 12
    with pytest.raises(ValueError):
        rope.at(torch.zeros(2, 5, dtype=torch.int32))
    with pytest.raises(ValueError):
        rope.at(torch.zeros(3, 5, dtype=torch.int64))
    r = rope.at(torch.zeros(3, 5, dtype=torch.int32))
    assert (r.rot_dim, r.axes, r.ldp) == (64, 3, 5)
    k = torch.zeros(2, 1, 4, 8)
    with pytest.raises(ValueError):   # host tensors
        KV.PagedCache(k, k, torch.zeros(1, 2, dtype=torch.int32))


def test_page_table_accounts_for_its_pages(lib):
    pytest.importorskip("torch")
    from paper_2607_29221_gb300 import kvcache as KV
    t = KV.PageTable(3, 4, 7, 16, device="cpu")        # pages 1..6 to give
    t.resize(0, 17)
    t.resize(2, 64)
    assert [len(o) for o in t.owned] == [2, 0, 4] and not t.free
    assert t.table[0, :2].tolist() == t.owned[0] and t.table[2].tolist() == t.owned[2]
    with pytest.raises(ValueError):
        t.resize(1, 1)
    t.resize(2, 16)
    assert len(t.free) == 3
    t.resize(1, 48)
    pages = sum(t.owned, [])
    assert sorted(pages) == [1, 2, 3, 4, 5, 6] and 0 not in pages
    with pytest.raises(ValueError):
        t.resize(0, 65)
    t.resize(0, 0)
    assert t.owned[0] == []


def test_rows_that_share_memory_have_no_leading_dimension(lib):
    """An expanded or overlapping view must not be given a stride that walks past its storage."""
    torch = pytest.importorskip("torch")
    from paper_2607_29221_gb300 import kvcache as KV
    rope = KV.Rope(64, sections=[8, 12, 12], device="cpu")
    pos = torch.arange(5, dtype=torch.int32)
    for bad in (pos[None].expand(3, 5), torch.arange(9, dtype=torch.int32).as_strided((3, 5), (2, 1))):
        with pytest.raises(ValueError, match="share memory"):
            rope.at(bad)
    assert rope.at(pos[None].expand(3, 5).contiguous()).ldp == 5
    assert rope.at(torch.arange(24, dtype=torch.int32).reshape(3, 8)[:, :5]).ldp == 8
    one = KV.Rope(64, device="cpu")
    assert one.at(pos).ldp == 5 and one.at(pos[:1]).ldp == 1
    for bad in (torch.zeros(1, 4, 8).expand(3, 4, 8), torch.zeros(64).as_strided((3, 4, 8), (16, 8, 1))):
        with pytest.raises(ValueError, match="share memory"):
            KV._rows(bad, "out", 3, 4, 8, -1)
    assert KV._rows(torch.zeros(1, 4, 8), "q", 1, 4, 8, -1) == 32
    assert KV._rows(torch.zeros(0, 4, 8), "q", 0, 4, 8, -1) == 32
    assert KV._rows(torch.zeros(3, 40)[:, 8:].unflatten(1, (4, 8)), "q", 3, 4, 8, -1) == 40


def test_append_refuses_a_rope_on_another_device(lib, monkeypatch):
    """Host pointers must not reach a kernel.  The handle is a stand-in on host tensors whose library calls only
    count."""
    torch = pytest.importorskip("torch")
    from paper_2607_29221_gb300 import kvcache as KV
    monkeypatch.setattr(M, "_stream", lambda s: 0)
    c, calls = object.__new__(KV.PagedCache), []
    c.head_dim, c.kv_heads, c.device, c._ref = 8, 1, torch.device("cpu"), None
    c._calls = [lambda *a: calls.append(a) or 0] * 3
    c._index = 0                                     # the cache's device is cuda:0; host tensors report -1
    rope, at = KV.Rope(8, device="cpu"), torch.zeros(2, dtype=torch.int32)

    class OnDevice(torch.Tensor):                    # host tensors that say that they lie on cuda:0
        def get_device(self):
            return 0
    ints, qkv = at.as_subclass(OnDevice), torch.zeros(2, 24).as_subclass(OnDevice)
    with pytest.raises(ValueError, match="another device"):
        c.append(qkv, 1, ints, ints, ints, rope=rope, pos=at)
    assert not calls


@pytest.mark.parametrize("call", ["append", "attend", "evict"])
def test_calls_refuse_while_another_device_is_current(lib, monkeypatch, call):
    """The stream is the current device's: a launch there would run on the wrong GPU.  Host tensors and library
    calls that only count stand in."""
    torch = pytest.importorskip("torch")
    from paper_2607_29221_gb300 import kvcache as KV
    monkeypatch.setattr(M, "_stream", lambda s: 0)
    c, calls = object.__new__(KV.PagedCache), []
    c.head_dim, c.kv_heads, c.seqs, c.device, c._ref, c._index = 8, 1, 2, torch.device("cpu"), None, -1
    c._calls = [lambda *a: calls.append(a) or 0] * 3
    c._bytes = lambda *a: 0
    ints = torch.zeros(2, dtype=torch.int32)
    run = {"append": lambda: c.append(torch.zeros(2, 24), 1, ints, ints, ints),
           "attend": lambda: c.attend(torch.zeros(2, 1, 8), ints, 5), "evict": lambda: c.evict(ints, 5, 2)}[call]
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    run()
    assert len(calls) == 1
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(ValueError, match="not the current one"):
        run()
    assert len(calls) == 1


@pytest.mark.parametrize("slots,status", [((1 << 31) - 1, SHAPE), ((1 << 31) - 1023, SHAPE), ((1 << 31) - 1024, OK)])
def test_slots_are_counted_in_31_bits(lib, slots, status):
    """A unit of slots that begins inside a sequence must end below 2^31 too.  No compute call is made: the refused
    calls fail validation, and an accepted cache is only asked for its workspace."""
    c = cache(kv_heads=1, head_dim=8, page_size=1, table_cols=slots, ld_table=slots, page_stride=8, head_stride=8,
              slot_stride=8)
    r = ctypes.byref(c)
    assert (lib.mosaic_kv_evict_workspace(r, slots, 5) > 0) == (status == OK)
    assert (lib.mosaic_kv_attention_workspace(r, 1, slots) > 0) == (status == OK)
    if status != OK:
        assert attention(lib, c, heads=1, ldq=8, ldo=8) == append(lib, c, heads=1) == evict(lib, c) == status


def test_a_cache_without_sequences_needs_no_table(lib):
    c = cache(seqs=0, table=None)
    assert attention(lib, c) == evict(lib, c) == append(lib, c, l=0) == OK
    assert lib.mosaic_kv_evict_workspace(ctypes.byref(c), 300, 100) == 0


@pytest.mark.parametrize("given", [False, True])
def test_a_layer_keeps_no_qkv_rows_past_its_attention(monkeypatch, given):
    """The largest intermediate of a pass but one: its memory is free for the linears that follow.  The layer's parts
    are stand-ins on host tensors."""
    torch = pytest.importorskip("torch")
    import weakref
    from paper_2607_29221_gb300 import decoder as D
    layer, seen = object.__new__(D.SecureDecoderLayer), []
    layer.s = D.LayerShape(hidden=8, n_heads=2, n_kv=1, head_dim=4, ffn=8)
    monkeypatch.setattr(D, "rmsnorm", lambda x, eps: x * 1.0)
    monkeypatch.setattr(D, "swiglu", lambda gu, ffn: gu[:, :ffn] * 1.0)

    def linear(i, x, masks, mark, compose):
        if i == 1:
            assert seen[0]() is None
        y = torch.ones(x.shape[0], (16, 8, 16, 8)[i])
        seen.append(weakref.ref(y))
        return y
    layer._linear = linear
    attend = (lambda qkv: qkv[:, :8] * 2.0) if given else None
    y = layer.forward(torch.ones(3, 8), masks=[None] * 4, attend=attend)
    assert y.shape == (3, 8) and len(seen) == 4

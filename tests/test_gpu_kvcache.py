"""Key/value cache on the GPU: append, attention of one token and eviction
against plain implementations in 64 bits (a sequence and head at a time).

Tolerances, set from the number formats before any run:

  attention  a product carried to 22 bits and summed in fp32 over at most 256
             channels moves a score by at most E = 2^-20 scale sum |q_d k_d|;
             a probability by 2 E relative, and exp, the sums and the join add
             at most 2^-19: |d out| <= (2 E + 2^-19) sum p |v|, and
             |d weight| <= (2 E + 2^-19) weight.
  append     phase 2^-25 turns, sine and cosine 2 ulp, three roundings:
             2^-20 (|a| + |b|) for a pair, and the cache's own rounding
             (2^-8 or 2^-11 relative).
  eviction   exact.
"""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2607_29221_gb300 import build
    build.build()
    yield


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def make(lens, kv, dim, page, typ, layout="head", seed=0, cols=None, poison=True, gap=0):
    """A cache whose slots in use hold N(0, 1); everything else holds NaN, and
    table entries past a sequence's pages are no pages at all."""
    from paper_2607_29221_gb300 import kvcache as KV
    g = gen(seed)
    need = [-(-n // page) for n in lens]
    cols = max(1, max(need)) if cols is None else cols
    pages = sum(need) + 2
    order = torch.randperm(pages, generator=g, device="cuda").tolist()
    table = torch.full((len(lens), cols + gap), 0x7fffffff, dtype=torch.int32, device="cuda")[:, :cols]
    table[::2] = -1
    at = 0
    shape = (pages, kv, page, dim)
    pools = []
    used = torch.zeros(pages, page, dtype=torch.bool, device="cuda")
    for i, n in enumerate(lens):
        ids = torch.tensor(order[at: at + need[i]], dtype=torch.int32, device="cuda")
        table[i, : need[i]] = ids
        at += need[i]
        if n:
            u = torch.arange(need[i] * page, device="cuda").reshape(-1, page) < n
            used[ids.long()] = u
    for _ in range(2):
        x = torch.randn(shape, generator=g, device="cuda").to(TYPES[typ])
        if poison:
            x[~used[:, None, :].expand(-1, kv, -1)] = math.nan
        if layout == "token":
            x = x.transpose(1, 2).contiguous().transpose(1, 2)
        elif layout == "padded":         # rows of a wider buffer
            wide = torch.full((pages, kv, page, dim + 16), math.nan, dtype=x.dtype, device="cuda")
            wide[..., 8: 8 + dim] = x
            x = wide[..., 8: 8 + dim]
        pools.append(x)
    weight = torch.rand(shape[:3], generator=g, device="cuda") * 3
    position = torch.zeros(shape[:3], dtype=torch.int32, device="cuda")
    c = KV.PagedCache(*pools, table, position=position, weight=weight)
    c.used, c.lens = used, lens
    return c


def rows(c, pool, i, n):
    """Slots 0..n of sequence i: kv x n (x dim), in 64 bits."""
    page = c.k.shape[2]
    ids = c.table[i, : -(-n // page)].long()
    x = pool[ids].transpose(0, 1)
    return x.reshape(x.shape[0], -1, *x.shape[3:])[:, :n].double()


def reference(c, q, scale, first=None, decay=1.0):
    """out, its tolerance, weight, its tolerance (dicts by sequence for the weights)."""
    b, heads, d = q.shape
    out = torch.zeros(b, heads, d, dtype=torch.float64, device="cuda")
    tol = torch.zeros_like(out)
    weights = {}
    for i, n in enumerate(c.lens):
        if not n:
            continue
        k, v = rows(c, c.k, i, n), rows(c, c.v, i, n)
        qi = q[i].double().reshape(c.kv_heads, -1, d)
        s = torch.einsum("hgd,hnd->hgn", qi, k) * scale
        err = 2.0 ** -20 * abs(scale) * torch.einsum("hgd,hnd->hgn", qi.abs(), k.abs())
        if first is not None:
            s = s.masked_fill(rows(c, c.position, i, n)[:, None] < int(first[i]), -math.inf)
        p = torch.softmax(s, 2)
        p = torch.where(torch.isnan(p) & (s == -math.inf).all(2, keepdim=True), 0.0, p)
        rel = 2 * err.amax(2, keepdim=True) + 2.0 ** -19
        out[i] = torch.einsum("hgn,hnd->hgd", p, v).reshape(heads, d)
        tol[i] = (rel * torch.einsum("hgn,hnd->hgd", p, v.abs())).reshape(heads, d)
        w = rows(c, c.weight, i, n) * decay + p.sum(1)
        weights[i] = (w, w.abs() * rel.amax(1) + 1e-30)
    return out, tol, weights


CASES = [
    # lens, heads, kv, dim, page, layout
    ([1], 1, 1, 8, 1, "head"),
    ([1, 0, 2], 8, 8, 128, 16, "head"),
    ([63, 64, 65, 127, 128, 129, 1, 0], 64, 8, 128, 16, "head"),
    ([255, 256, 257, 513], 28, 4, 128, 32, "token"),
    ([1000, 3, 77, 0, 640], 24, 8, 64, 20, "token"),
    ([333, 1025], 12, 12, 80, 7, "padded"),
    ([2049, 31], 32, 2, 96, 64, "head"),
    ([700, 1, 15, 16, 17], 3, 1, 256, 8, "head"),
    ([130, 513], 64, 1, 40, 3, "head"),
    ([4100], 17, 1, 128, 128, "head"),
    ([20011, 5], 8, 1, 128, 16, "head"),
]


@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("window", [False, True])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention(case, window, typ):
    lens, heads, kv, dim, page, layout = CASES[case]
    c = make(lens, kv, dim, page, typ, layout, seed=case, gap=3)
    g = gen(100 + case)
    q = torch.randn(len(lens), heads, dim, generator=g, device="cuda") * 1.5
    first = None
    if window:   # scattered positions; the second sequence has no live slot
        c.position.copy_(torch.randint(0, 1000, c.position.shape, generator=g, device="cuda"))
        first = torch.full((len(lens),), 300, dtype=torch.int32, device="cuda")
        first[1:2] = 1000
    scale, decay = dim ** -0.5, 0.75
    want, tol, weights = reference(c, q, scale, first, decay)
    before = c.weight.clone()
    out = c.attend(q, torch.tensor(lens, dtype=torch.int32, device="cuda"), max(lens), first=first, decay=decay)
    assert torch.isfinite(out).all()
    assert ((out.double() - want).abs() <= tol).all(), float(((out.double() - want).abs() / (tol + 1e-300)).max())
    for i, n in enumerate(lens):
        if not n or (window and i == 1):
            assert (out[i] == 0).all()
        if n:
            w, wt = weights[i]
            got = rows(c, c.weight, i, n)
            assert ((got - w).abs() <= wt).all(), float(((got - w).abs() / wt).max())
    mark = c.used[:, None, :].expand_as(before)
    assert torch.equal(c.weight[~mark], before[~mark])   # nothing else is written


@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("seqs,most,heads,kv,dim,page,layout,window", [
    (20, 1100, 64, 8, 128, 16, "head", False),      # shared jobs, two heads a unit
    (40, 1200, 24, 8, 64, 8, "token", True),        # four
    (44, 1030, 16, 8, 128, 5, "head", True),        # four, copied by lanes
    (36, 1500, 32, 8, 128, 32, "padded", False),    # four, boxes of several heads
    (48, 300, 24, 8, 128, 64, "head", True),        # whole jobs, two heads a unit
    (100, 130, 16, 8, 128, 16, "token", False),     # four
    (24, 90, 64, 32, 64, 128, "head", True),
    (70, 1100, 24, 2, 64, 16, "head", False),       # 12 query heads a key/value head
    (6, 1200, 40, 1, 64, 16, "head", True),         # 40
    (9, 200, 4, 2, 8, 16, "head", False),           # rows shorter than a copy's 128 bytes
    (30, 1050, 12, 4, 24, 8, "token", True),
    (5, 1300, 20, 2, 256, 8, "head", False),
])
def test_attention_of_many_sequences(seqs, most, heads, kv, dim, page, layout, window, typ):
    """The ways in which jobs are shared out: heads a unit, whole jobs, boxes."""
    lens = [(most * (i + 1) // seqs) if i % 7 != 3 else 0 for i in range(seqs)]
    c = make(lens, kv, dim, page, typ, layout, seed=seqs)
    g = gen(seqs + 1)
    q = torch.randn(seqs, heads, dim, generator=g, device="cuda") * 1.5
    first = None
    if window:     # most of the units, some heads and some sequences have no live slot
        c.position.copy_(torch.randint(0, 1000, c.position.shape, generator=g, device="cuda"))
        c.position[:, 0] //= 4
        first = torch.full((seqs,), 250, dtype=torch.int32, device="cuda")
        first[2::5] = 998
        first[4::5] = 1000
    want, tol, weights = reference(c, q, dim ** -0.5, first, 0.5)
    out = c.attend(q, torch.tensor(lens, dtype=torch.int32, device="cuda"), most, first=first, decay=0.5)
    assert ((out.double() - want).abs() <= tol).all(), float(((out.double() - want).abs() / (tol + 1e-300)).max())
    for i, n in enumerate(lens):
        if n:
            w, wt = weights[i]
            assert ((rows(c, c.weight, i, n) - w).abs() <= wt).all(), i
    from paper_2607_29221_gb300 import mosaic as M
    M.mosaic_device_status()


@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
def test_attention_of_strided_rows_on_another_stream_in_a_graph(typ):
    """q and out rows of wider buffers, a stream of its own, no weights, a
    max_len beyond every length; then a replay with other lengths."""
    lens = [300, 5, 129]
    c = make(lens, 2, 128, 16, typ, cols=40)
    c2 = type(c)(c.k, c.v, c.table, position=c.position)
    c2.lens = lens
    g = gen(3)
    wide = torch.randn(3, 16 * 128 + 36, generator=g, device="cuda")
    q = wide[:, 5: 5 + 16 * 128].unflatten(1, (16, 128))
    buf = torch.full((3, 16 * 128 + 7), 9.0, device="cuda")
    out = buf[:, 3: 3 + 16 * 128].unflatten(1, (16, 128))
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        c2.attend(q, n, 640, out=out)
    s.synchronize()
    want, tol, _ = reference(c, q, 128 ** -0.5)
    assert ((out.double() - want).abs() <= tol).all()
    assert (buf[:, :3] == 9).all() and (buf[:, 3 + 16 * 128:] == 9).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c2.attend(q, n, 640, out=out)
    c.lens = [64, 1, 128]
    n.copy_(torch.tensor(c.lens, dtype=torch.int32))
    graph.replay()
    torch.cuda.synchronize()
    want, tol, _ = reference(c, q, 128 ** -0.5)
    assert ((out.double() - want).abs() <= tol).all()


@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
def test_attention_of_extreme_values(typ):
    """Large scores (one slot takes everything), equal ones, a live NaN, a live
    infinity (counts as NaN), negative zeros and a steep softmax."""
    lens = [200] * 6
    c = make(lens, 1, 64, 16, typ, seed=5, poison=False)
    q = torch.randn(6, 4, 64, generator=gen(6), device="cuda")
    page = lambda i, s: (int(c.table[i, s // 16]), 0, s % 16)
    c.k[page(0, 77)] = (q[0, 0] * 40).to(c.k.dtype)              # a score far above the others
    q[1] = 0.0                                                   # equal scores
    c.k[page(2, 3)] = math.nan                                   # one score NaN: every output
    c.v[page(3, 199)] = math.inf                                 # an infinite value
    c.k[page(4, 9)] = -0.0
    q[4, 1] = -0.0
    q[5] *= 1e4 if typ != "f16" else 1e3                         # a steep softmax
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    want, tol, _ = reference(c, q, 0.125)
    out = c.attend(q, n, 200)
    assert torch.isnan(out[2]).all()
    assert not torch.isfinite(out[3]).any()
    for i in (0, 1, 4):
        assert ((out[i].double() - want[i]).abs() <= tol[i]).all(), i
    assert torch.isfinite(out[5]).all()
    top = torch.einsum("hd,nd->hn", q[5].double(), rows(c, c.k, 5, 200)[0]).argmax(1)
    assert torch.allclose(out[5], rows(c, c.v, 5, 200)[0][top].float(), rtol=2e-3, atol=2e-3)


def test_attention_without_lengths():
    """All lengths zero, negative or beyond max_len and the table (clamped)."""
    c = make([40, 40, 40], 2, 64, 16, "bf16")
    q = torch.randn(3, 4, 64, generator=gen(1), device="cuda")
    zero = c.attend(q, torch.tensor([0, -5, 0], dtype=torch.int32, device="cuda"), 40)
    assert (zero == 0).all()
    none = c.attend(q, torch.tensor([7, 7, 7], dtype=torch.int32, device="cuda"), 0)
    assert (none == 0).all()
    c.lens = [33, 33, 33]
    c.weight.zero_()
    want, tol, _ = reference(c, q, 0.125)
    out = c.attend(q, torch.tensor([1 << 30, 33, 40], dtype=torch.int32, device="cuda"), 33)
    assert ((out.double() - want).abs() <= tol).all()


def test_attention_repeats_bit_for_bit():
    lens = [5000, 100, 0, 64, 3001]
    c = make(lens, 4, 128, 16, "bf16", seed=9)
    q = torch.randn(5, 32, 128, generator=gen(2), device="cuda")
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    start = c.weight.clone()
    first = None
    for _ in range(3):
        c.weight.copy_(start)
        got = (c.attend(q, n, 5000), c.weight.clone())
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(first, got))


def test_scratch_of_streams_threads_and_graphs_is_apart():
    """Calls on several streams and host threads and replays of a graph, all at
    once, with scratch that grows: each gives what it gives alone."""
    import threading
    lens = [3000, 1700, 40, 2100]
    c = make(lens, 8, 64, 16, "bf16", seed=13)
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    qs = [torch.randn(4, h, 64, generator=gen(h), device="cuda") for h in (8, 64, 16, 32)]
    bare = type(c)(c.k, c.v, c.table, position=c.position)
    want = [bare.attend(q, n, 3000) for q in qs]
    first = torch.randn(4, 8, 64, generator=gen(99), device="cuda")
    alone = bare.attend(first, n, 3000)
    graph, out = torch.cuda.CUDAGraph(), torch.empty_like(first)
    with torch.cuda.graph(graph):
        bare.attend(first, n, 3000, out=out)
    torch.cuda.synchronize()
    bad = []

    def work(k):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(30):
                if not torch.equal(bare.attend(qs[k], n, 3000), want[k]):
                    bad.append(k)
    threads = [threading.Thread(target=work, args=(k,)) for k in range(4)]
    for t in threads:
        t.start()
    side = torch.cuda.Stream()
    for _ in range(30):
        out.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        got = [bare.attend(q, n, 3000) for q in qs]
        torch.cuda.synchronize()
        assert torch.equal(out, alone) and all(torch.equal(a, b) for a, b in zip(got, want))
    for t in threads:
        t.join()
    assert not bad


def test_offsets_past_32_bits():
    """Pages more than 2^31 elements apart: append, attention and eviction reach them."""
    from paper_2607_29221_gb300 import kvcache as KV
    stride = (1 << 31) + 1024
    base = torch.zeros(2 * stride + 1 * 16 * 64 * 2, dtype=torch.bfloat16, device="cuda")
    view = lambda off: base.as_strided((3, 1, 16, 64), (stride, 16 * 64, 64, 1), off)
    k, v = view(0), view(16 * 64)
    table = torch.tensor([[2, 0, 1]], dtype=torch.int32, device="cuda")
    c = KV.PagedCache(k, v, table, torch.zeros(3, 1, 16, dtype=torch.int32, device="cuda"),
                      torch.zeros(3, 1, 16, device="cuda"))
    c.lens = [40]
    qkv = torch.randn(40, 6 * 64, generator=gen(7), device="cuda")
    i = torch.arange(40, dtype=torch.int32, device="cuda")
    c.append(qkv, 4, torch.zeros_like(i), i, i)
    assert torch.equal(rows(c, k, 0, 40)[0], qkv[:, 4 * 64: 5 * 64].bfloat16().double())
    assert torch.equal(rows(c, v, 0, 40)[0], qkv[:, 5 * 64:].bfloat16().double())
    q = torch.randn(1, 4, 64, generator=gen(8), device="cuda")
    want, tol, _ = reference(c, q, 0.125)
    n = torch.tensor([40], dtype=torch.int32, device="cuda")
    assert ((c.attend(q, n, 40).double() - want).abs() <= tol).all()
    c.weight.zero_()
    for s in range(20, 40):
        c.weight[int(table[0, s // 16]), 0, s % 16] = 1.0
    keys = rows(c, k, 0, 40)
    assert c.evict(n, 40, 20).tolist() == [20]
    assert torch.equal(rows(c, k, 0, 20), keys[:, 20:])


# ---------------------------------------------------------------------------
@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("l,heads,kv,dim,rot,sections,inter,page,layout,pad", [
    (1, 64, 8, 128, 128, None, False, 16, "head", 0),
    (37, 8, 8, 64, 64, [8, 12, 12], True, 16, "token", 0),
    (130, 28, 4, 128, 64, [10, 22], False, 5, "padded", 12),
    (5, 3, 1, 80, 40, None, True, 1, "head", 1),
    (700, 12, 12, 8, 8, [1, 1, 1, 1], False, 64, "head", 3),
    (64, 4, 2, 256, 256, [0, 128], True, 32, "head", 0),
    (9, 5, 5, 24, 0, None, False, 16, "token", 2),
])
def test_append(l, heads, kv, dim, rot, sections, inter, page, layout, pad, typ):
    from paper_2607_29221_gb300 import kvcache as KV
    seqs = 3
    lens = [l + 20] * seqs
    c = make(lens, kv, dim, page, typ, layout, seed=l, poison=False)
    g = gen(l + 1)
    wide = torch.randn(l, (heads + 2 * kv) * dim + pad, generator=g, device="cuda")
    qkv = wide[:, : (heads + 2 * kv) * dim]
    at = torch.randperm(seqs * (l + 20), generator=g, device="cuda")[:l]
    seq, slot = (at // (l + 20)).int(), (at % (l + 20)).int()
    if l > 3:       # not stored: a padding row, a slot past the table, a sequence that is none
        slot[0], slot[1], seq[2] = -1, 1 << 30, seqs
    index = torch.randint(0, 1 << 31, (l,), generator=g, device="cuda").int()
    rope, pos, base = None, None, 500000.0
    if rot:
        rope = KV.Rope(rot, base, sections, inter)
        pos = torch.randint(0, 200000, (rope.axes, l), generator=g, device="cuda", dtype=torch.int32)
        if l > 3:
            pos[:, 3] = (1 << 31) - 1
            pos[:, 4] = -77
    old = [x.clone() for x in (c.k, c.v, c.position, c.weight)]
    q = c.append(qkv, heads, seq, slot, index, rope=rope, pos=pos)

    x = qkv.double().reshape(l, heads + 2 * kv, dim)
    y, tol = x.clone(), x.abs() * 0
    if rot:
        # Phases in exact integers: pos * round(2^64 freq / 2 pi) modulo a turn.
        turns = [int(t) for t in KV.M.mosaic_rope_turns(rot, base)]
        axis = np.repeat(np.arange(rope.axes), sections or [rot // 2])
        P = pos.cpu().tolist()
        ang = torch.tensor([[((P[axis[j]][t] * turns[j]) % 2 ** 64) / 2 ** 64 * 2 * math.pi for j in range(rot // 2)]
                            for t in range(l)], dtype=torch.float64, device="cuda")[:, None]
        a, b = ((slice(0, rot, 2), slice(1, rot, 2)) if inter else (slice(0, rot // 2), slice(rot // 2, rot)))
        xa, xb = x[..., a], x[..., b]
        y[..., a], y[..., b] = xa * ang.cos() - xb * ang.sin(), xb * ang.cos() + xa * ang.sin()
        tol[..., a] = tol[..., b] = 2.0 ** -20 * (xa.abs() + xb.abs())
        y[:, heads + kv:], tol[:, heads + kv:] = x[:, heads + kv:], 0
    assert ((q.double() - y[:, :heads]).abs() <= tol[:, :heads]).all()
    ulp = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}[typ]
    live = [t for t in range(l) if 0 <= int(slot[t]) < c.table.shape[1] * page and int(seq[t]) < seqs]
    page_of = c.table[seq[live].long(), (slot[live] // page).long()].long()
    off = (slot[live] % page).long()
    kk, vv = c.k[page_of, :, off], c.v[page_of, :, off]
    wk, wt = y[live, heads: heads + kv], tol[live, heads: heads + kv]
    assert ((kk.double() - wk).abs() <= wt + ulp * wk.abs() + 2.0 ** -24).all()
    assert torch.equal(vv, x[live, heads + kv:].to(TYPES[typ]))
    assert (c.position[page_of, :, off] == index[live][:, None]).all() and (c.weight[page_of, :, off] == 0).all()
    for new, was in zip((c.k, c.v, c.position, c.weight), old):     # nothing else is written
        was[page_of, :, off] = new[page_of, :, off]
        assert torch.equal(new, was)


def test_append_matches_a_product_of_rotations():
    """q . k depends on the difference of the positions only (up to roundings), at far positions too."""
    from paper_2607_29221_gb300 import kvcache as KV
    c = make([4], 1, 128, 16, "f32")
    x = torch.randn(1, 3 * 128, generator=gen(4), device="cuda").repeat(2, 1)
    rope = KV.Rope(128, 10000.0)
    dots = []
    for far in (5, 1 << 30):
        pos = torch.tensor([far, far + 7], dtype=torch.int32, device="cuda")
        i = torch.arange(2, dtype=torch.int32, device="cuda")
        q = c.append(x, 1, i * 0, i, i, rope=rope, pos=pos)
        dots.append(float(q[1, 0].double() @ rows(c, c.k, 0, 1)[0, 0]))
    assert abs(dots[0] - dots[1]) <= 2.0 ** -18 * float(x[0, :128].double().abs() @ x[0, 128:256].double().abs())


# ---------------------------------------------------------------------------
def evict_reference(weight, position, n, keep, start):
    """(new length, {destination: source}) of one head."""
    if n <= keep:
        return n, {}
    rank = []
    for s in range(n):
        w = float(weight[s])
        w = -math.inf if math.isnan(w) else w
        if start is not None and int(position[s]) >= start:
            w = math.inf
        rank.append((w, s))
    gone = {s for _, s in sorted(rank)[: n - keep]}
    holes = [s for s in range(keep) if s in gone]
    stay = [s for s in range(keep, n) if s not in gone]
    assert len(holes) == len(stay)
    return keep, dict(zip(holes, stay))


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("lens,kv,dim,page,keep,recent,layout,kind", [
    ([1, 0, 5], 2, 64, 16, 1, 0, "head", "random"),
    ([65, 64, 63, 200, 0], 8, 128, 16, 64, 16, "head", "random"),
    ([1025, 3, 999], 3, 24, 7, 1000, 100, "token", "ties"),
    ([3000], 4, 64, 20, 1, 0, "padded", "ties"),
    ([5000, 2600], 2, 128, 16, 2500, 2600, "head", "random"),       # more spared slots than the budget
    ([777, 778], 1, 256, 1, 400, 30, "head", "odd"),
    ([4096, 4097, 4098], 2, 8, 128, 4096, 0, "head", "equal"),
    ([40000, 9000], 1, 16, 64, 8200, 64, "head", "random"),
    ([70001], 2, 8, 16, 35000, 1000, "head", "ties"),
    ([420001], 1, 8, 64, 200000, 1000, "head", "ties"),             # more slots than a cluster holds keys of
    ([420001], 1, 8, 64, 419990, 0, "head", "random"),
    ([130, 129, 128, 1], 2, 64, 6, 128, 10, "head", "random"),      # a few over the budget, odd pages
    ([130, 129, 128, 1], 2, 64, 8, 128, 0, "token", "equal"),
])
def test_evict(lens, kv, dim, page, keep, recent, layout, kind, typ):
    c = make(lens, kv, dim, page, typ, layout, seed=keep, poison=False)
    g = gen(keep + 1)
    w = torch.randn(c.weight.shape, generator=g, device="cuda").exp()
    if kind == "ties":
        w = torch.randint(0, 4, w.shape, generator=g, device="cuda").float()
    elif kind == "equal":
        w = torch.full_like(w, 2.0)
    elif kind == "odd":      # NaN, infinities, both zeros, negatives, subnormals
        some = torch.tensor([math.nan, math.inf, -math.inf, 0.0, -0.0, -1.0, 1e-42, -1e-42, 3.0], device="cuda")
        w = some[torch.randint(0, len(some), w.shape, generator=g, device="cuda")]
    c.weight.copy_(w)
    c.position.copy_(torch.randint(0, 1 << 20, c.position.shape, generator=g, device="cuda"))
    start = None
    if recent:
        start = torch.tensor([int((1 << 20) * (1 - recent / max(n, 1))) for n in lens], device="cuda").int()
    pools = (c.k, c.v, c.position, c.weight)
    want = [x.clone() for x in pools]
    for i, n in enumerate(lens):
        for h in range(kv):
            _, moves = evict_reference(rows(c, c.weight, i, n)[h], rows(c, c.position, i, n)[h], n, keep,
                                       None if start is None else int(start[i]))
            if moves:
                to, frm = (torch.tensor(list(x), device="cuda") for x in (moves.keys(), moves.values()))
                tp, fp = c.table[i, to // page].long(), c.table[i, frm // page].long()
                for x, y in zip(want, pools):
                    x[tp, h, to % page] = y[fp, h, frm % page]
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    new = c.evict(n, max(lens), keep, recent_from=start)
    assert new.tolist() == [min(x, keep) for x in lens] and n.tolist() == lens
    for x, y in zip(want, pools):
        bits = {4: torch.int32, 2: torch.int16}[x.element_size()]
        assert torch.equal(x.contiguous().view(bits), y.contiguous().view(bits))


def test_evict_writes_lengths_in_place_and_clamps():
    c = make([50, 50, 9], 2, 64, 16, "bf16", poison=False)
    n = torch.tensor([1 << 30, 30, -4], dtype=torch.int32, device="cuda")
    assert c.evict(n, 48, 20, new_lens=n) is n
    assert n.tolist() == [20, 20, 0]


def test_evicted_cache_is_read_like_any_other():
    """append, attend, evict, append, attend: the serving loop, against the reference."""
    lens = [100, 100]
    c = make(lens, 2, 64, 16, "bf16", cols=8)
    c.position.copy_(torch.arange(c.position.numel(), device="cuda").reshape(c.position.shape))
    q = torch.randn(2, 8, 64, generator=gen(11), device="cuda")
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    c.weight.zero_()
    c.attend(q, n, 100)
    n = c.evict(n, 100, 60)
    i = torch.arange(2, dtype=torch.int32, device="cuda")
    qkv = torch.randn(2, 12 * 64, generator=gen(12), device="cuda")
    q = c.append(qkv, 8, i, n.clone(), i + 100)
    n += 1
    c.lens = [61, 61]
    want, tol, _ = reference(c, q, 0.125)
    assert ((c.attend(q, n, 61).double() - want).abs() <= tol).all()


def test_python_refusals():
    from paper_2607_29221_gb300 import kvcache as KV
    from paper_2607_29221_gb300 import mosaic as M
    c = make([20], 2, 64, 16, "bf16")
    n = torch.tensor([20], dtype=torch.int32, device="cuda")
    q = torch.zeros(1, 4, 64, device="cuda")
    for bad in (q.half(), q.cpu(), torch.zeros(2, 4, 64, device="cuda"), torch.zeros(1, 4, 32, device="cuda"),
                torch.zeros(1, 64, 4, device="cuda").transpose(1, 2)):
        with pytest.raises(ValueError):
            c.attend(bad, n, 20)
    for bad in (n.long(), n.cpu(), n.repeat(2)):
        with pytest.raises(ValueError):
            c.attend(q, bad, 20)
        with pytest.raises(ValueError):
            c.evict(bad, 20, 10)
    with pytest.raises(M.MosaicError):
        c.attend(torch.zeros(1, 3, 64, device="cuda"), n, 20)      # 3 query heads on 2 key/value heads
    with pytest.raises(M.MosaicError):
        c.evict(n, 20, 0)
    with pytest.raises(M.MosaicError):
        KV.PagedCache(c.k, c.v, c.table).evict(n, 20, 10)          # no weights
    with pytest.raises(ValueError):
        KV.PagedCache(c.k, c.v.float(), c.table)
    with pytest.raises(ValueError):
        KV.PagedCache(c.k, c.v, c.table.long())
    with pytest.raises(ValueError):
        KV.PagedCache(c.k, c.v, c.table, weight=c.weight.double())
    with pytest.raises(ValueError):
        c.append(torch.zeros(1, 7 * 64, device="cuda"), 4, n, n, n)


def test_expanded_rows_are_refused():
    """Rows that share memory, wherever a call takes rows: nothing is launched."""
    from paper_2607_29221_gb300 import kvcache as KV
    from paper_2607_29221_gb300 import mosaic as M
    c = make([20, 20, 20], 2, 64, 16, "bf16")
    n = torch.tensor([20, 20, 20], dtype=torch.int32, device="cuda")
    q, one = torch.zeros(3, 4, 64, device="cuda"), torch.zeros(1, 4, 64, device="cuda")
    row = torch.zeros(1, 8 * 64, device="cuda")
    rope = KV.Rope(64, sections=[8, 12, 12])
    pos = torch.zeros(1, 3, dtype=torch.int32, device="cuda")
    before = M.mosaic_kernel_launches()
    for call in (lambda: c.attend(one.expand(3, 4, 64), n, 20), lambda: c.attend(q, n, 20, out=one.expand(3, 4, 64)),
                 lambda: c.append(row.expand(3, 512), 4, n, n, n),
                 lambda: c.append(row.repeat(3, 1), 4, n, n, n, out=one.expand(3, 4, 64)),
                 lambda: c.append(row.repeat(3, 1), 4, n, n, n, rope=rope, pos=pos.expand(3, 3)),
                 lambda: KV.PagedCache(c.k, c.v, c.table[:1].expand(3, 2))):
        with pytest.raises(ValueError, match="share memory"):
            call()
    assert M.mosaic_kernel_launches() == before
    same = c.append(row.repeat(3, 1), 4, n - n - 1, n - n - 1, n, rope=rope, pos=pos.expand(3, 3).contiguous())
    assert (same == 0).all()


@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("lens,heads,kv,dim,page,layout", [
    ([200, 90], 8, 2, 64, 16, "head"),
    ([200, 90], 32, 2, 128, 7, "token"),
    ([3000, 700], 16, 4, 128, 16, "head"),
    ([3000, 700], 12, 1, 256, 5, "head"),
    ([1100] * 20, 16, 8, 64, 8, "head"),
])
@pytest.mark.parametrize("value", [math.inf, -math.inf])
def test_attention_counts_live_infinities_as_nan(lens, heads, kv, dim, page, layout, value, typ):
    """A live infinite key makes its head's rows NaN and a live infinite value
    its channel, whatever the signs of the queries, in the first slots and later
    ones; other heads, sequences and channels keep their results, and so does a
    row whose bound leaves the slot out."""
    bad = []
    group = heads // kv
    q = torch.randn(len(lens), heads, dim, generator=gen(21), device="cuda")
    q[:, 0] = q[:, 0].abs()
    q[:, 1 % group] = -q[:, 1 % group].abs()
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    for slot in (0, 5, lens[0] // 2, lens[0] - 1):
        c = make(lens, kv, dim, page, typ, layout, seed=slot, poison=False)
        c.position.zero_()
        at = int(c.table[0, slot // page]), slot % page
        c.position[at[0], :, at[1]] = -1
        want, tol, _ = reference(c, q, 0.125)
        c.k[at[0], 0, at[1], 3] = value
        c.v[at[0], kv - 1, at[1], 6] = value
        out = c.attend(q, n, max(lens), scale=0.125)
        nan = torch.zeros_like(out, dtype=torch.bool)
        nan[0, :group] = True
        nan[0, heads - group:, 6] = True
        if not torch.isnan(out[nan]).all():
            bad.append((slot, "nan", float(torch.isnan(out[nan]).float().mean())))
        if not ((out.double() - want).abs() <= tol)[~nan].all():
            bad.append((slot, "rest"))
        keep = c.attend(q, n, max(lens), first=torch.zeros_like(n), scale=0.125)
        if not torch.isfinite(keep).all():
            bad.append((slot, "left out"))
    assert not bad, bad


@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("lens,heads,kv,dim,page", [([300, 40], 8, 1, 64, 16), ([300, 40], 24, 2, 128, 5),
                                                    ([5000, 700], 16, 8, 128, 16), ([900, 40], 12, 1, 256, 8)])
@pytest.mark.parametrize("depth", [12.0, 20.0, 28.0, 45.0])
def test_attention_of_small_probabilities(lens, heads, kv, dim, page, depth, typ):
    """One slot with a value of zero takes nearly all of the weight: the output is
    what the others' probabilities of about e^-depth make of theirs."""
    g = gen(31)
    c = make(lens, kv, dim, page, typ, seed=3, poison=False)
    q = torch.randn(len(lens), heads, dim, generator=g, device="cuda")
    q[..., 0] = 4.0
    c.k[..., 0] = 0.0
    for i, n in enumerate(lens):
        page_of = int(c.table[i, (n // 3) // page]), slice(None), (n // 3) % page
        c.k[page_of] = 0.0
        c.k[(*page_of, 0)] = depth * dim ** 0.5 / 4.0
        c.v[page_of] = 0.0
    c.weight.zero_()
    want, tol, weights = reference(c, q, dim ** -0.5)
    out = c.attend(q, torch.tensor(lens, dtype=torch.int32, device="cuda"), max(lens))
    assert ((out.double() - want).abs() <= tol).all(), float(((out.double() - want).abs() / tol).max())
    for i, n in enumerate(lens):
        w, wt = weights[i]
        assert ((rows(c, c.weight, i, n) - w).abs() <= wt).all()


@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("lens,heads,kv,dim,page", [([300, 40], 8, 1, 64, 16), ([300, 40], 24, 2, 128, 5),
                                                    ([900, 40], 12, 1, 256, 8)])
@pytest.mark.parametrize("spread", [14, 20, 26])
def test_attention_of_queries_with_a_wide_spread(lens, heads, kv, dim, page, spread, typ):
    """A channel 2^spread above the others meets keys of zero: the score is the others'."""
    g = gen(33)
    c = make(lens, kv, dim, page, typ, seed=4, poison=False)
    q = torch.randn(len(lens), heads, dim, generator=g, device="cuda") * 2.0 ** -12
    q[..., 5] = 2.0 ** (spread - 12)
    c.k[:] = (c.k.float() * 2.0 ** 13).to(c.k.dtype)
    c.k[..., 5] = 0.0
    want, tol, _ = reference(c, q, dim ** -0.5)
    out = c.attend(q, torch.tensor(lens, dtype=torch.int32, device="cuda"), max(lens))
    assert ((out.double() - want).abs() <= tol).all(), float(((out.double() - want).abs() / tol).max())


def test_scratch_ends_with_its_thread_and_streams():
    """Host threads that have ended leave nothing behind, and a thread keeps the scratch of a few streams only."""
    import threading
    c = make([3000, 1700], 8, 64, 16, "bf16", seed=13)
    n = torch.tensor([3000, 1700], dtype=torch.int32, device="cuda")
    q = torch.randn(2, 64, 64, generator=gen(1), device="cuda")
    out = torch.empty_like(q)
    c.attend(q, n, 3000, out=out)
    before = torch.cuda.memory_allocated()
    for _ in range(4):
        t = threading.Thread(target=lambda: c.attend(q, n, 3000, out=out))
        t.start()
        t.join()
    assert torch.cuda.memory_allocated() == before
    used = []
    for stream in [torch.cuda.Stream() for _ in range(12)]:
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            c.attend(q, n, 3000, out=out)
        stream.synchronize()
        used.append(torch.cuda.memory_allocated())
    assert used[-1] == used[5] and used[-1] - before <= 4 * (used[0] - before)


def test_an_empty_batch():
    """No sequences: attention and eviction have nothing to do, an append only rotates."""
    from paper_2607_29221_gb300 import kvcache as KV
    c = make([20], 2, 64, 16, "bf16")
    e = KV.PagedCache(c.k, c.v, c.table[:0], c.position, c.weight)
    n = torch.zeros(0, dtype=torch.int32, device="cuda")
    assert e.attend(torch.zeros(0, 4, 64, device="cuda"), n, 20).shape == (0, 4, 64)
    assert e.evict(n, 20, 10).shape == (0,)
    before = c.weight.clone()
    x, i = torch.randn(3, 8 * 64, generator=gen(2), device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    assert torch.equal(e.append(x, 4, i, i, i), x[:, :256].unflatten(1, (4, 64)))
    assert torch.equal(c.weight, before)
    assert e.append(x[:0], 4, n, n, n).shape == (0, 4, 64)


@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
def test_append_of_more_tokens_than_a_grid_axis_holds(typ):
    l = 70001
    c = make([l], 1, 8, 16, typ, poison=False)
    qkv = torch.randn(l, 24, generator=gen(41), device="cuda")
    i = torch.arange(l, dtype=torch.int32, device="cuda")
    slot = i.flip(0).contiguous()
    q = c.append(qkv, 1, torch.zeros_like(i), slot, i + 5)
    assert torch.equal(q[:, 0], qkv[:, :8])
    back = qkv.flip(0)
    assert torch.equal(rows(c, c.k, 0, l)[0], back[:, 8:16].to(TYPES[typ]).double())
    assert torch.equal(rows(c, c.v, 0, l)[0], back[:, 16:].to(TYPES[typ]).double())
    assert torch.equal(rows(c, c.position, 0, l)[0], (i + 5).flip(0).double())


def test_a_captured_step_equals_the_eager_one():
    """append, attend and evict in one graph, replayed with other inputs."""
    lens = [90, 64, 1]

    def step(c, qkv, seq, n, out, new):
        q = c.append(qkv, 8, seq, n, n)
        c.attend(q, n + 1, 101, out=out)
        c.evict(n + 1, 101, 64, recent_from=n - 8, new_lens=new)
    results = []
    for graphed in (False, True):
        c = make([v + 10 for v in lens], 2, 64, 16, "bf16", seed=6, poison=False)
        c.position.copy_(torch.arange(c.position.numel(), device="cuda").reshape(c.position.shape) % 97)
        seq = torch.arange(3, dtype=torch.int32, device="cuda")
        qkv, n = torch.zeros(3, 12 * 64, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
        out, new = torch.zeros(3, 8, 64, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
        pools = (c.k, c.v, c.position, c.weight)
        kept = [x.clone() for x in pools]
        if graphed:
            n.copy_(torch.tensor(lens, dtype=torch.int32))
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step(c, qkv, seq, n, out, new)
            assert all(torch.equal(x, y) for x, y in zip(pools, kept))
        got = []
        for turn in range(3):
            qkv.copy_(torch.randn(3, 12 * 64, generator=gen(50 + turn), device="cuda"))
            n.copy_(torch.tensor(lens, dtype=torch.int32) if turn == 0 else new)
            graph.replay() if graphed else step(c, qkv, seq, n, out, new)
            got += [x.clone() for x in (out, new, *pools)]
        results.append(got)
    assert results[0][1].tolist() == [64, 64, 2]
    assert all(torch.equal(a, b) for a, b in zip(*results))


@pytest.mark.parametrize("lens,keep", [([300], 200), ([3000, 2100], 1500), ([70001], 35000)])
def test_evict_leaves_slots_without_a_page(lens, keep):
    """They rank as +inf; a move from or to one is left out."""
    kv, dim, page = 2, 16, 16
    c = make(lens, kv, dim, page, "bf16", seed=8, poison=False)
    for i, n in enumerate(lens):
        c.table[i, : -(-n // page): 5] = -1
    w = torch.rand(c.weight.shape, generator=gen(9), device="cuda")
    c.weight.copy_(w)
    want = [x.clone() for x in (c.k, c.v, c.position, c.weight)]
    for i, n in enumerate(lens):
        ids = c.table[i, : -(-n // page)].long().cpu().numpy()
        at, off = ids[np.arange(n) // page], np.arange(n) % page
        for h in range(kv):
            rank = np.where(at < 0, np.inf, c.weight[:, h].cpu().numpy()[at, off])
            gone = np.zeros(n, dtype=bool)
            gone[np.argsort(rank, kind="stable")[: n - keep]] = True
            to, frm = np.flatnonzero(gone[:keep]), keep + np.flatnonzero(~gone[keep:])
            real = (at[to] >= 0) & (at[frm] >= 0)
            to, frm = to[real], frm[real]
            for x, y in zip(want, (c.k, c.v, c.position, c.weight)):
                x[at[to], h, off[to]] = y[at[frm], h, off[frm]]
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    assert c.evict(n, max(lens), keep).tolist() == [keep] * len(lens)
    for x, y in zip(want, (c.k, c.v, c.position, c.weight)):
        assert torch.equal(x, y)


def test_library_calls_equal_the_handle():
    from paper_2607_29221_gb300 import kvcache as KV
    from paper_2607_29221_gb300 import mosaic as M
    lens, results = [70, 33], []
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    seq = torch.arange(2, dtype=torch.int32, device="cuda")
    qkv = torch.randn(2, 8 * 64, generator=gen(14), device="cuda")
    rope, pos = KV.Rope(64), torch.tensor([70, 33], dtype=torch.int32, device="cuda")
    for direct in (False, True):
        c = make([80, 80], 2, 64, 16, "f16", seed=15, poison=False)
        q, out = torch.empty(2, 4, 64, device="cuda"), torch.empty(2, 4, 64, device="cuda")
        new = torch.empty_like(n)
        if direct:
            scratch = lambda size: torch.empty(max(size, 256), dtype=torch.uint8, device="cuda")
            M.mosaic_kv_append(c._c, qkv, 512, 2, 4, seq, n, pos, rope.at(pos), q, 256)
            M.mosaic_kv_attention(c._c, q, 256, 4, n, 70, None, 0.125, 0.5, out, 256,
                                  scratch(M.mosaic_kv_attention_workspace(c._c, 4, 70)))
            M.mosaic_kv_evict(c._c, n, 70, 40, None, new, scratch(M.mosaic_kv_evict_workspace(c._c, 70, 40)))
        else:
            c.append(qkv, 4, seq, n, pos, rope=rope, pos=pos, out=q)
            c.attend(q, n, 70, decay=0.5, out=out)
            c.evict(n, 70, 40, new_lens=new)
        results.append([x.clone() for x in (q, out, new, c.k, c.v, c.position, c.weight)])
    assert all(torch.equal(a, b) for a, b in zip(*results))

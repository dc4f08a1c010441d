"""4-bit key/value cache and head norms on the GPU, against plain
implementations in 64 bits (and, where every step is an IEEE operation, bit for
bit).

Tolerances, set from the number formats before any run:

  attention  as for the other caches (a product carried to 22 bits and summed in
             fp32 over at most 256 channels moves a score by at most E = 2^-20
             scale sum |q_d k_d|, a probability by 2 E relative, and exp, the sums
             and the join add at most 2^-19); besides, the lower fp16 terms are off by
             up to 2^-25, of queries scaled to 2^14 or more a head (2^-39 of the
             largest) and of weights scaled to 2^15 (2^-40 of the row's largest):
             E + 2^-39 scale max|q| sum |k_d|, and
             |d out| <= (2 E + 2^-19) sum p |v| + 2^-40 max p sum |v|.
  append     the bytes of a row are defined by IEEE operations on sines, cosines
             and 1 / rms rounded once: equal.  Queries: phase 2^-25 turns, three
             roundings of the rotation and the norm's sum of 256 squares, root and
             two products (2^-19 together): 2^-18 (|a| + |b|) for a pair.
  rows       equal.
  eviction   equal.
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


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------------------
# The format, on the host: numpy rounds float64 to float16 directly, once.
def values(rows, dim):
    """Packed rows (uint8 tensor, ... x bytes) as float64."""
    r = rows.cpu().numpy()
    code = np.empty(r.shape[:-1] + (dim,), np.float64)
    code[..., 0::2], code[..., 1::2] = r[..., : dim // 2] & 15, r[..., : dim // 2] >> 4
    pair = np.ascontiguousarray(r[..., dim // 2: dim // 2 + dim // 8]).view(np.float16).astype(np.float64)
    step, base = np.repeat(pair[..., 0::2], 32, -1), np.repeat(pair[..., 1::2], 32, -1)
    with np.errstate(all="ignore"):
        y = (base + code * step).astype(np.float16).astype(np.float64)
    return torch.from_numpy(y).to(rows.device)


def pack(y):
    """Rows of float32 channels (numpy) as the first 5 dim / 8 bytes of packed rows."""
    f = np.float32
    x = y.reshape(y.shape[:-1] + (-1, 32)).astype(f)
    with np.errstate(all="ignore"):
        fine = np.isfinite(x).all(-1)
        x = np.where(fine[..., None], np.clip(x, f(-65000), f(65000)), f(0))
        least, most = x.min(-1), x.max(-1)
        base = np.where(fine, least, f(np.nan)).astype(np.float16)
        step = ((most - least).astype(f) * f(1.0 / 15.0)).astype(f).astype(np.float16)
        s = step.astype(f)
        inv = np.where(s > 0, f(1) / np.where(s > 0, s, f(1)), f(0)).astype(f)
        code = np.rint((x - least.astype(np.float16).astype(f)[..., None]).astype(f) * inv[..., None])
    code = np.where(fine[..., None], np.clip(code, 0, 15), 0).astype(np.uint8).reshape(y.shape)
    step[~fine] = 0
    scales = np.stack([step, base], -1).reshape(y.shape[:-1] + (-1,))
    return np.concatenate([code[..., 0::2] | code[..., 1::2] << 4, np.ascontiguousarray(scales).view(np.uint8)], -1)


def same_bytes(got, want, dim):
    """Equal rows; a NaN base is any NaN."""
    g, w = got.cpu().numpy()[..., : 5 * dim // 8], want
    gs = np.ascontiguousarray(g[..., dim // 2:]).view(np.uint16)
    ws = np.ascontiguousarray(w[..., dim // 2:]).view(np.uint16)
    nan = lambda u: (u & 0x7fff) > 0x7c00
    return np.array_equal(g[..., : dim // 2], w[..., : dim // 2]) and bool(
        ((gs == ws) | (nan(gs) & nan(ws))).all())


def random_rows(shape, dim, g):
    """Rows as normal channels would pack: codes of every value, steps and bases of every sign and some offset."""
    from paper_2607_29221_gb300 import kvcache as KV
    x = torch.full((*shape, KV.row_bytes(dim)), 255, dtype=torch.uint8, device="cuda")
    x[..., : dim // 2] = torch.randint(0, 256, (*shape, dim // 2), generator=g, device="cuda", dtype=torch.uint8)
    step = torch.exp(0.5 * torch.randn(*shape, dim // 32, generator=g, device="cuda")) * 0.25
    base = step * (torch.randn(step.shape, generator=g, device="cuda") - 7.5)
    s = torch.stack([step, base], -1).flatten(-2).half()
    x[..., dim // 2: 5 * dim // 8] = s.contiguous().view(torch.uint8)
    return x


def make(lens, kv, dim, page, layout="head", seed=0, gap=0):
    """A 4-bit cache; rows not in use hold NaN, and table entries past a sequence's pages are no pages at all."""
    from paper_2607_29221_gb300 import kvcache as KV
    g = gen(seed)
    need = [-(-n // page) for n in lens]
    cols, pages = max(1, max(need)), sum(need) + 2
    order = torch.randperm(pages, generator=g, device="cuda").tolist()
    table = torch.full((len(lens), cols + gap), 0x7fffffff, dtype=torch.int32, device="cuda")[:, :cols]
    table[::2] = -1
    used = torch.zeros(pages, page, dtype=torch.bool, device="cuda")
    at = 0
    for i, n in enumerate(lens):
        ids = ints(order[at: at + need[i]])
        table[i, : need[i]] = ids
        at += need[i]
        if n:
            used[ids.long()] = torch.arange(need[i] * page, device="cuda").reshape(-1, page) < n
    pools = []
    for _ in range(2):
        x = random_rows((pages, kv, page), dim, g)
        x[~used[:, None, :].expand(-1, kv, -1)] = 255           # codes 15, steps and bases NaN
        if layout == "token":
            x = x.transpose(1, 2).contiguous().transpose(1, 2)
        elif layout == "padded":                                 # rows of a wider buffer
            wide = torch.full((*x.shape[:3], x.shape[3] + 48), 255, dtype=torch.uint8, device="cuda")
            wide[..., 16: 16 + x.shape[3]] = x
            x = wide[..., 16: 16 + x.shape[3]]
        pools.append(x)
    c = KV.PagedCache(*pools, table, position=torch.zeros(pages, kv, page, dtype=torch.int32, device="cuda"),
                      weight=torch.rand(pages, kv, page, generator=g, device="cuda") * 3)
    assert c.head_dim == dim
    c.used, c.lens = used, list(lens)
    return c


def slots(c, pool, i, n):
    """Slots 0..n of sequence i: kv x n (x ...)."""
    x = pool[c.table[i, : -(-n // c.k.shape[2])].long()].transpose(0, 1)
    return x.reshape(x.shape[0], -1, *x.shape[3:])[:, :n]


def reference(c, q, scale, first=None, decay=1.0):
    """out, its tolerance, and weights with theirs by sequence, in 64 bits."""
    b, heads, d = q.shape
    out = torch.zeros(b, heads, d, dtype=torch.float64, device="cuda")
    tol, weights = torch.zeros_like(out), {}
    for i, n in enumerate(c.lens):
        if not n:
            continue
        k, v = (values(slots(c, x, i, n), d) for x in (c.k, c.v))
        qi = q[i].double().reshape(c.kv_heads, -1, d)
        s = torch.einsum("hgd,hnd->hgn", qi, k) * scale
        err = abs(scale) * (2.0 ** -20 * torch.einsum("hgd,hnd->hgn", qi.abs(), k.abs())
                            + 2.0 ** -39 * qi.abs().amax(2, keepdim=True) * k.abs().sum(2)[:, None])
        if first is not None:
            s = s.masked_fill(slots(c, c.position, i, n)[:, None] < int(first[i]), -math.inf)
        gone = s == -math.inf
        p = torch.where(gone.all(2, keepdim=True), 0.0, torch.softmax(s, 2))
        rel = 2 * err.amax(2, keepdim=True) + 2.0 ** -19
        out[i] = torch.einsum("hgn,hnd->hgd", p, v).reshape(heads, d)
        small = 2.0 ** -40 * p.amax(2, keepdim=True)
        tol[i] = (rel * torch.einsum("hgn,hnd->hgd", p, v.abs()) + small * v.abs().sum(1)[:, None]).reshape(heads, d)
        w = slots(c, c.weight, i, n).double() * decay + p.sum(1)
        weights[i] = (w, w.abs() * rel.amax(1) + 1e-30)
    return out, tol, weights


def check(c, q, out, ref, quiet=()):
    want, tol, weights = ref
    off = (out.double() - want).abs()
    assert (off <= tol).all(), float((off / (tol + 1e-300)).max())
    for i, n in enumerate(c.lens):
        if n:
            w, wt = weights[i]
            assert ((slots(c, c.weight, i, n).double() - w).abs() <= wt).all(), i
        if not n or i in quiet:
            assert (out[i] == 0).all()


CASES = [
    # lens, heads, kv, dim, page, layout
    ([1], 1, 1, 32, 1, "head"),
    ([1, 0, 2], 8, 8, 128, 16, "head"),
    ([15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 1, 0], 64, 8, 128, 16, "head"),
    ([255, 256, 257, 513], 28, 4, 128, 32, "token"),
    ([1000, 3, 77, 0, 640], 24, 8, 64, 20, "token"),
    ([333, 1025], 12, 12, 96, 7, "padded"),
    ([2049, 31], 32, 2, 192, 64, "head"),
    ([700, 1, 15, 16, 17], 3, 1, 256, 8, "head"),
    ([130, 513], 64, 1, 32, 3, "head"),
    ([4100], 17, 1, 128, 128, "head"),
    ([300, 40], 64, 2, 64, 24, "padded"),
    ([900, 40], 20, 1, 160, 16, "token"),
    ([20011, 5], 8, 1, 128, 16, "head"),
]


@pytest.mark.parametrize("window", [False, True])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention(case, window):
    lens, heads, kv, dim, page, layout = CASES[case]
    c = make(lens, kv, dim, page, layout, seed=case, gap=3)
    g = gen(100 + case)
    q = torch.randn(len(lens), heads, dim, generator=g, device="cuda") * 1.5
    first = None
    if window:   # scattered positions; the second sequence has no live slot
        c.position.copy_(torch.randint(0, 1000, c.position.shape, generator=g, device="cuda"))
        first = torch.full((len(lens),), 300, dtype=torch.int32, device="cuda")
        first[1:2] = 1000
    ref = reference(c, q, dim ** -0.5, first, 0.75)
    before, pools = c.weight.clone(), (c.k.clone(), c.v.clone())
    out = c.attend(q, ints(lens), max(lens), first=first, decay=0.75)
    check(c, q, out, ref, quiet=(1,) if window else ())
    mark = c.used[:, None, :].expand_as(before)
    assert torch.equal(c.weight[~mark], before[~mark])   # nothing else is written
    assert torch.equal(c.k, pools[0]) and torch.equal(c.v, pools[1])


@pytest.mark.parametrize("seqs,most,heads,kv,dim,page,layout,window", [
    (20, 1100, 64, 8, 128, 16, "head", False),      # shared jobs, heads that share a unit
    (40, 1200, 24, 8, 64, 8, "token", True),
    (44, 1030, 16, 8, 128, 5, "head", True),        # copied by lanes
    (36, 1500, 32, 8, 128, 32, "padded", False),
    (48, 300, 24, 8, 128, 64, "head", True),        # whole jobs
    (100, 130, 16, 8, 128, 16, "token", False),
    (24, 90, 64, 32, 64, 128, "head", True),
    (70, 1100, 24, 2, 64, 16, "head", False),       # 12 query heads a key/value head
    (6, 1200, 40, 1, 64, 16, "head", True),         # 40
    (9, 200, 4, 2, 32, 16, "head", False),
    (30, 1050, 12, 4, 96, 8, "token", True),
    (5, 1300, 20, 2, 256, 8, "head", False),
    (80, 1100, 16, 8, 256, 16, "head", True),
    (70, 1200, 32, 2, 128, 16, "head", True),
    (20, 2100, 64, 8, 128, 16, "head", True),       # shared jobs with a lower bound
    (40, 2100, 24, 8, 64, 20, "token", True),
    (300, 1, 128, 8, 256, 16, "token", False),
])
def test_attention_of_many_sequences(seqs, most, heads, kv, dim, page, layout, window):
    """The ways in which jobs are shared out: heads a unit, whole jobs, boxes."""
    lens = [(most * (i + 1) // seqs) if i % 7 != 3 else 0 for i in range(seqs)]
    c = make(lens, kv, dim, page, layout, seed=seqs)
    g = gen(seqs + 1)
    q = torch.randn(seqs, heads, dim, generator=g, device="cuda") * 1.5
    first = None
    if window:     # most of the units, some heads and some sequences have no live slot
        c.position.copy_(torch.randint(0, 1000, c.position.shape, generator=g, device="cuda"))
        c.position[:, 0] //= 4
        first = torch.full((seqs,), 250, dtype=torch.int32, device="cuda")
        first[2::5] = 998
        first[4::5] = 1000
    ref = reference(c, q, dim ** -0.5, first, 0.5)
    out = c.attend(q, ints(lens), most, first=first, decay=0.5)
    check(c, q, out, ref)
    from paper_2607_29221_gb300 import mosaic as M
    M.mosaic_device_status()


def test_attention_without_weights_or_lengths():
    """No weights kept; lengths zero, negative, or beyond max_len and the table (clamped)."""
    c = make([40, 40, 40], 2, 64, 16)
    q = torch.randn(3, 4, 64, generator=gen(1), device="cuda")
    bare = type(c)(c.k, c.v, c.table)
    assert (bare.attend(q, ints([0, -5, 0]), 40) == 0).all()
    assert (bare.attend(q, ints([7, 7, 7]), 0) == 0).all()
    c.lens = [33, 33, 33]
    want, tol, _ = reference(c, q, 0.125)
    assert ((bare.attend(q, ints([1 << 30, 33, 40]), 33).double() - want).abs() <= tol).all()
    c.lens = [40, 40, 40]
    long = torch.cat([c.table, torch.full((3, 5), -1, dtype=torch.int32, device="cuda")], 1)
    far = type(c)(c.k, c.v, long)                         # slots without a page are masked
    want, tol, _ = reference(c, q, 0.125)
    c.lens = [48, 48, 48]                                  # (of the last page, 8 slots hold NaN)
    assert torch.isnan(far.attend(q, ints([128, 128, 128]), 128)).all()
    assert ((far.attend(q, ints([40, 40, 40]), 128).double() - want).abs() <= tol).all()


def test_attention_of_extreme_values():
    """Large scores, equal ones, live NaN and infinite steps and bases (they count as NaN), values of both ends of
    fp16, queries of wide range."""
    c = make([200] * 8, 1, 64, 16, seed=5)
    q = torch.randn(8, 4, 64, generator=gen(6), device="cuda")
    at = lambda i, s: (int(c.table[i, s // 16]), 0, s % 16)

    def scales(pool, i, s, step, base):
        pool[at(i, s)][32: 40] = torch.tensor([step, base] * 2, dtype=torch.float16, device="cuda").view(torch.uint8)
    q[1] = 0.0
    scales(c.k, 2, 3, 0.25, math.nan)
    scales(c.v, 3, 199, math.inf, 0.0)
    scales(c.k, 4, 9, 0.0, -0.0)
    scales(c.k, 5, 50, 4096.0, -30720.0)
    scales(c.v, 5, 51, 4333.0, -65000.0)
    q[6] *= 1e3                                            # a steep softmax
    scales(c.k, 7, 20, 0.0, -math.inf)
    q[7] = q[7].abs()                                      # a score of -inf is no masked slot
    want, tol, _ = reference(c, q, 0.125)
    out = c.attend(q, ints([200] * 8), 200)
    for i in (2, 7):
        assert torch.isnan(out[i]).all()
    assert not torch.isfinite(out[3]).any()
    for i in (0, 1, 4, 5, 6):
        off = (out[i].double() - want[i]).abs()
        assert (off <= tol[i]).all(), (i, float((off / tol[i]).max()))
    q[0, 0, 5], q[1, 2, 7] = math.nan, math.inf
    out = c.attend(q, ints([200] * 8), 200)
    assert torch.isnan(out[0, 0]).all() and torch.isnan(out[1, 2]).all()
    assert torch.isfinite(out[0, 1:]).all() and torch.isfinite(out[1, :2]).all()


def test_attention_of_strided_rows_on_another_stream_in_a_graph():
    lens = [300, 5, 129]
    c = make(lens, 2, 128, 16, seed=2)
    table = torch.cat([c.table, torch.full((3, 21), -1, dtype=torch.int32, device="cuda")], 1)
    bare = type(c)(c.k, c.v, table, position=c.position)
    wide = torch.randn(3, 16 * 128 + 36, generator=gen(3), device="cuda")
    q = wide[:, 5: 5 + 16 * 128].unflatten(1, (16, 128))
    buf = torch.full((3, 16 * 128 + 7), 9.0, device="cuda")
    out = buf[:, 3: 3 + 16 * 128].unflatten(1, (16, 128))
    n = ints(lens)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        bare.attend(q, n, 640, out=out)
    s.synchronize()
    want, tol, _ = reference(c, q, 128 ** -0.5)
    assert ((out.double() - want).abs() <= tol).all()
    assert (buf[:, :3] == 9).all() and (buf[:, 3 + 16 * 128:] == 9).all()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    outs = [out, torch.empty_like(q)]
    for gr, o in zip(graphs, outs):                        # graphs have scratch of their own
        with torch.cuda.graph(gr):
            bare.attend(q, n, 640, out=o)
    c.lens = [64, 1, 128]
    n.copy_(ints(c.lens))
    with torch.cuda.stream(s):
        graphs[0].replay()
    graphs[1].replay()
    torch.cuda.synchronize()
    want, tol, _ = reference(c, q, 128 ** -0.5)
    for o in outs:
        assert ((o.double() - want).abs() <= tol).all()


def test_attention_repeats_bit_for_bit():
    lens = [5000, 100, 0, 64, 3001]
    c = make(lens, 4, 128, 16, seed=9)
    q = torch.randn(5, 32, 128, generator=gen(2), device="cuda")
    start, first = c.weight.clone(), None
    for _ in range(3):
        c.weight.copy_(start)
        got = (c.attend(q, ints(lens), 5000), c.weight.clone())
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(first, got))


def test_attention_past_2_to_31_bytes():
    """Pages whose rows begin past 2^31 and 2^32 bytes of a pool."""
    from paper_2607_29221_gb300 import kvcache as KV
    pages, page = 3400000, 16                              # 4.35 GB a pool
    k, v = (torch.empty(pages, 1, page, 80, dtype=torch.uint8, device="cuda") for _ in range(2))
    table = ints([[3, 1700000, 3399999, 2000001]])
    for i, x in enumerate((k, v)):
        x[table[0].long()] = random_rows((4, 1, page), 128, gen(40 + i))
    c = KV.PagedCache(k, v, table)
    c.lens = [60]
    q = torch.randn(1, 8, 128, generator=gen(4), device="cuda")
    kk, vv = (values(slots(c, x, 0, 60), 128)[0] for x in (k, v))
    p = torch.softmax(q[0].double() @ kk.T * 128 ** -0.5, 1)
    out = c.attend(q, ints([60]), 60)
    assert ((out[0].double() - p @ vv).abs() <= 2.0 ** -15 * (p @ vv.abs())).all()   # scores below 2^3: E below 2^-17
    at = ints([0, 0, 0]), ints([15, 47, 60])
    for got, x in zip(c.rows(*at), (k, v)):
        assert torch.equal(got.double(), values(torch.stack([x[t, 0, s] for t, s in ((3, 15), (3399999, 15), (2000001, 12))]), 128)[:, None])


# ---------------------------------------------------------------------------
def spin(x, c, s, rot, interleaved):
    """Rotates tokens x heads x dim in the type of its arguments, every operation rounded on its own."""
    y = x.copy()
    c, s = c[:, None], s[:, None]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., : rot // 2], x[..., rot // 2: rot])
    u, w = a * c - b * s, b * c + a * s
    if interleaved:
        y[..., 0:rot:2], y[..., 1:rot:2] = u, w
    else:
        y[..., : rot // 2], y[..., rot // 2: rot] = u, w
    return y


def append_case(l, heads, kv, dim, rot, page=16, axes=1, interleaved=False, layout="head", typ="q4", seed=0, pad=0,
                norm=True, big=False):
    """Inputs of an append, the cache and the expected queries, keys and values (keys in float32, IEEE operations)."""
    from paper_2607_29221_gb300 import kvcache as KV
    g, rng = gen(seed), np.random.default_rng(seed)
    n = [l - l // 3, l // 3]
    if typ == "q4":
        c = make([x + 5 for x in n], kv, dim, page, layout, seed=seed)
    else:
        pages = sum(-(-(x + 5) // page) for x in n) + 2
        cols = -(-(n[0] + 5) // page)
        table = torch.arange(2 * cols, dtype=torch.int32, device="cuda").reshape(2, cols) % pages
        c = KV.PagedCache.empty(pages + cols, kv, page, dim, table + 1, TYPES[typ])
        c.weight.fill_(3.0)
    seq = ints([0] * n[0] + [1] * n[1])
    slot = ints([i + 3 for i in range(n[0])] + [i + 5 for i in range(n[1])])
    if l > 5:
        slot[2] = -1
    pos = ints(rng.integers(0, 1 << 20 if big else 5000, (axes, l)).tolist())
    wide = torch.randn(l, (heads + 2 * kv) * dim + pad, generator=g, device="cuda")
    wide *= torch.exp(2 * torch.randn(l, 1, generator=g, device="cuda"))
    qkv = wide[:, : (heads + 2 * kv) * dim]
    sections = None if axes == 1 else [rot // 2 - (axes - 1) * (rot // 2 // axes)] + [rot // 2 // axes] * (axes - 1)
    rope = KV.Rope(rot, 500000.0, sections, interleaved) if rot else None
    gains = [torch.exp(torch.randn(dim, generator=g, device="cuda") / 3) for _ in range(2)]
    hn = KV.HeadNorm(dim, 1e-6, *gains) if norm else None
    x = qkv.cpu().numpy().reshape(l, heads + 2 * kv, dim)
    qk, v = x[:, : heads + kv], x[:, heads + kv:]
    ref = qk.astype(np.float64)
    if norm:
        r = 1 / np.sqrt((ref * ref).mean(-1, keepdims=True) + np.float64(np.float32(1e-6)))
        gq, gk = (t.cpu().numpy() for t in gains)
        gain = np.concatenate([np.broadcast_to(gq, (heads, dim)), np.broadcast_to(gk, (kv, dim))])
        ref = ref * r * gain
        qk = qk * r.astype(np.float32) * gain
    if rot:
        phase = (rope.turns.cpu().numpy().view(np.uint64)[:, None] * pos.cpu().numpy().astype(np.uint64)[rope.axis.cpu().numpy()]) >> 32
        angle = phase.astype(np.uint32).view(np.int32).T.astype(np.float64) * (2 * np.pi / 2 ** 32)
        ref = spin(ref, np.cos(angle), np.sin(angle), rot, interleaved)
        qk = spin(qk, np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32), rot, interleaved)
    assert qk.dtype == np.float32
    return c, qkv, seq, slot, pos, rope, hn, ref[:, :heads], qk[:, heads:], v


APPENDS = [
    # l, heads, kv, dim, rot, page, axes, interleaved, layout, pad, norm
    (1, 1, 1, 32, 32, 1, 1, False, "head", 0, True),
    (5, 64, 8, 128, 128, 16, 1, False, "head", 0, True),
    (33, 28, 4, 128, 64, 32, 3, True, "token", 12, False),
    (40, 6, 3, 96, 96, 7, 2, False, "padded", 3, True),
    (17, 3, 1, 192, 64, 16, 1, True, "head", 1, True),
    (9, 40, 40, 64, 0, 16, 1, False, "token", 0, True),
    (50, 2, 2, 256, 256, 8, 4, False, "head", 0, False),
    (21, 5, 5, 160, 80, 20, 1, False, "head", 0, True),
    (700, 64, 8, 128, 128, 16, 1, False, "head", 0, True),
]


@pytest.mark.parametrize("case", range(len(APPENDS)))
@pytest.mark.parametrize("big", [False, True])
def test_append_packs_bit_for_bit(case, big):
    l, heads, kv, dim, rot, page, axes, inter, layout, pad, norm = APPENDS[case]
    c, qkv, seq, slot, pos, rope, hn, wq, wk, wv = append_case(l, heads, kv, dim, rot, page, axes, inter, layout,
                                                               seed=case, pad=pad, norm=norm, big=big)
    before = [t.clone() for t in (c.k, c.v, c.weight, c.position)]
    index = torch.arange(l, dtype=torch.int32, device="cuda") + 77
    q = c.append(qkv, heads, seq, slot, index, rope=rope, pos=pos if rot else None, norm=hn)
    half = np.abs(wq).reshape(l, heads, dim)
    # |a| + |b| of a pair is at most sqrt(2) times the norm of the pair, which the rotation keeps.
    if rot:
        a, b = (half[..., 0:rot:2], half[..., 1:rot:2]) if inter else (half[..., : rot // 2], half[..., rot // 2: rot])
        pair = np.sqrt(2.0) * np.hypot(a, b)
        bound = half.copy()
        if inter:
            bound[..., 0:rot:2] = bound[..., 1:rot:2] = pair
        else:
            bound[..., : rot // 2] = bound[..., rot // 2: rot] = pair
    else:
        bound = half
    assert (np.abs(q.cpu().numpy() - wq) <= 2.0 ** -18 * bound).all()
    live = (slot >= 0).cpu().numpy()
    page_of = c.table[seq.long(), slot.clamp(min=0).long() // page].long()
    mark = torch.zeros(c.weight.shape[0], page, dtype=torch.bool, device="cuda")
    mark[page_of[slot >= 0], slot[slot >= 0].long() % page] = True
    for pool, y in ((c.k, wk), (c.v, wv)):
        got = pool[page_of, :, slot.clamp(min=0).long() % page]
        assert same_bytes(got[slot >= 0], pack(np.ascontiguousarray(y[live])), dim)
    for t, b in zip((c.k, c.v, c.weight, c.position), before):   # nothing else is written
        other = ~mark[:, None].expand(-1, kv, -1)
        assert torch.equal(t[other], b[other])
    assert torch.equal(c.k[..., 5 * dim // 8:], before[0][..., 5 * dim // 8:])   # nor the padding
    sel = (page_of[slot >= 0], slice(None), slot[slot >= 0].long() % page)
    assert (c.weight[sel] == 0).all() and torch.equal(c.position[sel], index[slot >= 0][:, None].expand(-1, kv))


@pytest.mark.parametrize("typ", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("l,heads,kv,dim,rot,axes,inter,pad,gains", [
    (1, 1, 1, 8, 8, 1, False, 0, True), (37, 64, 8, 128, 128, 1, False, 0, True), (20, 3, 2, 80, 40, 2, True, 5, True),
    (11, 5, 1, 256, 256, 1, False, 0, False), (9, 33, 11, 40, 0, 1, False, 2, True), (650, 8, 8, 64, 32, 1, False, 0, True)])
def test_norms_into_caches_of_16_and_32_bits(l, heads, kv, dim, rot, axes, inter, pad, gains, typ):
    """Keys as queries, then rounded once to the cache's type."""
    from paper_2607_29221_gb300 import kvcache as KV
    c, qkv, seq, slot, pos, rope, hn, wq, wk, wv = append_case(l, heads, kv, dim, rot, 16, axes, inter, typ=typ,
                                                               seed=l, pad=pad)
    if not gains:     # gains of one, in 64 bits
        hn = KV.HeadNorm(dim, 1e-6)
        ones = KV.HeadNorm(dim, 1e-6, *(torch.ones(dim, device="cuda") for _ in range(2)))
        a = c.append(qkv, heads, seq, slot, slot, rope=rope, pos=pos, norm=hn)
        k = c.k.clone()
        assert torch.equal(a, c.append(qkv, heads, seq, slot, slot, rope=rope, pos=pos, norm=ones))
        assert torch.equal(k, c.k)
        return
    q = c.append(qkv, heads, seq, slot, slot, rope=rope, pos=pos if rot else None, norm=hn)

    def pairs(y):
        h = np.abs(y.astype(np.float64))
        b = h.copy()
        for i, j in [(slice(0, rot, 2), slice(1, rot, 2)) if inter else (slice(0, rot // 2), slice(rot // 2, rot))] if rot else []:
            b[..., i] = b[..., j] = np.sqrt(2.0) * np.hypot(h[..., i], h[..., j])
        return b
    assert (np.abs(q.cpu().numpy() - wq) <= 2.0 ** -18 * pairs(wq)).all()
    live = slot >= 0
    at = (c.table[seq.long(), slot.clamp(min=0).long() // 16].long()[live], slice(None), slot[live].long() % 16)
    rel, tiny = {"f32": (0.0, 0.0), "bf16": (2.0 ** -8, 0.0), "f16": (2.0 ** -11, 2.0 ** -25)}[typ]
    wk, wv = wk[live.cpu().numpy()].astype(np.float64), wv[live.cpu().numpy()]
    off = np.abs(c.k[at].double().cpu().numpy() - wk)
    err = 2.0 ** -17 * pairs(wk)                           # wk is fp32 too
    assert (off <= err + rel * (np.abs(wk) + err) + tiny).all()
    assert torch.equal(c.v[at], torch.from_numpy(wv).cuda().to(TYPES[typ]))
    assert (c.weight[at] == 0).all()


def test_append_of_extreme_rows():
    """Equal channels, zeros, tiny and huge ones, NaN and infinities, a zero row under the norm."""
    from paper_2607_29221_gb300 import kvcache as KV
    l, dim = 9, 64
    c = make([l], 1, dim, 16)
    x = torch.randn(l, 3, dim, generator=gen(1), device="cuda")
    x[0, 1:] = 0.75
    x[1, 1:] = 0.0
    x[2, 1:] *= 1e-8
    x[3, 1:] *= 1e6                                        # cut to 65000
    x[4, 1, 3], x[4, 2, 40] = math.nan, math.inf
    x[5, 1:, ::2], x[5, 1:, 1::2] = 65504.0, -65504.0
    x[6, 1:] += 1000.0                                     # an offset far above the range
    x[7, 1:] *= 1e30
    x[8, 1:] = -0.0
    at = torch.arange(l, dtype=torch.int32, device="cuda")
    zero = torch.zeros_like(at)
    q = c.append(x.reshape(l, -1), 1, zero, at, at)
    assert torch.equal(q[:, 0], x[:, 0])                   # no rotation: queries as they are
    k, v = (slots(c, p, 0, l)[0] for p in (c.k, c.v))
    y = x.cpu().numpy()
    assert same_bytes(k, pack(y[:, 1]), dim) and same_bytes(v, pack(y[:, 2]), dim)
    got = c.rows(zero, at)
    for g, p in zip(got, (k, v)):
        assert torch.equal(torch.nan_to_num(g[:, 0].double(), nan=7.5), torch.nan_to_num(values(p, dim), nan=7.5))
    assert torch.isnan(got[0][4, 0, :32]).all() and torch.isfinite(got[0][4, 0, 32:]).all()
    assert torch.isfinite(got[0][[0, 1, 2, 3, 5, 6, 7, 8]]).all()
    norm = KV.HeadNorm(dim, 1e-6)
    q = c.append(x.reshape(l, -1), 1, zero, at, at, norm=norm)
    assert torch.isfinite(q[[0, 1, 2, 3, 5, 6, 8]]).all()
    assert (c.rows(zero, at)[0][1] == 0).all()             # 0 / sqrt(eps)
    q = c.append(torch.zeros_like(x).reshape(l, -1), 1, zero, at, at, norm=KV.HeadNorm(dim, 0.0))
    assert torch.isnan(q).all() and torch.isnan(c.rows(zero, at)[0]).all()   # 0 / 0, as rmsnorm has it


def test_append_without_slots():
    """Negative slots, slots past the table, sequences that are none, slots without a page: rotated, not stored."""
    c = make([20, 20], 2, 64, 16)
    before = (c.k.clone(), c.v.clone(), c.weight.clone(), c.position.clone())
    x = torch.randn(6, 5 * 64, generator=gen(2), device="cuda")
    c.table[1, 1] = 0x7fffffff
    q = c.append(x, 1, ints([0, 0, -1, 2, 1, 0]), ints([-1, 32, 3, 3, 17, 1 << 30]), ints([0] * 6))
    assert torch.equal(q.reshape(6, 64), x[:, :64])
    assert all(torch.equal(a, b) for a, b in zip(before, (c.k, c.v, c.weight, c.position)))
    k, v = c.rows(ints([0, 0, -1, 2, 1, 0]), ints([-1, 32, 3, 3, 17, 1 << 30]))
    assert (k == 0).all() and (v == 0).all() and k.shape == (6, 2, 64)


@pytest.mark.parametrize("typ", ["q4", "f32", "bf16", "f16"])
@pytest.mark.parametrize("l,kv,dim,page", [(0, 2, 32, 4), (1, 1, 32, 1), (77, 8, 128, 16), (300, 3, 96, 7), (45, 2, 256, 64)])
def test_rows(l, kv, dim, page, typ):
    from paper_2607_29221_gb300 import kvcache as KV
    lens = [300, 40, 120]
    c = make(lens, kv, dim, page, seed=l)
    if typ != "q4":
        shape = (c.k.shape[0], kv, page, dim)
        c = KV.PagedCache(*(torch.randn(shape, generator=gen(i), device="cuda").to(TYPES[typ]).transpose(1, 2).contiguous().transpose(1, 2)
                            for i in range(2)), c.table)
    rng = np.random.default_rng(l)
    seq = rng.integers(0, 3, l)
    slot = np.array([rng.integers(0, lens[i]) for i in seq], dtype=np.int64)
    k, v = c.rows(ints(seq.tolist()), ints(slot.tolist()))
    kt, vt = c.rows(ints(seq.tolist()), ints(slot.tolist()), token_major=False)
    assert k.shape == (l, kv, dim) and kt.shape == (kv, l, dim)
    assert torch.equal(k, kt.transpose(0, 1)) and torch.equal(v, vt.transpose(0, 1))
    at = c.table[torch.tensor(seq, device="cuda"), torch.tensor(slot // page, device="cuda")].long()
    for got, pool in ((k, c.k), (v, c.v)):
        want = pool[at, :, torch.tensor(slot % page, device="cuda")]
        if typ == "q4":
            assert got.dtype == torch.float16 and torch.equal(got.double(), values(want, dim))
        else:
            assert torch.equal(got, want)
    if l > 1:
        a, b = c.read(1, 33)
        assert a.shape == b.shape == (kv, 33, dim)
        want = slots(c, c.k, 1, 33)
        assert torch.equal(a.double(), values(want, dim) if typ == "q4" else want.double())


def test_every_code_step_and_base():
    """All 16 codes with steps and bases of any exponent and sign, one fp16 rounding of the sum."""
    from paper_2607_29221_gb300 import kvcache as KV
    n, dim = 4096, 64
    rng = np.random.default_rng(3)
    raw = rng.integers(0, 256, (n, 1, 1, KV.row_bytes(dim)), dtype=np.uint8)
    half = raw[..., dim // 2: dim // 2 + 8].view(np.uint16)
    half[(half & 0x7c00) == 0x7c00] &= 0x83ff              # finite
    k = torch.from_numpy(raw).cuda()
    c = KV.PagedCache(k, k.clone(), torch.arange(n, dtype=torch.int32, device="cuda")[:, None])
    got = c.rows(torch.arange(n, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda"))
    assert torch.equal(got[0][:, 0].double(), values(k[:, 0, 0], dim)) and torch.equal(got[0], got[1])


# ---------------------------------------------------------------------------
@pytest.mark.parametrize("most,keep,recent,page,layout", [(300, 299, 0, 16, "head"), (300, 100, 20, 16, "token"),
                                                         (9000, 2500, 64, 20, "head"), (70, 64, 10, 7, "padded")])
def test_eviction_moves_packed_rows(most, keep, recent, page, layout):
    kv, dim = 2, 96
    lens = [most, most // 2, 0, most - 1]
    c = make(lens, kv, dim, page, layout, seed=most)
    for i, n in enumerate(lens):
        ids = c.table[i, : -(-n // page)].long()
        c.position[ids] = torch.arange(len(ids) * page, dtype=torch.int32, device="cuda").reshape(-1, 1, page).expand(-1, kv, -1)
    tags = [[slots(c, x, i, n).clone() for x in (c.k, c.v, c.position, c.weight)] for i, n in enumerate(lens)]
    low = ints([n - recent for n in lens])
    new = c.evict(ints(lens), most, keep, recent_from=low if recent else None)
    assert new.tolist() == [min(n, keep) for n in lens]
    for i, n in enumerate(lens):
        if not n:
            continue
        for h in range(kv):
            w = tags[i][3][h].double().clone()
            if recent:
                w[n - recent:] = math.inf
            gone = torch.zeros(n, dtype=torch.bool, device="cuda")
            if n > keep:
                gone[torch.argsort(w, stable=True)[: n - keep]] = True
            src = torch.arange(n, device="cuda")[: min(n, keep)]
            holes = gone[:keep].nonzero()[:, 0]
            src = src.clone()
            src[holes] = keep + (~gone[keep:]).nonzero()[:, 0]
            for tag, pool in zip(tags[i], (c.k, c.v, c.position, c.weight)):
                got = slots(c, pool, i, min(n, keep))[h]
                want = tag[h][src]
                if got.dtype == torch.uint8:
                    got, want = got[:, : 5 * dim // 8], want[:, : 5 * dim // 8]
                assert torch.equal(got, want)


def test_a_decode_loop_of_all_of_them():
    """append with norms, attend with weights, evict, append again, read: the cache's own bytes are the reference's."""
    from paper_2607_29221_gb300 import kvcache as KV
    seqs, heads, kv, dim, page = 3, 8, 2, 128, 16
    table = torch.arange(1, 1 + seqs * 6, dtype=torch.int32, device="cuda").reshape(seqs, 6)
    c = KV.PagedCache.empty(seqs * 6 + 1, kv, page, dim, table, KV.INT4)
    rope, g = KV.Rope(dim, 500000.0), gen(11)
    norm = KV.HeadNorm(dim, 1e-6, *(torch.rand(dim, generator=g, device="cuda") + 0.5 for _ in range(2)))
    host, seen = [0] * seqs, 0
    rows = torch.arange(seqs, dtype=torch.int32, device="cuda")
    for step in range(70):
        x = torch.randn(seqs, (heads + 2 * kv) * dim, generator=g, device="cuda")
        lens, pos = ints(host), ints([seen] * seqs)
        q = c.append(x, heads, rows, lens, pos, rope=rope, pos=pos, norm=norm)
        host, seen = [n + 1 for n in host], seen + 1
        c.lens = host
        ref = reference(c, q, dim ** -0.5, ints([seen - 50] * seqs), 0.9)
        out = c.attend(q, ints(host), max(host), first=ints([seen - 50] * seqs), decay=0.9)
        check(c, q, out, ref)
        if max(host) > 40:
            new = c.evict(ints(host), max(host), 40, recent_from=ints([seen - 8] * seqs))
            host = new.tolist()
    k, v = c.read(1, host[1])
    assert torch.equal(k.double(), values(slots(c, c.k, 1, host[1]), dim))
    assert torch.equal(v.double(), values(slots(c, c.v, 1, host[1]), dim))


def test_append_and_rows_on_another_stream_in_a_graph():
    from paper_2607_29221_gb300 import kvcache as KV
    c, qkv, seq, slot, pos, rope, hn, wq, wk, wv = append_case(33, 8, 2, 128, 128, seed=4)
    d = type(c)(c.k.clone(), c.v.clone(), c.table, position=c.position.clone())
    index = slot.clone()
    want_q = d.append(qkv, 8, seq, slot, index, rope=rope, pos=pos, norm=hn)
    want = d.rows(seq, slot)
    s, graph, out = torch.cuda.Stream(), torch.cuda.CUDAGraph(), torch.empty(33, 8, 128, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        c.append(qkv, 8, seq, slot, index, rope=rope, pos=pos, norm=hn, out=out)
        got = c.rows(seq, slot)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want_q) and all(torch.equal(a, b) for a, b in zip(got, want))
    # One token at a time gives what all of them give together.
    e = type(c)(torch.zeros_like(c.k), torch.zeros_like(c.v), c.table)
    for t in range(33):
        q1 = e.append(qkv[t: t + 1], 8, seq[t: t + 1], slot[t: t + 1], rope=rope, pos=pos[:, t: t + 1], norm=hn)
        assert torch.equal(q1[0], want_q[t])
    assert all(torch.equal(a, b) for a, b in zip(e.rows(seq, slot), want))


def test_read_takes_the_table_as_other_types_do():
    """Sequences are counted from the end where negative, none past the table is read, and slots end with the table."""
    from paper_2607_29221_gb300 import kvcache as KV
    c = make([12, 7], 2, 64, 4, seed=3)
    shape = (c.k.shape[0], 2, 4, 64)
    f = KV.PagedCache(torch.zeros(shape, device="cuda"), torch.zeros(shape, device="cuda"), torch.zeros_like(c.table))
    most = c.table.shape[1] * 4
    for n in (1, 5, most, most + 9):
        assert [x.shape for x in c.read(1, n)] == [x.shape for x in f.read(1, n)]
    assert all(torch.equal(a, b) for a, b in zip(c.read(-2, 12), c.read(0, 12)))
    for seq in (2, -3):
        for cache in (c, f):
            with pytest.raises(IndexError):
                cache.read(seq, 4)


def test_a_session_refuses_norms_of_another_head():
    from paper_2607_29221_gb300 import decoder as DEC, kvcache as KV, mosaic as M, protocol as PR, workloads as wl
    from paper_2607_29221_gb300.session import DecodeSession
    s = DEC.LayerShape(hidden=256, n_heads=8, n_kv=2, head_dim=64, ffn=512)
    layer = DEC.SecureDecoderLayer(PR.Protocol(wl.mask_key(), M.default_params()), DEC.LayerWeights(s))
    for norm in (KV.HeadNorm(32), KV.HeadNorm(64, 1e-6, torch.ones(64))):      # its size, host gains
        with pytest.raises(ValueError, match="norm"):
            DecodeSession(layer, seqs=1, max_len=16, dtype=KV.INT4, norm=norm)


def test_a_session_on_a_4_bit_cache():
    """Prefill, steps and a budget through a masked layer: every step's attention is that over the cache's own values."""
    from paper_2607_29221_gb300 import decoder as DEC, kvcache as KV, mosaic as M, protocol as PR, workloads as wl
    from paper_2607_29221_gb300.session import DecodeSession
    s = DEC.LayerShape(hidden=256, n_heads=8, n_kv=2, head_dim=64, ffn=512)
    layer = DEC.SecureDecoderLayer(PR.Protocol(wl.mask_key(), M.default_params()), DEC.LayerWeights(s))
    norm = KV.HeadNorm(64, 1e-6, torch.full((64,), 1.25, device="cuda"))
    ses = DecodeSession(layer, seqs=2, max_len=64, keep=24, recent=4, dtype=KV.INT4, norm=norm)
    assert ses.cache.k.dtype == KV.INT4
    g = gen(5)
    ses.prefill(0, torch.randn(20, 256, generator=g, device="cuda"))
    ses.prefill(1, torch.randn(9, 256, generator=g, device="cuda"))
    plain = ses.cache.attend

    def attend(q, lens, max_len, **kw):
        ses.cache.lens = lens.tolist()
        ref = reference(ses.cache, q, 64 ** -0.5)
        out = plain(q, lens, max_len, **kw)
        check(ses.cache, q, out, ref)
        return out
    ses.cache.attend = attend
    for _ in range(12):
        y = ses.step(torch.randn(2, 256, generator=g, device="cuda"))
        assert torch.isfinite(y).all()
    assert max(ses.host_lens) <= 24 and ses.lens.tolist() == ses.host_lens


# ---------------------------------------------------------------------------
# Scores in units of log2: the scale whose product with log2(e) is one in fp32.
def unit_scale():
    f = np.float32
    near = [f(math.log(2))]
    for _ in range(4):
        near += [np.nextafter(near[-1], f(1))]
    near += [np.nextafter(f(math.log(2)), f(0))]
    return float(next(x for x in near if f(x * f(1.44269504088896341)) == 1))


def level(pool, group, dim, base):
    """Channels of a group of 32 of all rows: `base`, whatever the codes."""
    at = dim // 2 + 4 * group
    pool[..., at: at + 4] = torch.stack([torch.zeros_like(base), base], -1).half().contiguous().view(torch.uint8)


@pytest.mark.parametrize("lens,heads,kv,dim,page,window", [
    ([5, 40, 300], 16, 2, 64, 16, False), ([5, 40, 300], 24, 2, 64, 20, True), ([5, 40, 300, 5000], 16, 2, 128, 16, True),
    ([33, 3000], 16, 1, 128, 20, False), ([40, 700], 32, 2, 256, 8, True)])
def test_attention_of_large_equal_scores(lens, heads, kv, dim, page, window):
    """Scores of 2^23 to 2^119 of both signs, the same in every slot: means of the values, whatever the score.
    Probabilities are the same power of two; what remains is the sums' and the join's 2^-19."""
    c = make(lens, kv, dim, page, seed=7)
    for group in range(dim // 32):
        level(c.k, group, dim, torch.full(c.k.shape[:3], 1.0, device="cuda"))
    tops = [2.0 ** 23 + 1, 16777240.0, 3e7, 1e8, 2.0 ** 28 + 32, 1e10, 1e20, 5e35]
    q = torch.zeros(len(lens), heads, dim, device="cuda")
    q[..., 1] = torch.tensor([t * s for s in (1, -1) for t in tops] * 2, device="cuda")[:heads]
    first = None
    if window:
        c.position.copy_(torch.randint(0, 1000, c.position.shape, generator=gen(8), device="cuda"))
        first = torch.full((len(lens),), 300, dtype=torch.int32, device="cuda")
    want, _, weights = reference(c, torch.zeros_like(q), 1.0, first, 0.5)      # equal scores: those of no query
    size = torch.zeros_like(want)
    for i, n in enumerate(lens):
        on = slots(c, c.position, i, n) >= (-1 if first is None else 300)
        v = values(slots(c, c.v, i, n), dim).abs() * on[..., None]
        size[i] = (v.sum(1) / on.sum(1, keepdim=True).clamp(min=1)).repeat_interleave(heads // kv, 0)
    out = c.attend(q, ints(lens), max(lens), first=first, scale=unit_scale(), decay=0.5)
    off = (out.double() - want).abs()
    assert (off <= 2.0 ** -19 * size).all(), [h for h in range(heads) if not (off[:, h] <= 2.0 ** -19 * size[:, h]).all()]
    for i, n in enumerate(lens):
        w = weights[i][0]
        assert ((slots(c, c.weight, i, n).double() - w).abs() <= 2.0 ** -18 * w + 1e-30).all(), i


@pytest.mark.parametrize("top", [2.0 ** 24, -2.0 ** 24, 2.0 ** 25, -2.0 ** 25 - 8, 2.0 ** 26 - 512, -2.0 ** 26 + 512])
@pytest.mark.parametrize("lens", [[9, 50, 400], [31, 2000, 5000]])
def test_attention_of_large_scores_that_differ(lens, top):
    """Scores top - 8 j, j < 4: multiples of 8 below 2^26 + 2^25, exact in fp32 and in two fp16 terms of the
    queries (2^25 and 1, scaled to 2^14 and 2^-11); probabilities 2^-8j are exact too."""
    dim, kv, heads = 64, 2, 16
    c = make(lens, kv, dim, 16, seed=3)
    j = torch.randint(0, 4, c.k.shape[:3], generator=gen(4), device="cuda").float()
    level(c.k, 0, dim, torch.ones_like(j))
    level(c.k, 1, dim, -8.0 * j)
    q = torch.zeros(len(lens), heads, dim, device="cuda")
    q[..., 1], q[..., 40] = top, 1.0
    out = c.attend(q, ints(lens), max(lens), scale=unit_scale())
    for i, n in enumerate(lens):
        p = 2.0 ** (-8.0 * slots(c, j, i, n).double())
        p = p / p.sum(1, keepdim=True)
        v = values(slots(c, c.v, i, n), dim)
        got = out[i].reshape(kv, heads // kv, dim).double()
        want, size = (torch.einsum("hn,hnd->hd", p, x)[:, None] for x in (v, v.abs()))
        tol = 2.0 ** -19 * size + (2.0 ** -40 * p.amax(1)[:, None] * v.abs().sum(1))[:, None]
        assert ((got - want).abs() <= tol).all(), (i, float(((got - want).abs() / tol).max()))


@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("lens,heads,kv,page", [([5, 32, 40, 300, 77], 16, 2, 16), ([5, 40, 300, 5000, 9], 48, 2, 20),
                                                ([1, 2, 3, 31, 33], 2, 2, 8)])
def test_attention_of_scores_beyond_fp32(lens, heads, kv, page, sign):
    """A finite query and a finite key whose product is beyond fp32, of either sign: the score counts as NaN, and so
    do the row's output and the weights of its key/value head; not where the slot does not count."""
    dim = 64
    c = make(lens, kv, dim, page, seed=13)
    at = lambda i, s: (int(c.table[i, s // page]), slice(None), s % page)
    level(c.k, 0, dim, torch.zeros(c.k.shape[:3], device="cuda"))
    q = torch.randn(len(lens), heads, dim, generator=gen(14), device="cuda")
    per = heads // kv
    q[..., :32] = 0.0
    q[:, per - 1] = 0.0
    q[:, per - 1, 4] = sign * 1e37                              # the first key/value head's last query
    last = len(lens) - 1
    first = torch.zeros(len(lens), dtype=torch.int32, device="cuda")
    first[last] = 1
    c.position.fill_(1)
    for i, n in enumerate(lens):
        row = c.k[at(i, n // 2)]
        row[..., dim // 2: dim // 2 + 4] = torch.tensor([0.0, 65000.0], dtype=torch.float16, device="cuda").view(torch.uint8)
        c.k[at(i, n // 2)] = row
    c.position[at(last, lens[last] // 2)] = 0                   # of the last sequence that slot is below the bound
    calm = q.clone()
    calm[:, per - 1, 4] = 0.0
    want, tol, weights = reference(c, calm, 0.125, first)
    out = c.attend(q, ints(lens), max(lens), first=first)
    other = [h for h in range(heads) if h != per - 1]
    assert torch.isnan(out[:last, per - 1]).all()
    assert ((out[:, other].double() - want[:, other]).abs() <= tol[:, other]).all()
    assert ((out[last].double() - want[last]).abs() <= tol[last]).all()
    for i, n in enumerate(lens):
        w, wt = weights[i]
        got = slots(c, c.weight, i, n).double()
        assert ((got[1] - w[1]).abs() <= wt[1]).all()
        if i < last:
            assert torch.isnan(got[0]).all(), i
        else:
            assert ((got[0] - w[0]).abs() <= wt[0]).all()
    bare = type(c)(c.k, c.v, c.table, position=c.position)     # and without weights
    again = bare.attend(q, ints(lens), max(lens), first=first)
    assert torch.equal(torch.nan_to_num(again, nan=7.5), torch.nan_to_num(out, nan=7.5))


@pytest.mark.parametrize("typ", ["q4", "f32", "bf16", "f16"])
@pytest.mark.parametrize("eps", [0.0, 1e-6, 1e-38, 3e38])
@pytest.mark.parametrize("dim,heads,kv,rot", [(64, 3, 2, 64), (96, 5, 3, 32), (256, 2, 1, 0), (32, 40, 8, 32)])
def test_norms_of_heads_of_any_size(dim, heads, kv, rot, eps, typ):
    """Heads from 2^-140 to 2^122 in one call, beside ordinary ones: what their squares are does not matter.
    1 / rms is rounded once to 24 bits, whatever its exponent: rows of 4 bits are equal, the rest as elsewhere."""
    from paper_2607_29221_gb300 import kvcache as KV
    f = np.float32
    powers = [0, -140, -126, -80, -63, -62, -50, -49, -20, 20, 49, 50, 51, 60, 63, 64, 100, 120]
    l, rng = len(powers), np.random.default_rng(dim)
    x = rng.standard_normal((l, heads + 2 * kv, dim)).astype(f)
    power = np.stack([np.roll(powers, h) for h in range(heads + kv)], 1)       # a token has heads of several sizes
    x[:, : heads + kv] = np.ldexp(x[:, : heads + kv], power[..., None].astype(np.int32))
    x[:, : heads + kv, 1] = np.ldexp(x[:, : heads + kv, 1], -20)               # and a head channels of several
    gains = [np.exp(rng.standard_normal(dim) / 3).astype(f) for _ in range(2)]
    qk = x[:, : heads + kv].astype(np.float64)
    gain = np.concatenate([np.broadcast_to(g, (n, dim)) for g, n in zip(gains, (heads, kv))])
    # Scaled by a power of two: r keeps its 24 bits.
    up = np.maximum(np.frexp(np.abs(qk).max(-1, keepdims=True))[1], np.frexp(np.sqrt(np.float64(f(eps))))[1] if eps else -10000)
    near = np.ldexp(qk, -up)
    r = 1 / np.sqrt((near * near).mean(-1, keepdims=True) + np.ldexp(np.float64(f(eps)), -2 * up))
    ref = near * r * gain
    y = (near * r.astype(f).astype(np.float64)).astype(f) * gain
    rope = KV.Rope(rot, 500000.0) if rot else None
    pos = ints(rng.integers(0, 5000, l).tolist())
    if rot:
        phase = (rope.turns.cpu().numpy().view(np.uint64)[:, None] * pos.cpu().numpy().astype(np.uint64)[None]) >> 32
        angle = phase.astype(np.uint32).view(np.int32).T.astype(np.float64) * (2 * np.pi / 2 ** 32)
        ref = spin(ref, np.cos(angle), np.sin(angle), rot, False)
        y = spin(y, np.cos(angle).astype(f), np.sin(angle).astype(f), rot, False)
    assert y.dtype == f
    table = torch.arange(1, 4, dtype=torch.int32, device="cuda")[None]
    c = KV.PagedCache.empty(4, kv, 8, dim, table, KV.INT4 if typ == "q4" else TYPES[typ])
    at, zero = torch.arange(l, dtype=torch.int32, device="cuda"), torch.zeros(l, dtype=torch.int32, device="cuda")
    hn = KV.HeadNorm(dim, eps, *(torch.from_numpy(g).cuda() for g in gains))
    q = c.append(torch.from_numpy(x.reshape(l, -1)).cuda(), heads, zero, at, at, rope=rope, pos=pos if rot else None, norm=hn)

    def pairs(z):
        b = np.abs(z)
        if rot:
            half = b.copy()
            b[..., : rot // 2] = b[..., rot // 2: rot] = np.sqrt(2.0) * np.hypot(half[..., : rot // 2], half[..., rot // 2: rot])
        return b
    # Of results near the end of fp32: a scaled channel is off by up to 2^-150, times r (at most 16 here), a gain
    # (below 8) and two terms of a rotation; five roundings besides.
    tiny = 2.0 ** -141
    assert (np.abs(q.cpu().numpy() - ref[:, :heads]) <= 2.0 ** -18 * pairs(ref[:, :heads]) + tiny).all()
    k = slots(c, c.k, 0, l).transpose(0, 1)
    if typ == "q4":
        assert same_bytes(k, pack(np.ascontiguousarray(y[:, heads:])), dim)
        return
    rel, least = {"f32": (0.0, tiny), "bf16": (2.0 ** -8, 2.0 ** -134), "f16": (2.0 ** -11, 2.0 ** -25)}[typ]
    want = ref[:, heads:]
    err = 2.0 ** -18 * pairs(want) + tiny
    assert (np.abs(k.double().cpu().numpy() - want) <= err + rel * (np.abs(want) + err) + least).all()

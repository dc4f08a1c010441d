"""A key/value cache held in 4 bits, and per-head norms on the way into a cache, as measurable cases.

A case is one call of one operator, as a serving loop makes it between the
secure linears of a decoder layer:

  attend  attention of one new token per sequence over the pages of a 4-bit
          cache, with the accumulated attention weight of every slot if kept
  append  norms and rotates the queries and keys of new tokens, packs keys and
          values into 4 bits on the way into the pages, and reads the new rows
          back as a prefill does (the values that they now stand for)
  norm    the same norms and rotation into a cache of 16 or 32 bits
  read    the rows of a list of cached tokens out of a 4-bit cache

``own`` says who computes: the framework's kernels, or elementary torch
operations in 32 bits.

A row of the 4-bit cache is head_dim codes of 4 bits (channel 0 in the low half
of byte 0), then for each 32 channels a step and a base in fp16, padded to 16
bytes.  Code c stands for base + c step, rounded once to fp16.  base is the least
channel of the 32 and step 1/15 of their range, each rounded to fp16; the code is
(y - base) / step, rounded to nearest.  Channels are cut to 65000 before that.

Head counts are those of the 70B layer (64 query and 8 key/value heads of 128)
and of the 7B projections (32 heads of 128), and generic ones.  Keys have a few
outlier channels; accumulated weights are log-normal.  Pages of a sequence are
scattered over the pool.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "q4": torch.uint8}
ROPE_BASE = 500000.0
EPS = 1e-6
GROUP = 32          # channels that share a step and a base
MOST = 65000.0


def listed():
    return [
        # The first tokens of a conversation: one short sequence, latency is all of it.
        {"name": "attend4_70b_1x37", "kind": "attend", "seqs": 1, "max_len": 37, "lens": "full", "heads": 64, "kv": 8,
         "dim": 128, "page": 16, "type": "q4", "weights": False, "window": 0, "layout": "head", "decay": 1.0},
        # One user with a very long document: what a cache of 4 bits is for.
        {"name": "attend4_70b_1x131071", "kind": "attend", "seqs": 1, "max_len": 131071, "lens": "full", "heads": 64,
         "kv": 8, "dim": 128, "page": 64, "type": "q4", "weights": False, "window": 0, "layout": "head",
         "decay": 1.0},
        # A full serving batch of the 70B layer with lengths of every kind, weights kept for eviction.
        {"name": "attend4_70b_64x16384", "kind": "attend", "seqs": 64, "max_len": 16384, "lens": "ragged", "heads": 64,
         "kv": 8, "dim": 128, "page": 16, "type": "q4", "weights": True, "window": 0, "layout": "head",
         "decay": 1.0},
        # A 7B model's batch: every query head has a key/value head of its own.
        {"name": "attend4_7b_48x2000", "kind": "attend", "seqs": 48, "max_len": 2000, "lens": "ragged", "heads": 32,
         "kv": 32, "dim": 128, "page": 32, "type": "q4", "weights": False, "window": 0, "layout": "head",
         "decay": 1.0},
        # Many short chats with a sliding window on a token-major cache; some sequences are empty.
        {"name": "attend4_window_400x1500", "kind": "attend", "seqs": 400, "max_len": 1500, "lens": "zeros",
         "heads": 24, "kv": 8, "dim": 64, "page": 20, "type": "q4", "weights": False, "window": 512,
         "layout": "token", "decay": 1.0},
        # A decode step of 32 sequences of the 70B layer, with norms.
        {"name": "append4_70b_32", "kind": "append", "tokens": 32, "seqs": 32, "max_len": 2048, "heads": 64, "kv": 8,
         "dim": 128, "rot": 128, "axes": 1, "interleaved": False, "page": 16, "type": "q4", "pad": 0,
         "layout": "head", "norm": True},
        # Prefill of 2048 tokens of the 70B layer, with norms.
        {"name": "append4_70b_2048", "kind": "append", "tokens": 2048, "seqs": 1, "max_len": 2048, "heads": 64,
         "kv": 8, "dim": 128, "rot": 128, "axes": 1, "interleaved": False, "page": 16, "type": "q4", "pad": 0,
         "layout": "head", "norm": True},
        # A clip's frames with positions in time, height and width, rows padded to a wider product, no norms.
        {"name": "append4_video_9001", "kind": "append", "tokens": 9001, "seqs": 2, "max_len": 4501, "heads": 28,
         "kv": 4, "dim": 128, "rot": 128, "axes": 3, "interleaved": True, "page": 32, "type": "q4", "pad": 12,
         "layout": "token", "norm": False},
        # A decode step of 32 sequences into a 16-bit cache.
        {"name": "norm_70b_32", "kind": "norm", "tokens": 32, "seqs": 32, "max_len": 2048, "heads": 64, "kv": 8,
         "dim": 128, "rot": 128, "axes": 1, "interleaved": False, "page": 16, "type": "bf16", "pad": 0,
         "layout": "head", "norm": True},
        # Prefill of a batch of prompts into the unrounded cache of the fp32 glue, half of each head rotated.
        {"name": "norm_f32_5003", "kind": "norm", "tokens": 5003, "seqs": 5, "max_len": 1100, "heads": 32, "kv": 32,
         "dim": 128, "rot": 64, "axes": 1, "interleaved": False, "page": 16, "type": "f32", "pad": 0,
         "layout": "head", "norm": True},
        # A short prompt's keys and values for the attention over it.
        {"name": "read4_70b_61", "kind": "read", "tokens": 61, "seqs": 1, "max_len": 61, "kv": 8, "dim": 128,
         "page": 16, "type": "q4", "layout": "head"},
        # A long document's, for the next piece of its prefill.
        {"name": "read4_70b_32768", "kind": "read", "tokens": 32768, "seqs": 1, "max_len": 32768, "kv": 8, "dim": 128,
         "page": 64, "type": "q4", "layout": "head"},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "attend", "append", "append", "norm", "read"])
    typ = rng.choice(["bf16", "f16", "f32"]) if kind == "norm" else "q4"
    dim = rng.choice([128, 128, 128, 64, 96, 256, 32, 192] if typ == "q4" else [128, 128, 64, 80, 256, 40])
    kv = rng.choice([1, 2, 4, 8, 8, 32])
    group = rng.choice([1, 2, 3, 4, 7, 8, 8, 16]) if kv < 32 else rng.choice([1, 2])
    page = rng.choice([16, 16, 16, 32, 64, 8, 20, 1])
    case = {"kind": kind, "kv": kv, "dim": dim, "page": page, "type": typ,
            "layout": rng.choice(["head", "head", "token"])}
    if kind == "attend":
        seqs, lens = _log(rng, 1, 400), rng.choice(["full", "ragged", "ragged", "zeros"])
        max_len = _log(rng, 1, 131072)
        heads = kv * group
        while seqs * max_len * max(kv * dim, heads * dim // 8) > (64 * 16384 if lens == "ragged" else 131072) * 8 * 128:
            max_len = -(-max_len // 2)
            seqs = max(1, seqs // 2) if max_len < 64 else seqs
        return {**case, "seqs": seqs, "max_len": max_len, "lens": lens, "heads": heads, "weights": rng.random() < 0.5,
                "window": rng.choice([0, 0, 0, _log(rng, 1, 4096)]), "decay": rng.choice([1.0, 0.9375])}
    if kind == "read":
        tokens, seqs = _log(rng, 1, 32768), _log(rng, 1, 64)
        while tokens * kv * dim > 32768 * 8 * 128:
            tokens //= 2
        seqs = min(tokens, seqs)
        return {**case, "tokens": tokens, "seqs": seqs, "max_len": -(-tokens // seqs) + rng.randint(0, 500)}
    tokens, axes, heads = _log(rng, 1, 9000), rng.choice([1, 1, 2, 3, 4]), min(64, kv * group)
    while tokens * (heads + 2 * kv) * dim > 9000 * 36 * 128:
        tokens //= 2
    seqs = min(tokens, _log(rng, 1, 64))
    return {**case, "tokens": tokens, "seqs": seqs, "max_len": -(-tokens // seqs) + rng.randint(0, 500),
            "heads": heads, "rot": dim if rng.random() < 0.75 or dim % 16 else dim // 2, "axes": axes,
            "interleaved": rng.random() < 0.4, "pad": rng.choice([0, 0, 4, 37]),
            "norm": kind == "norm" or rng.random() < 0.5}


# ---------------------------------------------------------------------------
def _row(case):
    """Bytes (4-bit caches) or channels of a cached row."""
    return -(-5 * case["dim"] // 128) * 16 if case["type"] == "q4" else case["dim"]


def _gen(seed, salt=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(1_000_003 * seed + salt)
    return g


def _lengths(case):
    """Lengths of the sequences, the same for every seed up to their order."""
    n, most = case["seqs"], case["max_len"]
    if case["lens"] == "full":
        return [most] * n
    lens = [max(1, most * (i + 1) // n) for i in range(n)]
    return [0 if case["lens"] == "zeros" and i % 8 == 3 else v for i, v in enumerate(lens)]


def _table(case, lens, g):
    """Page table (seqs x columns) of scattered pages; entries past a sequence's last page are 0."""
    page = case["page"]
    need = [-(-v // page) for v in lens]
    cols, pages = max(1, max(need)), sum(need) + 3
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    counts = torch.tensor(need, device="cuda")
    at = torch.cumsum(counts, 0) - counts
    col = torch.arange(cols, device="cuda")
    ids = order[(at[:, None] + col[None]).clamp(max=pages - 1)]
    return torch.where(col[None] < counts[:, None], ids, torch.zeros_like(ids)), pages


def _pool(case, pages, g, outliers):
    """Pages of N(0, 1) rows, the same few channels of a head four times as large in keys."""
    shape = ((pages, case["kv"], case["page"]) if case["layout"] == "head" else (pages, case["page"], case["kv"]))
    x = torch.empty(*shape, _row(case), dtype=TYPES[case["type"]], device="cuda")
    if case["type"] == "q4":
        x.zero_()
    rows = x.view(-1, x.shape[-1])
    at = torch.randperm(case["dim"], generator=g, device="cuda")[:2]
    for i in range(0, rows.shape[0], 1 << 20):
        part = rows[i: i + (1 << 20)]
        y = torch.randn(part.shape[0], case["dim"], generator=g, device="cuda")
        if outliers:
            y[:, at] *= 4.0
        if case["type"] == "q4":
            packed = _pack(y)
            part[:, : packed.shape[1]] = packed
        else:
            part.copy_(y)
    return x if case["layout"] == "head" else x.transpose(1, 2)


def _turns(rot):
    """Frequencies of the rotary pairs in turns a position, scaled by 2^64."""
    freq = ROPE_BASE ** (-2.0 * np.arange(rot // 2, dtype=np.float64) / rot)
    return np.rint(freq / (2.0 * math.pi) * 2.0 ** 64).astype(np.int64)


def _sections(case):
    """Rotary pairs of each axis: a quarter to the first, the rest shared."""
    pairs, axes = case["rot"] // 2, case["axes"]
    if axes == 1:
        return [pairs]
    first = max(1, pairs // 4)
    rest = [(pairs - first) // (axes - 1)] * (axes - 1)
    rest[-1] += pairs - first - sum(rest)
    return [first] + rest


def _inputs(case, seed):
    """The tensors of a case: what `prepare` and `exact` start from."""
    g = _gen(seed)
    s = {"case": case, "scale": 1.0 / math.sqrt(case["dim"])}
    kind, page, kv, dim = case["kind"], case["page"], case["kv"], case["dim"]
    if kind == "attend":
        lens = torch.tensor(_lengths(case), device="cuda")[torch.randperm(case["seqs"], generator=g, device="cuda")]
        s["lens"] = lens.to(torch.int32)
        s["table"], pages = _table(case, lens.tolist(), g)
    else:
        tokens, seqs = case["tokens"], case["seqs"]
        per = [tokens // seqs + (i < tokens % seqs) for i in range(seqs)]
        start = [(37 * i + 11) % (case["max_len"] - per[i] + 1) for i in range(seqs)]
        s["table"], pages = _table(case, [a + b for a, b in zip(start, per)], g)
        s["seq"] = torch.repeat_interleave(torch.arange(seqs, device="cuda"),
                                           torch.tensor(per, device="cuda")).to(torch.int32)
        first = torch.tensor(np.cumsum([0] + per[:-1]), device="cuda")
        nth = torch.arange(tokens, device="cuda") - first[s["seq"].long()]
        s["slot"] = (nth + torch.tensor(start, device="cuda")[s["seq"].long()]).to(torch.int32)
    s["k"], s["v"] = _pool(case, pages, g, True), _pool(case, pages, g, False)
    if kind == "read":
        return s
    shape = (pages, kv, page)
    s["weight"] = torch.randn(shape, generator=g, device="cuda").mul_(2.0).exp_()
    s["position"] = torch.zeros(shape, dtype=torch.int32, device="cuda")
    if kind != "attend":
        s["index"] = s["slot"] + 1000                      # 1000 earlier tokens have been evicted
        if tokens > 16:
            s["slot"][-1] = -1                             # a padding row of a static batch
        # Text: one running position; video: frames of 16 x 9 patches after the text before them.
        at = s["index"]
        axes = [at, 1000 + nth % 144 // 9, 1000 + nth % 9, at // 2]
        if case["axes"] > 1:
            axes[0] = 1000 + nth // 144
        s["pos"] = torch.stack([a.to(torch.int32) for a in axes[: case["axes"]]]).contiguous()
        width = (case["heads"] + 2 * kv) * dim
        s["qkv"] = torch.randn(tokens, width + case["pad"], generator=g, device="cuda")[:, :width]
        s["turns"] = torch.from_numpy(_turns(case["rot"])).to("cuda")
        s["axis"] = torch.repeat_interleave(torch.arange(case["axes"], device="cuda"),
                                            torch.tensor(_sections(case), device="cuda"))
        if case["norm"]:                                   # trained gains
            s["gain"] = torch.exp(0.3 * torch.randn(2, dim, generator=g, device="cuda"))
        return s
    # Positions of the cached slots: ascending, with gaps where slots have been evicted.
    cols = s["table"].shape[1]
    slot = torch.arange(cols * page, device="cuda").reshape(cols, page)
    used = torch.arange(cols, device="cuda")[None] * page < lens[:, None]
    where = used.nonzero()
    s["position"][s["table"][used].long()] = (slot * 5 // 4)[where[:, 1]][:, None, :].expand(-1, kv, -1).to(torch.int32)
    s["q"] = 1.25 * torch.randn(case["seqs"], case["heads"], dim, generator=g, device="cuda")
    s["first"] = None
    if case["window"]:
        s["first"] = (lens * 5 // 4 - case["window"]).to(torch.int32)
        s["first"][5::16] = 1 << 30                        # every slot has left the window
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:                                                # the handles that a serving loop keeps
        from paper_2607_29221_gb300 import kvcache as KV
        s["cache"] = KV.PagedCache(s["k"], s["v"], s["table"], position=s.get("position"),
                                   weight=s.get("weight") if case.get("weights", True) else None)
        if "turns" in s:
            s["rope"] = KV.Rope(case["rot"], base=ROPE_BASE, sections=_sections(case),
                                interleaved=case["interleaved"], device="cuda")
            s["norm"] = KV.HeadNorm(case["dim"], EPS, s["gain"][0], s["gain"][1]) if case["norm"] else None
    torch.cuda.synchronize()
    return s


def run(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "attend":
        if own:
            out = s["cache"].attend(s["q"], s["lens"], case["max_len"], first=s["first"], scale=s["scale"],
                                    decay=case["decay"])
        else:
            out = _attend(s)
        return {"out": out, "weight": s["weight"]} if case["weights"] else {"out": out}
    if kind == "read":
        k, v = s["cache"].rows(s["seq"], s["slot"]) if own else _rows(s)
        return {"k": k, "v": v}
    if own:
        q = s["cache"].append(s["qkv"], case["heads"], s["seq"], s["slot"], s["index"], rope=s["rope"],
                              pos=s["pos"], norm=s["norm"])
    else:
        q = _append(s)
    out = {"q": q, "position": s["position"], "weight": s["weight"]}
    if kind == "norm":
        return {**out, "k": s["k"], "v": s["v"]}
    k, v = s["cache"].rows(s["seq"], s["slot"]) if own else _rows(s)
    return {**out, "k": k, "v": v}


# ---------------------------------------------------------------------------
# The plain forms.
def _pack(y):
    """Rows of channels (fp32) as codes, steps and bases: the bytes of a row but for its padding."""
    x = y.unflatten(-1, (-1, GROUP))
    fine = torch.isfinite(x).all(-1)
    x = x.clamp(-MOST, MOST)
    least, most = x.amin(-1), x.amax(-1)
    base = torch.where(fine, least, math.nan).half()
    step = torch.where(fine, (most - least) * (1.0 / 15.0), 0.0).half()
    inv = torch.where(step > 0, 1.0 / step.float(), 0.0)
    code = torch.round((x - base.float()[..., None]) * inv[..., None]).clamp(0, 15).nan_to_num(0.0)
    code = code.to(torch.uint8).flatten(-2)
    packed = code[..., 0::2] | code[..., 1::2] << 4
    scales = torch.stack([step, base], -1).flatten(-2).contiguous().view(torch.uint8)
    return torch.cat([packed, scales], -1)


def _values(rows, dim):
    """What packed rows stand for, in fp16 (base + code step is exact in fp32 unless a base is 512 steps away)."""
    packed = rows[..., : dim // 2]
    code = torch.stack([packed & 15, packed >> 4], -1).flatten(-2).unflatten(-1, (-1, GROUP)).float()
    scales = rows[..., dim // 2: dim // 2 + dim // 8].contiguous().view(torch.float16).float()
    return (code * scales[..., 0::2, None] + scales[..., 1::2, None]).half().flatten(-2)


def _rotate(x, c, sn, rot, interleaved):
    """x: tokens x heads x dim; c, sn: tokens x rot / 2."""
    c, sn = c[:, None, :], sn[:, None, :]
    y = x.clone()
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = a * c - b * sn, b * c + a * sn
    else:
        a, b = x[..., : rot // 2], x[..., rot // 2: rot]
        y[..., : rot // 2], y[..., rot // 2: rot] = a * c - b * sn, b * c + a * sn
    return y


def _append(s):
    case = s["case"]
    h, kv, d, page = case["heads"], case["kv"], case["dim"], case["page"]
    # The phase in 2^-64 turns, modulo one turn; then its signed upper half in radians.  Angles and the norm's sum
    # in 64 bits, rounded once: a key next to a border between two codes must not depend on them.
    phase = (s["pos"][s["axis"]].long() * s["turns"][:, None]) >> 32
    angle = phase.double().T * (2.0 * math.pi / 2.0 ** 32)
    c, sn = torch.cos(angle).float(), torch.sin(angle).float()
    x = s["qkv"].reshape(-1, h + 2 * kv, d)
    v = x[:, h + kv:]
    x = x[:, : h + kv]
    if case["norm"]:
        r = torch.rsqrt(x.double().square().mean(-1, keepdim=True) + EPS).float()
        x = x * r
        x = torch.cat([x[:, :h] * s["gain"][0], x[:, h:] * s["gain"][1]], 1)
    x = _rotate(x, c, sn, case["rot"], case["interleaved"])
    live = s["slot"] >= 0
    slot, seq = s["slot"][live].long(), s["seq"][live].long()
    at, off = s["table"][seq, slot // page].long(), slot % page
    for pool, y in ((s["k"], x[live][:, h:]), (s["v"], v[live])):
        if case["type"] == "q4":
            pool[..., : 5 * d // 8][at, :, off] = _pack(y)
        else:
            pool[at, :, off] = y.to(pool.dtype)
    s["position"][at, :, off] = s["index"][live][:, None].expand(-1, kv)
    s["weight"][at, :, off] = 0.0
    return x[:, :h]


def _rows(s):
    """The rows of the tokens (seq, slot) of a 4-bit cache, tokens x heads x dim; zeros without a slot."""
    page, dim = s["case"]["page"], s["case"]["dim"]
    live = s["slot"] >= 0
    slot = s["slot"].clamp(min=0).long()
    at = s["table"][s["seq"].long(), slot // page].long()
    return [torch.where(live[:, None, None], _values(pool[at, :, slot % page], dim), 0.0) for pool in (s["k"], s["v"])]


def _gather(s, pool):
    """Pages of a pool as seqs x kv heads x slots (x dim)."""
    x = pool[s["table"].long()].transpose(1, 2)
    return x.reshape(x.shape[0], x.shape[1], -1, *x.shape[4:])


def _attend(s):
    case = s["case"]
    b, kv, page, dim = case["seqs"], case["kv"], case["page"], case["dim"]
    n = s["table"].shape[1] * page
    inside = (torch.arange(n, device="cuda")[None] < s["lens"][:, None])[:, None].expand(b, kv, n)
    live = inside if s["first"] is None else inside & (_gather(s, s["position"]) >= s["first"][:, None, None])
    q = s["q"].reshape(b, kv, -1, dim)
    k = _values(_gather(s, s["k"]), dim).float()
    sc = torch.where(live[:, :, None], torch.matmul(q, k.transpose(2, 3)) * s["scale"], -math.inf)
    del k
    top = sc.amax(3, keepdim=True)
    e = torch.exp(sc - torch.where(top == -math.inf, 0.0, top))
    total = e.sum(3, keepdim=True)
    p = e / torch.where(total == 0.0, 1.0, total)
    v = torch.where(live[..., None], _values(_gather(s, s["v"]), dim), 0.0).float()
    out = torch.matmul(p, v).reshape(b, case["heads"], dim)
    if case["weights"]:
        seq, head, slot = inside.nonzero(as_tuple=True)
        at = s["table"][seq, slot // page].long()
        new = s["weight"][at, head, slot % page] * case["decay"] + p.sum(2)[seq, head, slot]
        s["weight"][at, head, slot % page] = new
    return out


# ---------------------------------------------------------------------------
def work(case):
    kv, dim = case["kv"], case["dim"]
    row = 5 * dim // 8 if case["type"] == "q4" else dim * (4 if case["type"] == "f32" else 2)
    if case["kind"] == "attend":
        slots = sum(_lengths(case))
        if case["window"]:                                 # positions advance by 5 in 4 slots
            slots = sum(min(n, -(-case["window"] * 4 // 5)) for n in _lengths(case))
        byts = slots * kv * (2 * row + (8 if case["weights"] else 0)) + 8 * case["seqs"] * case["heads"] * dim
        if case["window"]:
            byts += 4 * kv * sum(_lengths(case))
        return {"bytes": byts, "flops": 4 * slots * case["heads"] * dim}
    l = case["tokens"]
    read = l * kv * (2 * row + 4 * dim) + 8 * l            # packed rows in, fp16 out
    if case["kind"] == "read":
        return {"bytes": read, "flops": 4 * l * kv * dim}
    h = case["heads"]
    byts = 4 * l * (2 * h + 2 * kv) * dim + 2 * l * kv * row + 8 * l * kv + 4 * l * (3 + case["axes"])
    if case["kind"] == "append":
        byts += l * kv * 4 * dim                           # the values read back
    return {"bytes": byts, "flops": l * (h + kv) * (3 * case["rot"] + (4 * dim if case["norm"] else 0))}


# ---------------------------------------------------------------------------
def _meaning(rows, dim):
    """Packed rows in 64 bits, channel by channel pair of a byte."""
    byte = rows[..., : dim // 2].int()
    pair = rows[..., dim // 2: dim // 2 + dim // 8].contiguous().view(torch.float16).double().unflatten(-1, (-1, 2))
    out = torch.empty(*rows.shape[:-1], dim, dtype=torch.float64, device=rows.device)
    out[..., 0::2], out[..., 1::2] = (byte % 16).double(), (byte // 16).double()
    each = pair.repeat_interleave(GROUP, dim=-2)
    return (out * each[..., 0] + each[..., 1]).half().double()


def _nearest(y):
    """Channels in 64 bits to the values of the 4-bit format that they are packed as."""
    x = y.unflatten(-1, (-1, GROUP)).clamp(-MOST, MOST)
    base = x.min(-1, keepdim=True).values.half().double()
    step = ((x.max(-1, keepdim=True).values - x.min(-1, keepdim=True).values) / 15).half().double()
    code = torch.where(step > 0, ((x - base) / step).round(), 0.0).clamp(0, 15)
    return (base + code * step).half().double().flatten(-2)


def exact(case, seed):
    """The operators' definitions in 64 bits, attention a sequence at a time."""
    s = _inputs(case, seed)
    kv, page, dim = case["kv"], case["page"], case["dim"]
    if case["kind"] == "attend":
        out = torch.zeros(case["seqs"], case["heads"], dim, dtype=torch.float64, device="cuda")
        weight = s["weight"].double()
        for i, n in enumerate(s["lens"].tolist()):
            if not n:
                continue
            ids = s["table"][i, : -(-n // page)].long()
            k, v = (_meaning(s[x][ids].transpose(0, 1).reshape(kv, -1, _row(case))[:, :n], dim) for x in ("k", "v"))
            sc = torch.einsum("hgd,hnd->hgn", s["q"][i].double().reshape(kv, -1, dim), k) * s["scale"]
            if s["first"] is not None:
                gone = s["position"][ids].transpose(0, 1).reshape(kv, -1)[:, :n] < s["first"][i]
                sc = sc.masked_fill(gone[:, None], -math.inf)
            p = torch.softmax(sc, 2).nan_to_num(0.0)       # a row without a live slot gives zeros
            out[i] = torch.einsum("hgn,hnd->hgd", p, v).reshape(-1, dim)
            if case["weights"]:
                w = weight[ids].transpose(0, 1).reshape(kv, -1)
                w[:, :n] = w[:, :n] * case["decay"] + p.sum(1)
                weight[ids] = w.reshape(kv, -1, page).transpose(0, 1)
        return {"out": out, "weight": weight} if case["weights"] else {"out": out}
    t = (s["slot"] >= 0).nonzero()[:, 0]
    slot = s["slot"].long()[t]
    at = s["table"].long()[s["seq"][t].long(), slot // page]
    if case["kind"] == "read":
        return {x: _meaning(s[x][at, :, slot % page], dim) for x in ("k", "v")}
    h, rot = case["heads"], case["rot"]
    freq = ROPE_BASE ** (-2.0 * torch.arange(rot // 2, device="cuda", dtype=torch.float64) / rot)
    angle = s["pos"].double()[s["axis"]].T * freq
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]
    y = s["qkv"].double().reshape(-1, h + 2 * kv, dim).clone()
    if case["norm"]:
        root = torch.sqrt((y * y).sum(-1, keepdim=True) / dim + EPS)
        y[:, :h] *= s["gain"][0].double() / root[:, :h]
        y[:, h: h + kv] *= s["gain"][1].double() / root[:, h: h + kv]
    part = y[:, : h + kv, :rot]
    pairs = part.unflatten(2, (-1, 2)) if case["interleaved"] else part.unflatten(2, (2, -1)).transpose(2, 3)
    spun = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    y[:, : h + kv, :rot] = (spun if case["interleaved"] else spun.transpose(2, 3)).flatten(2)
    weight = s["weight"].double()
    weight[at, :, slot % page] = 0.0
    out = {"q": y[:, :h], "position": None, "weight": weight}
    if case["kind"] == "append":
        k, v = (torch.zeros(case["tokens"], kv, dim, dtype=torch.float64, device="cuda") for _ in range(2))
        k[t], v[t] = _nearest(y[t, h: h + kv]), _nearest(y[t, h + kv:])
        return {**out, "k": k, "v": v}
    k, v = s["k"].double(), s["v"].double()
    k[at, :, slot % page], v[at, :, slot % page] = y[t, h: h + kv], y[t, h + kv:]
    return {**out, "k": k, "v": v}

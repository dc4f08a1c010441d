"""The operators of a decode step's key/value cache, as measurable cases.

A case is one call of one operator, as a serving loop makes it between the
secure linears of a decoder layer:

  append  rotates the queries and keys of new tokens by their positions (one
          axis for text; time, height and width for video) and writes keys and
          values into the pages of a cache
  attend  attention of one new token per sequence over its pages, with the
          accumulated attention weight of every cached slot if it is kept
  evict   shortens the cached sequences to a budget of slots, by that weight

``own`` says who computes: the framework's kernels, or elementary torch
operations in 32 bits.  Head counts are those of the 70B layer (64 query and 8
key/value heads of 128) and of the 7B projections (32 heads of 128), and
generic ones.  Queries and keys are N(0, 1)-like with a few outlier channels;
accumulated weights are log-normal.  Pages of a sequence are scattered over
the pool.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ROPE_BASE = 500000.0


def listed():
    return [
        # The first tokens of a conversation: one short sequence, latency is all of it.
        {"name": "attend_70b_1x37", "kind": "attend", "seqs": 1, "max_len": 37, "lens": "full", "heads": 64, "kv": 8,
         "dim": 128, "page": 16, "type": "bf16", "weights": False, "window": 0, "layout": "head", "decay": 1.0},
        # One user with a very long document: a single sequence has to fill the GPU.
        {"name": "attend_70b_1x131071", "kind": "attend", "seqs": 1, "max_len": 131071, "lens": "full", "heads": 64,
         "kv": 8, "dim": 128, "page": 64, "type": "bf16", "weights": False, "window": 0, "layout": "head",
         "decay": 1.0},
        # A full serving batch of the 70B layer with lengths of every kind, weights kept for eviction.
        {"name": "attend_70b_64x16384", "kind": "attend", "seqs": 64, "max_len": 16384, "lens": "ragged", "heads": 64,
         "kv": 8, "dim": 128, "page": 16, "type": "bf16", "weights": True, "window": 0, "layout": "head",
         "decay": 1.0},
        # A 7B model's batch: every query head has a key/value head of its own.
        {"name": "attend_7b_48x2000", "kind": "attend", "seqs": 48, "max_len": 2000, "lens": "ragged", "heads": 32,
         "kv": 32, "dim": 128, "page": 32, "type": "f16", "weights": False, "window": 0, "layout": "head",
         "decay": 1.0},
        # The unrounded cache of the fp32 glue, weights decaying from step to step.
        {"name": "attend_f32_8x6001", "kind": "attend", "seqs": 8, "max_len": 6001, "lens": "full", "heads": 64,
         "kv": 8, "dim": 128, "page": 16, "type": "f32", "weights": True, "window": 0, "layout": "head",
         "decay": 0.96875},
        # Many short chats with a sliding window on a token-major cache; some sequences are empty.
        {"name": "attend_window_400x1500", "kind": "attend", "seqs": 400, "max_len": 1500, "lens": "zeros",
         "heads": 24, "kv": 8, "dim": 64, "page": 20, "type": "bf16", "weights": False, "window": 512,
         "layout": "token", "decay": 1.0},
        # A decode step of 32 sequences of the 70B layer.
        {"name": "append_70b_32", "kind": "append", "tokens": 32, "seqs": 32, "max_len": 2048, "heads": 64, "kv": 8,
         "dim": 128, "rot": 128, "axes": 1, "interleaved": False, "page": 16, "type": "bf16", "pad": 0,
         "layout": "head"},
        # Prefill of 2048 tokens of the 70B layer.
        {"name": "append_70b_2048", "kind": "append", "tokens": 2048, "seqs": 1, "max_len": 2048, "heads": 64, "kv": 8,
         "dim": 128, "rot": 128, "axes": 1, "interleaved": False, "page": 16, "type": "bf16", "pad": 0,
         "layout": "head"},
        # A clip's frames with positions in time, height and width, rows padded to a wider product.
        {"name": "append_video_9001", "kind": "append", "tokens": 9001, "seqs": 2, "max_len": 4501, "heads": 28,
         "kv": 4, "dim": 128, "rot": 128, "axes": 3, "interleaved": True, "page": 32, "type": "f16", "pad": 12,
         "layout": "token"},
        # A steady decode batch at its budget: each step's new slot pushes one old slot out.
        {"name": "evict_32_one_over", "kind": "evict", "seqs": 32, "max_len": 4097, "lens": "full", "keep": 4096,
         "recent": 256, "kv": 8, "dim": 128, "page": 16, "type": "bf16", "layout": "head"},
        # After a batch of long prompts: every sequence is cut to half the longest.
        {"name": "evict_16_half", "kind": "evict", "seqs": 16, "max_len": 16384, "lens": "ragged", "keep": 8192,
         "recent": 512, "kv": 8, "dim": 128, "page": 16, "type": "bf16", "layout": "head"},
        # One very long document cut to a quarter.
        {"name": "evict_1_long", "kind": "evict", "seqs": 1, "max_len": 131072, "lens": "full", "keep": 32768,
         "recent": 1024, "kv": 8, "dim": 128, "page": 64, "type": "bf16", "layout": "head"},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "append", "evict"])
    typ = rng.choice(["bf16", "bf16", "f16", "f32"])
    dim = rng.choice([128, 128, 128, 64, 80, 96, 256])
    kv = rng.choice([1, 2, 4, 8, 8, 32])
    group = rng.choice([1, 2, 3, 4, 7, 8, 8, 16]) if kv < 32 else rng.choice([1, 2])
    page = rng.choice([16, 16, 16, 32, 64, 8, 20, 1])
    layout = rng.choice(["head", "head", "token"])
    case = {"kind": kind, "kv": kv, "dim": dim, "page": page, "type": typ, "layout": layout}
    row = 2 * kv * dim * (4 if typ == "f32" else 2)              # cache bytes of one token
    if kind == "append":
        tokens = _log(rng, 1, 9000)
        axes = rng.choice([1, 1, 2, 3, 4])
        heads = min(64, kv * group)
        while tokens * (heads + 2 * kv) * dim > 9000 * 36 * 128:
            tokens //= 2
        seqs = min(tokens, _log(rng, 1, 64))
        return {**case, "tokens": tokens, "seqs": seqs, "max_len": -(-tokens // seqs) + rng.randint(0, 500),
                "heads": heads, "rot": dim if rng.random() < 0.75 else dim // 2, "axes": axes,
                "interleaved": rng.random() < 0.4, "pad": rng.choice([0, 0, 4, 37])}
    seqs, lens = _log(rng, 1, 400), rng.choice(["full", "ragged", "ragged", "zeros"])
    max_len = _log(rng, 1, 131072)
    share = {"full": 1.0, "ragged": 0.5, "zeros": 0.44}[lens]
    while max_len * max(1.0, seqs * share) * row > (2.0e9 if kind == "attend" else 0.5e9):
        max_len = -(-max_len // 2)
        seqs = max(1, seqs // 2) if max_len < 64 else seqs
    case.update(seqs=seqs, max_len=max_len, lens=lens)
    if kind == "evict":
        keep = max(1, rng.choice([max_len - 1, max_len // 2, max_len // 4, int(max_len * rng.random())]))
        return {**case, "keep": keep, "recent": rng.choice([0, min(64, keep), keep // 8])}
    return {**case, "heads": kv * group, "weights": rng.random() < 0.5,
            "window": rng.choice([0, 0, 0, _log(rng, 1, 4096)]), "decay": rng.choice([1.0, 0.9375])}


# ---------------------------------------------------------------------------
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


def _pool(case, pages, g):
    shape = ((pages, case["kv"], case["page"], case["dim"]) if case["layout"] == "head"
             else (pages, case["page"], case["kv"], case["dim"]))
    x = torch.randn(shape, generator=g, device="cuda", dtype=TYPES[case["type"]])
    return x if case["layout"] == "head" else x.transpose(1, 2)


def _outliers(case, x, g):
    at = torch.randperm(case["dim"], generator=g, device="cuda")[:2]
    x[..., at] *= 4.0


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
    kind, page, kv = case["kind"], case["page"], case["kv"]
    if kind == "append":
        tokens, seqs = case["tokens"], case["seqs"]
        per = [tokens // seqs + (i < tokens % seqs) for i in range(seqs)]
        start = [(37 * i + 11) % (case["max_len"] - per[i] + 1) for i in range(seqs)]
        lens = [a + b for a, b in zip(start, per)]
        s["table"], pages = _table(case, lens, g)
        s["seq"] = torch.repeat_interleave(torch.arange(seqs, device="cuda"),
                                           torch.tensor(per, device="cuda")).to(torch.int32)
        first = torch.tensor(np.cumsum([0] + per[:-1]), device="cuda")
        nth = torch.arange(tokens, device="cuda") - first[s["seq"].long()]
        s["slot"] = (nth + torch.tensor(start, device="cuda")[s["seq"].long()]).to(torch.int32)
        s["index"] = s["slot"] + 1000                      # 1000 earlier tokens have been evicted
        if tokens > 16:
            s["slot"][-1] = -1                             # a padding row of a static batch
        # Text: one running position; video: frames of 16 x 9 patches after the text before them.
        at = s["index"]
        axes = [at, 1000 + nth % 144 // 9, 1000 + nth % 9, at // 2]
        if case["axes"] > 1:
            axes[0] = 1000 + nth // 144
        s["pos"] = torch.stack([a.to(torch.int32) for a in axes[: case["axes"]]]).contiguous()
        width = (case["heads"] + 2 * kv) * case["dim"]
        s["qkv"] = torch.randn(tokens, width + case["pad"], generator=g, device="cuda")[:, :width]
        s["turns"] = torch.from_numpy(_turns(case["rot"])).to("cuda")
        s["axis"] = torch.repeat_interleave(torch.arange(case["axes"], device="cuda"),
                                            torch.tensor(_sections(case), device="cuda"))
    else:
        lens = torch.tensor(_lengths(case), device="cuda")[torch.randperm(case["seqs"], generator=g, device="cuda")]
        s["lens"] = lens.to(torch.int32)
        s["table"], pages = _table(case, lens.tolist(), g)
    s["k"], s["v"] = _pool(case, pages, g), _pool(case, pages, g)
    shape = (pages, kv, page)
    s["weight"] = torch.randn(shape, generator=g, device="cuda").mul_(2.0).exp_()
    if kind == "append":
        s["position"] = torch.zeros(shape, dtype=torch.int32, device="cuda")
        return s
    # Positions of the cached slots: ascending, with gaps where slots have been evicted.
    cols = s["table"].shape[1]
    slot = torch.arange(cols * page, device="cuda").reshape(cols, page)
    s["position"] = torch.zeros(shape, dtype=torch.int32, device="cuda")
    used = torch.arange(cols, device="cuda")[None] * page < lens[:, None]
    where = used.nonzero()
    s["position"][s["table"][used].long()] = (slot * 5 // 4)[where[:, 1]][:, None, :].expand(-1, kv, -1).to(torch.int32)
    if kind == "attend":
        _outliers(case, s["k"], g)
        s["q"] = 1.25 * torch.randn(case["seqs"], case["heads"], case["dim"], generator=g, device="cuda")
        s["first"] = None
        if case["window"]:
            s["first"] = (lens * 5 // 4 - case["window"]).to(torch.int32)
            s["first"][5::16] = 1 << 30                    # every slot has left the window
    else:
        s["recent_from"] = ((lens - case["recent"]) * 5 // 4).to(torch.int32) if case["recent"] else None
        s["new_lens"] = torch.zeros_like(s["lens"])
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:                                                # the handles that a serving loop keeps
        from paper_2607_29221_gb300 import kvcache as KV
        s["cache"] = KV.PagedCache(s["k"], s["v"], s["table"], position=s["position"],
                                   weight=s["weight"] if _keeps_weight(case) else None)
        if case["kind"] == "append":
            s["rope"] = KV.Rope(case["rot"], base=ROPE_BASE, sections=_sections(case),
                                interleaved=case["interleaved"], device="cuda")
    torch.cuda.synchronize()
    return s


def _keeps_weight(case):
    return case["kind"] != "attend" or case["weights"]


def run(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "append":
        if own:
            q = s["cache"].append(s["qkv"], case["heads"], s["seq"], s["slot"], s["index"], rope=s["rope"],
                                  pos=s["pos"])
        else:
            q = _append(s)
        return {"q": q, "k": s["k"], "v": s["v"], "position": s["position"], "weight": s["weight"]}
    if kind == "attend":
        if own:
            out = s["cache"].attend(s["q"], s["lens"], case["max_len"], first=s["first"], scale=s["scale"],
                                    decay=case["decay"])
        else:
            out = _attend(s)
        return {"out": out, "weight": s["weight"]} if case["weights"] else {"out": out}
    if own:
        s["cache"].evict(s["lens"], case["max_len"], case["keep"], recent_from=s["recent_from"],
                         new_lens=s["new_lens"])
    else:
        _evict(s)
    return {"new_lens": s["new_lens"], "k": s["k"], "v": s["v"], "position": s["position"], "weight": s["weight"]}


# ---------------------------------------------------------------------------
# The plain forms.
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
    # The phase in 2^-64 turns, modulo one turn; then its signed upper half in radians.
    phase = (s["pos"][s["axis"]].long() * s["turns"][:, None]) >> 32
    angle = phase.float().T * (2.0 * math.pi / 2.0 ** 32)
    c, sn = torch.cos(angle), torch.sin(angle)
    x = s["qkv"].reshape(-1, h + 2 * kv, d)
    q = _rotate(x[:, :h], c, sn, case["rot"], case["interleaved"])
    k = _rotate(x[:, h: h + kv], c, sn, case["rot"], case["interleaved"])
    live = s["slot"] >= 0
    slot, seq = s["slot"][live].long(), s["seq"][live].long()
    at, off = s["table"][seq, slot // page].long(), slot % page
    s["k"][at, :, off] = k[live].to(s["k"].dtype)
    s["v"][at, :, off] = x[live][:, h + kv:].to(s["v"].dtype)
    s["position"][at, :, off] = s["index"][live][:, None].expand(-1, kv)
    s["weight"][at, :, off] = 0.0
    return q


def _gather(s, pool):
    """Pages of a pool as seqs x kv heads x slots (x dim)."""
    x = pool[s["table"].long()].transpose(1, 2)
    return x.reshape(x.shape[0], x.shape[1], -1, *x.shape[4:])


def _attend(s):
    case = s["case"]
    b, kv, page = case["seqs"], case["kv"], case["page"]
    k, v = _gather(s, s["k"]).float(), _gather(s, s["v"]).float()
    n = k.shape[2]
    inside = (torch.arange(n, device="cuda")[None] < s["lens"][:, None])[:, None].expand(b, kv, n)
    live = inside if s["first"] is None else inside & (_gather(s, s["position"]) >= s["first"][:, None, None])
    q = s["q"].reshape(b, kv, -1, case["dim"])
    sc = torch.where(live[:, :, None], torch.matmul(q, k.transpose(2, 3)) * s["scale"], -math.inf)
    top = sc.amax(3, keepdim=True)
    e = torch.exp(sc - torch.where(top == -math.inf, 0.0, top))
    total = e.sum(3, keepdim=True)
    p = e / torch.where(total == 0.0, 1.0, total)
    out = torch.matmul(p, torch.where(live[..., None], v, 0.0)).reshape(b, case["heads"], case["dim"])
    if case["weights"]:
        seq, head, slot = inside.nonzero(as_tuple=True)
        at = s["table"][seq, slot // page].long()
        new = s["weight"][at, head, slot % page] * case["decay"] + p.sum(2)[seq, head, slot]
        s["weight"][at, head, slot % page] = new
    return out


def _evict(s):
    case = s["case"]
    kv, page, keep = case["kv"], case["page"], case["keep"]
    key = _gather(s, s["weight"])
    key = torch.where(key.isnan(), -math.inf, key)
    if s["recent_from"] is not None:
        key = torch.where(_gather(s, s["position"]) >= s["recent_from"][:, None, None], math.inf, key)
    slot = torch.arange(key.shape[2], device="cuda")
    inside = (slot[None] < s["lens"][:, None])[:, None]
    order = torch.sort(torch.where(inside, key, math.inf), dim=2, stable=True).indices
    rank = torch.empty_like(order).scatter_(2, order, slot.expand_as(order).contiguous())
    out = rank < (s["lens"].long() - keep)[:, None, None]
    hole = out & (slot < keep)
    moved = inside & ~out & (slot >= keep)
    (b0, h0, to), (b1, h1, frm) = hole.nonzero(as_tuple=True), moved.nonzero(as_tuple=True)
    dst = (s["table"][b0, to // page].long(), h0, to % page)
    src = (s["table"][b1, frm // page].long(), h1, frm % page)
    for pool in (s["k"], s["v"], s["position"], s["weight"]):
        pool[dst] = pool[src]
    s["new_lens"].copy_(s["lens"].clamp(max=keep))


# ---------------------------------------------------------------------------
def _moves(case):
    """Rows that an eviction moves and slots that it ranks, per key/value head (expected values)."""
    moves = slots = 0.0
    for n in _lengths(case):
        if n <= case["keep"]:
            continue
        slots += n
        recent = min(case["recent"], n)
        safe = min(recent, n - case["keep"])
        moves += safe + (n - case["keep"] - safe) * max(0.0, case["keep"] - recent) / max(1, n - recent)
    return moves, slots


def work(case):
    kv, dim = case["kv"], case["dim"]
    es = 4 if case["type"] == "f32" else 2
    if case["kind"] == "append":
        l, h = case["tokens"], case["heads"]
        return {"bytes": 4 * l * (2 * h + 2 * kv) * dim + 2 * es * l * kv * dim + 8 * l * kv + 4 * l * (3 + case["axes"]),
                "flops": 3 * l * (h + kv) * case["rot"]}
    if case["kind"] == "attend":
        slots = sum(_lengths(case))
        if case["window"]:                                 # positions advance by 5 in 4 slots
            slots = sum(min(n, -(-case["window"] * 4 // 5)) for n in _lengths(case))
        byts = slots * kv * (2 * dim * es + (8 if case["weights"] else 0)) + 8 * case["seqs"] * case["heads"] * dim
        if case["window"]:
            byts += 4 * kv * sum(_lengths(case))
        return {"bytes": byts, "flops": 4 * slots * case["heads"] * dim}
    moves, slots = _moves(case)
    return {"bytes": kv * (slots * (8 if case["recent"] else 4) + moves * (4 * dim * es + 16)) + 8 * case["seqs"],
            "flops": kv * slots}


# ---------------------------------------------------------------------------
def exact(case, seed):
    """The operators' definitions in 64 bits, a sequence at a time."""
    s = _inputs(case, seed)
    kv, page, dim = case["kv"], case["page"], case["dim"]
    if case["kind"] == "append":
        h, rot = case["heads"], case["rot"]
        freq = ROPE_BASE ** (-2.0 * torch.arange(rot // 2, device="cuda", dtype=torch.float64) / rot)
        angle = s["pos"].double()[s["axis"]].T * freq
        turn = torch.polar(torch.ones_like(angle), angle)[:, None]
        x = s["qkv"].double().reshape(-1, h + 2 * kv, dim)
        y = x.clone()
        part = x[:, : h + kv, :rot]
        pairs = part.unflatten(2, (-1, 2)) if case["interleaved"] else part.unflatten(2, (2, -1)).transpose(2, 3)
        spun = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        y[:, : h + kv, :rot] = (spun if case["interleaved"] else spun.transpose(2, 3)).flatten(2)
        k, v = s["k"].double(), s["v"].double()
        weight = s["weight"].double()
        slot = s["slot"].long()
        t = (slot >= 0).nonzero()[:, 0]
        at = s["table"].long()[s["seq"][t].long(), slot[t] // page]
        k[at, :, slot[t] % page], v[at, :, slot[t] % page] = y[t, h: h + kv], y[t, h + kv:]
        weight[at, :, slot[t] % page] = 0.0
        return {"q": y[:, :h], "k": k, "v": v, "position": None, "weight": weight}
    lens = s["lens"].tolist()
    if case["kind"] == "attend":
        out = torch.zeros(case["seqs"], case["heads"], dim, dtype=torch.float64, device="cuda")
        weight = s["weight"].double()
        for i, n in enumerate(lens):
            if not n:
                continue
            ids = s["table"][i, : -(-n // page)].long()
            k, v = (s[x][ids].transpose(0, 1).reshape(kv, -1, dim)[:, :n].double() for x in ("k", "v"))
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
    k, v, w, at = s["k"].double(), s["v"].double(), s["weight"].double(), s["position"].double()
    for i, n in enumerate(lens):
        gone = n - case["keep"]
        if gone <= 0:
            continue
        ids = s["table"][i, : -(-n // page)].long()
        for h in range(kv):
            rank = w[ids, h].reshape(-1)[:n].clone()
            if s["recent_from"] is not None:
                rank[at[ids, h].reshape(-1)[:n] >= s["recent_from"][i]] = math.inf
            left = torch.zeros(n, dtype=torch.bool, device="cuda")
            left[torch.argsort(rank, stable=True)[:gone]] = True
            to = left[: case["keep"]].nonzero()[:, 0]
            frm = case["keep"] + (~left[case["keep"]:]).nonzero()[:, 0]
            for x in (k, v, w, at):
                x[ids[to // page], h, to % page] = x[ids[frm // page], h, frm % page]
    return {"new_lens": None, "k": k, "v": v, "position": None, "weight": w}

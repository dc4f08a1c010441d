"""Cached decoding through a masked decoder layer: prefill and steps against
full causal passes whose attention (with rotary positions) is written here in
64 bits, and the budget of slots.

At sigma = 0 a secure linear is exact up to its quantisation, which depends on
the token's own row only.  The two passes differ by the fp32 of the attention,
and where that moves a value across a rounding edge, by one code of 2 q_max:
the update's difference stays below the quantisation error that a pass has by
itself, 2.5 / q_max (a rotated row's absmax is about 4 standard deviations:
1.15 / q_max a rounded operand)."""
import numpy as np
import pytest

from paper_2607_29221_gb300 import workloads as wl

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

SHAPE = dict(hidden=256, n_heads=8, n_kv=2, head_dim=32, ffn=384)
BASE = 500000.0


@pytest.fixture(scope="module")
def layer():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2607_29221_gb300 import build
    build.build()
    from paper_2607_29221_gb300 import decoder as D
    from paper_2607_29221_gb300 import mosaic as M
    from paper_2607_29221_gb300 import protocol as PR
    proto = PR.Protocol(wl.mask_key(), M.default_params(sigma=0.0), variant=M.GEMM_AUTO)
    return D.SecureDecoderLayer(proto, D.LayerWeights(D.LayerShape(**SHAPE), seed=51))


def rotary_attention(qkv):
    """Causal grouped-query attention with rotated queries and keys, fp64 numpy."""
    H, KV, d = SHAPE["n_heads"], SHAPE["n_kv"], SHAPE["head_dim"]
    x = qkv.double().cpu().numpy()
    l = x.shape[0]
    ang = np.arange(l)[:, None] * BASE ** (-2.0 * np.arange(d // 2) / d)
    c, s = np.cos(ang), np.sin(ang)

    def rot(v):
        a, b = v[:, : d // 2], v[:, d // 2:]
        return np.concatenate([a * c - b * s, b * c + a * s], 1)

    out = np.zeros((l, H * d))
    future = np.triu(np.ones((l, l), dtype=bool), 1)
    for h in range(H):
        g = h // (H // KV)
        q, k = rot(x[:, h * d:(h + 1) * d]), rot(x[:, (H + g) * d:(H + g + 1) * d])
        sc = q @ k.T / np.sqrt(d)
        sc[future] = -np.inf
        p = np.exp(sc - sc.max(1, keepdims=True))
        out[:, h * d:(h + 1) * d] = (p / p.sum(1, keepdims=True)) @ x[:, (H + KV + g) * d:(H + KV + g + 1) * d]
    return torch.from_numpy(out).float().cuda()


def test_prefill_and_steps_match_full_passes(layer):
    from paper_2607_29221_gb300 import mosaic as M
    from paper_2607_29221_gb300 import protocol as PR
    from paper_2607_29221_gb300.session import DecodeSession
    prompt, steps = [40, 17, 1], 6
    xs = [torch.from_numpy(wl.activations(n + steps, SHAPE["hidden"], seed=60 + i)).cuda() for i, n in enumerate(prompt)]
    ses = DecodeSession(layer, 3, 64, page_size=16, dtype=torch.float32)
    got = [[ses.prefill(i, xs[i][:n])] for i, n in enumerate(prompt)]
    for t in range(steps):
        y = ses.step(torch.stack([xs[i][n + t] for i, n in enumerate(prompt)]))
        for i in range(3):
            got[i].append(y[i:i + 1])
    M.mosaic_device_status()
    qmin = min(M.mosaic_qmax(PR.pad_width(n)) for n in (SHAPE["hidden"], SHAPE["ffn"]))
    for i, n in enumerate(prompt):
        want = layer.forward(xs[i], attend=rotary_attention) - xs[i]
        diff = torch.cat(got[i]) - xs[i] - want
        assert torch.isfinite(diff).all()
        assert float(diff.norm() / want.norm()) < 2.5 / qmin
    assert ses.host_lens == [n + steps for n in prompt] == ses.lens.tolist() == ses.seen.tolist()


def test_a_budget_of_slots_is_kept(layer):
    from paper_2607_29221_gb300.session import DecodeSession
    keep, recent, slack = 24, 6, 3
    ses = DecodeSession(layer, 2, 64, page_size=8, keep=keep, recent=recent, slack=slack)
    x = torch.from_numpy(wl.activations(90, SHAPE["hidden"], seed=70)).cuda()
    ses.prefill(0, x[:50])
    assert len(ses.pages.owned[0]) == 7
    for t in range(30):
        y = ses.step(x[t:t + 2])
        assert torch.isfinite(y).all()
        assert max(ses.host_lens) <= keep + slack and ses.host_lens == ses.lens.tolist()
        for i in range(2):
            assert len(ses.pages.owned[i]) == -(-ses.host_lens[i] // 8)
    assert ses.seen.tolist() == [80, 30]
    assert len(ses.pages.owned[0]) <= 4        # pages of the prompt came back
    assert len(ses.pages.free) + sum(map(len, ses.pages.owned)) == 16
    for i in range(2):
        n, page = ses.host_lens[i], 8
        ids = ses.pages.table[i, : -(-n // page)].long()
        pos = ses.cache.position[ids].transpose(0, 1).reshape(SHAPE["n_kv"], -1)[:, :n].cpu().numpy()
        last = int(ses.seen[i])
        for h in range(SHAPE["n_kv"]):
            assert len(set(pos[h])) == n                                   # no slot twice
            assert set(range(last - recent, last)) <= set(pos[h])          # the newest are there


def test_refusals(layer):
    from paper_2607_29221_gb300 import kvcache as KV
    from paper_2607_29221_gb300.session import DecodeSession
    with pytest.raises(ValueError):
        DecodeSession(layer, 1, 64, keep=4, recent=5)
    with pytest.raises(ValueError):
        DecodeSession(layer, 1, 64, rope=KV.Rope(32, sections=[8, 8]))
    ses = DecodeSession(layer, 1, 8, page_size=4)
    x = torch.from_numpy(wl.activations(9, SHAPE["hidden"], seed=71)).cuda()
    with pytest.raises(ValueError):
        ses.prefill(0, x)
    ses.prefill(0, x[:8])
    with pytest.raises(ValueError):
        ses.prefill(0, x[:1])
    with pytest.raises(ValueError):
        ses.step(x[:1])


def test_a_budget_is_cut_back_at_max_len(layer):
    """A slack that reaches past max_len does not end the session there."""
    from paper_2607_29221_gb300.session import DecodeSession
    ses = DecodeSession(layer, 1, 16, page_size=8, keep=12, recent=3, slack=10)
    x = torch.from_numpy(wl.activations(40, SHAPE["hidden"], seed=72)).cuda()
    ses.prefill(0, x[:5])
    held = []
    for t in range(30):
        assert torch.isfinite(ses.step(x[5 + t:6 + t])).all()
        held.append(ses.host_lens[0])
    assert max(held) == 15 and held[-1] == int(ses.lens) and int(ses.seen) == 35
    full = DecodeSession(layer, 1, 8, page_size=4, keep=8)      # a budget of max_len: nothing can leave
    full.prefill(0, x[:8])
    with pytest.raises(ValueError):
        full.step(x[:1])


def test_attention_after_evictions(layer, monkeypatch):
    """Every step of a session over its budget: each cached row is the one that was appended at its position, and
    the outputs are the 64-bit attention over those rows.  Tolerance: scores to 2^-20 of their terms, probabilities
    to twice that and 2^-19, as for the operator alone."""
    from paper_2607_29221_gb300.session import DecodeSession
    keep, page, H, KV, d = 20, 8, SHAPE["n_heads"], SHAPE["n_kv"], SHAPE["head_dim"]
    ses = DecodeSession(layer, 2, 64, page_size=page, keep=keep, recent=5, slack=2)
    cache, made, attend, worst = ses.cache, {}, ses.cache.attend, []

    def rows(pool, i, n):
        ids = cache.table[i, : -(-n // page)].long()
        return pool[ids].transpose(0, 1).flatten(1, 2)[:, :n]

    def note(i, n):                      # rows appended since the last step
        k, v, at = (rows(x, i, n).cpu() for x in (cache.k, cache.v, cache.position))
        for h in range(KV):
            for s in range(n):
                row = k[h, s], v[h, s]
                old = made.setdefault((i, h, int(at[h, s])), row)
                assert torch.equal(old[0], row[0]) and torch.equal(old[1], row[1])

    def checked(q, lens, most):
        out = attend(q, lens, most)
        for i, n in enumerate(lens.tolist()):
            note(i, n)
            k, v = rows(cache.k, i, n).double(), rows(cache.v, i, n).double()
            x = q[i].double().reshape(KV, -1, d)
            p = torch.softmax(x @ k.transpose(1, 2) * d ** -0.5, 2)
            rel = 2.0 ** -19 * (1 + (x.abs() @ k.abs().transpose(1, 2) * d ** -0.5).amax(2, keepdim=True))
            err = (out[i].double().reshape(KV, -1, d) - p @ v).abs()
            assert (err <= rel * (p @ v.abs())).all()
        worst.append(max(lens.tolist()))
        return out
    monkeypatch.setattr(cache, "attend", checked)
    x = torch.from_numpy(wl.activations(100, SHAPE["hidden"], seed=75)).cuda()
    ses.prefill(0, x[:17])
    for t in range(25):
        ses.step(x[20 + 2 * t: 22 + 2 * t])
    assert max(worst) == keep + 3 and ses.host_lens[0] >= keep

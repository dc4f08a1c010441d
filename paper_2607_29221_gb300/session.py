"""Cached decoding through a masked decoder layer.

``DecodeSession`` runs the key/value cache's operators together as a serving
loop does: the four linears of a layer are outsourced as in
``decoder.SecureDecoderLayer``, and the trusted side keeps the cache
(``kvcache``).  A prompt is prefilled in one pass, then every step takes one
token of each sequence: append with rotary positions, attention over the
pages, and, past a budget of slots, eviction by gathered attention weight.

Prompts are for empty sequences, and a step takes all sequences together.
Weights are gathered by steps only: a prompt longer than the budget is cut by
the weights of the first step after it.

  session = DecodeSession(layer, seqs=4, max_len=4096, keep=1024, recent=128)
  session.prefill(0, x0)              # tokens x hidden of sequence 0
  y = session.step(x)                 # seqs x hidden: one token each
"""
from __future__ import annotations

import torch
import torch.nn.functional as F

from . import kvcache as KV
from .decoder import SecureDecoderLayer


class DecodeSession:
    """``keep``: slots a sequence may hold (None: no eviction); it may run over
    by ``slack`` slots (up to max_len) before it is cut back, without the
    ``recent`` newest tokens.  ``rope``: its positions are the tokens' ordinals (one axis);
    default: the usual rotation of the whole head at base 500000.  ``norm``: norms of
    the query and key heads.  ``dtype``: the cache's (``kvcache.INT4``: 4 bits)."""

    def __init__(self, layer: SecureDecoderLayer, seqs: int, max_len: int, page_size: int = 16,
                 dtype=torch.bfloat16, rope: KV.Rope | None = None, keep: int | None = None, recent: int = 0,
                 slack: int = 0, norm: KV.HeadNorm | None = None):
        s, dev = layer.s, torch.device(layer.proto.device)
        if keep is not None and not (0 <= recent <= keep and slack >= 0 and keep >= 1):
            raise ValueError("keep, recent and slack: 1 <= keep, 0 <= recent <= keep, 0 <= slack")
        if rope is not None and rope.axes != 1:
            raise ValueError("rope: one axis (a session's positions are the tokens' ordinals)")
        self.layer, self.seqs, self.max_len = layer, seqs, max_len
        self.keep, self.recent, self.slack = keep, recent, slack
        columns = -(-max_len // page_size)
        self.pages = KV.PageTable(seqs, columns, seqs * columns + 1, page_size, device=dev)
        self.cache = KV.PagedCache.empty(seqs * columns + 1, s.n_kv, page_size, s.head_dim, self.pages.table, dtype,
                                         weights=keep is not None)
        self.rope = KV.Rope(s.head_dim, 500000.0, device=dev) if rope is None else rope
        if norm is not None:
            norm.on(s.head_dim, self.cache.k.get_device())      # refused before a prompt takes pages
        self.norm = norm
        self.host_lens = [0] * seqs
        self.lens = torch.zeros(seqs, dtype=torch.int32, device=dev)     # cached slots
        self.seen = torch.zeros(seqs, dtype=torch.int32, device=dev)     # tokens so far
        self._rows = torch.arange(seqs, dtype=torch.int32, device=dev)

    def prefill(self, seq: int, x: torch.Tensor, masks=None) -> torch.Tensor:
        """The prompt of an empty sequence (x: tokens x hidden fp32), causal."""
        l, s = x.shape[0], self.layer.s
        if self.host_lens[seq] or not 0 < l <= self.max_len:
            raise ValueError(f"prefill: an empty sequence and 1 to {self.max_len} tokens")
        self.pages.resize(seq, l)
        at = torch.arange(l, dtype=torch.int32, device=x.device)

        def attend(qkv):
            q = self.cache.append(qkv, s.n_heads, torch.full_like(at, seq), at, at, rope=self.rope, pos=at,
                                  norm=self.norm)
            k, v = (t.float().repeat_interleave(s.n_heads // s.n_kv, dim=0) for t in self.cache.read(seq, l))
            out = F.scaled_dot_product_attention(q.transpose(0, 1)[None], k[None], v[None], is_causal=True)
            return out[0].transpose(0, 1).reshape(l, -1)

        y = self.layer.forward(x, masks, attend=attend)
        self.host_lens[seq] = l
        self.lens[seq] = l
        self.seen[seq] = l
        return y

    def step(self, x: torch.Tensor, masks=None) -> torch.Tensor:
        """One token of every sequence (x: seqs x hidden fp32)."""
        s = self.layer.s
        if max(self.host_lens) >= self.max_len:
            raise ValueError("step: a sequence is at max_len")
        for i, n in enumerate(self.host_lens):
            self.pages.resize(i, n + 1)
        after = max(self.host_lens) + 1

        def attend(qkv):
            q = self.cache.append(qkv, s.n_heads, self._rows, self.lens, self.seen, rope=self.rope, pos=self.seen,
                                  norm=self.norm)
            return self.cache.attend(q, self.lens + 1, after).reshape(self.seqs, -1)

        y = self.layer.forward(x, masks, attend=attend)
        self.lens += 1
        self.seen += 1
        self.host_lens = [n + 1 for n in self.host_lens]
        # No further step would fit at max_len.
        if self.keep is not None and after > min(self.keep + self.slack, self.max_len - 1):
            self.cache.evict(self.lens, after, self.keep, recent_from=self.seen - self.recent, new_lens=self.lens)
            self.host_lens = [min(n, self.keep) for n in self.host_lens]
            for i, n in enumerate(self.host_lens):
                self.pages.resize(i, n)
        return y

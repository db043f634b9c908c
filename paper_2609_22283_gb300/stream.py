"""One attention layer over a video that outgrows its cache.

Chunks come one after the other under clean history (every node reads level-0
states of earlier chunks).  The last `window` clean states are kept whole; when
one more is written, the oldest ones are condensed: head by head, the tokens that
got the most attention so far stay, in one state of a chunk's size, which every
later node reads in their place.  The cache so holds window + 3 states however
long the video is.

One update of a chunk (a denoising level, or the clean refresh at level 0):
  1. sva_rope_kv_write_headnorm: per-head RMSNorm of the new queries and keys, 3D
     RoPE, K' and V into the chunk's own slot;
  2. sva_attend_nodes over the condensed state, the window and the own chunk, with
     its log-sum-exps;
  3. sva_attend_weights: adds what every key got to its running weight;
and after a clean refresh that fills the window, sva_cache_condense.  All on one
stream: a released slot is written again only by later calls.
"""
from __future__ import annotations

import torch

from . import sva

CONDENSED = 1 << 20  # the level under which a condensed state is bound


class Stream:
    def __init__(self, H, d, F, Hp, Wp, pairs, max_frames, window=6, recent=3, decay=1.0, theta=10000.0,
                 device="cuda"):
        """window: clean states kept whole, up to MAX_CTX - 2; recent: how many of them stay whole when the
        older ones are condensed (1..window); decay: of the weights from update to update, 0..1."""
        if not 1 <= recent <= window or window + 2 > sva.MAX_CTX:
            raise ValueError(f"need 1 <= recent <= window <= {sva.MAX_CTX - 2}")
        g = sva.make_geometry(H, d, F, Hp, Wp, num_slots=window + 3, pairs=pairs, max_frames=max_frames,
                              theta=theta)
        self.cache = sva.Cache(g, device=device)
        self.device = self.cache.buf.device
        self.cache.set_workspace(torch.empty(self.cache.workspace_bytes(), dtype=torch.uint8, device=self.device))
        c = self.cache
        self.window, self.recent, self.decay = window, recent, decay
        self.weight = torch.zeros((g.num_slots, c.H, c.T), device=self.device)
        self.lse = torch.empty((1, c.H, c.T), device=self.device)
        self.index = torch.empty((c.H, c.T), dtype=torch.int32, device=self.device)
        self.clean = []        # (chunk, slot) of the clean states kept whole, oldest first
        self.condensed = None  # (chunk of its newest source, slot)

    def context(self):
        """The slots that the next update reads, oldest first."""
        return ([self.condensed[1]] if self.condensed else []) + [s for _, s in self.clean]

    def update(self, chunk, level, q, k, v, out, gamma_k=None, gamma_q=None, eps=1e-6):
        """One update of a chunk: q, k, v [1][T][H][d] (dense or parts of a packed projection), out
        [1][T][H][d] receives the attention.  Level 0 is the clean refresh, after which the chunk belongs to
        the history; other levels leave nothing behind but their share of the weights.  An update that
        raises leaves no state behind, so that it can be made again."""
        c = self.cache
        slot = c.bind(0, chunk, level)
        try:
            node = sva.make_nodes([dict(seq=0, chunk=chunk, level=level, own_slot=slot, ctx=self.context())])
            rotated = torch.empty_like(out)
            c.rope_kv_write_headnorm(node, k, v, q, rotated, gamma_k, gamma_q, eps)
            c.attend_nodes(node, rotated, out, self.lse)
            self.weight[slot].zero_()  # what the slot's last tenant left
            c.attend_weights(node, rotated, self.lse, self.weight, prev=self.weight, decay=self.decay)
        except BaseException:
            c.release(0, chunk, level)
            raise
        if level != 0:
            c.release(0, chunk, level)
            return
        self.clean.append((chunk, slot))
        if len(self.clean) > self.window:
            self._condense()

    def _condense(self):
        c = self.cache
        old, self.clean = self.clean[:-self.recent], self.clean[-self.recent:]
        newest = old[-1][0]
        dst = c.bind(0, newest, CONDENSED)
        c.condense(([self.condensed[1]] if self.condensed else []) + [s for _, s in old], dst, self.weight, self.index)
        if self.condensed:
            c.release(0, self.condensed[0], CONDENSED)
        for chunk, _ in old:
            c.release(0, chunk, 0)
        self.condensed = (newest, dst)

    def close(self):
        self.cache.close()

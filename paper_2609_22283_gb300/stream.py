"""One attention layer over a video that outgrows its cache, in two ways: Stream condenses old states,
PackedStream holds them in 4 bits.

Stream.  Chunks come one after the other under clean history (every node reads level-0
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


class PackedStream:
    """A layer that keeps a longer window: of its clean states the newest `recent` are whole, the others are held in 4
    bits, and the oldest one goes when a new one comes.  A video may branch: from fork() on, two sequences go on from
    the same history, each with updates of its own.

    One update of a chunk: sva_rope_kv_write_headnorm into the chunk's own slot, sva_attend_nodes_packed over the
    sequence's history and the own chunk, and after a clean refresh (level 0) sva_cache_pack of the state that leaves
    the newest ones.  fork() is sva_cache_copy of whole and of packed states."""

    def __init__(self, H, d, F, Hp, Wp, pairs, max_frames, window=12, recent=2, sequences=1, theta=10000.0, device="cuda"):
        """window: clean states that an update reads, up to MAX_CTX; recent: how many of them stay whole (0..window);
        sequences: how many there may be at once."""
        if not 0 <= recent <= window <= sva.MAX_CTX or window < 1 or sequences < 1:
            raise ValueError(f"need 0 <= recent <= window, 1 <= window <= {sva.MAX_CTX} and sequences >= 1")
        g = sva.make_geometry(H, d, F, Hp, Wp, num_slots=sequences * recent + 1, pairs=pairs, max_frames=max_frames,
                              theta=theta)
        self.cache = sva.Cache(g, device=device)
        c, self.device = self.cache, self.cache.buf.device
        c.set_workspace(torch.empty(c.workspace_bytes(), dtype=torch.uint8, device=self.device))
        if window > recent:
            n = sequences * (window - recent) + 1  # one to pack into before the oldest is let go
            c.set_packed(torch.empty(sva.packed_bytes(g, n), dtype=torch.uint8, device=self.device), n)
        self.window, self.recent, self.sequences = window, recent, sequences
        self.whole = {0: []}   # sequence -> [(chunk, slot)], oldest first
        self.packed = {0: []}  # and the packed ones before them

    def context(self, seq=0):
        """The slots that the next update of the sequence reads, oldest first."""
        return [s for _, s in self.packed[seq] + self.whole[seq]]

    def update(self, chunk, level, q, k, v, out, gamma_k=None, gamma_q=None, eps=1e-6, seq=0):
        """One update of a chunk, arguments as Stream.update.  One that raises leaves the sequence's history as it was
        and no state behind, so that it can be made again."""
        c, context = self.cache, self.context(seq)
        slot = c.bind(seq, chunk, level)
        try:
            node = sva.make_nodes([dict(seq=seq, chunk=chunk, level=level, own_slot=slot, ctx=context)])
            rotated = torch.empty_like(out)
            c.rope_kv_write_headnorm(node, k, v, q, rotated, gamma_k, gamma_q, eps)
            c.attend_nodes_packed(node, rotated, out)
            if level == 0:
                self._keep(seq, chunk, slot)
        except BaseException:
            c.release(seq, chunk, level)
            raise
        if level != 0:
            c.release(seq, chunk, level)

    def _keep(self, seq, chunk, slot):
        """The state joins the newest ones, and the oldest of these is packed if they are too many.  What may raise
        comes before the lists change: the new packed slot is one to spare, the window's oldest is still held."""
        c, whole, packed = self.cache, self.whole[seq], self.packed[seq]
        if len(whole) < self.recent:
            whole.append((chunk, slot))
            return
        old, at = (whole + [(chunk, slot)])[0]
        if self.window > self.recent:
            to = c.bind_packed(seq, old, 0)
            try:
                c.pack([at], [to])
            except BaseException:
                c.release_packed(seq, old, 0)
                raise
            packed.append((old, to))
            if len(packed) > self.window - self.recent:
                c.release_packed(seq, packed.pop(0)[0], 0)
        whole.append((chunk, slot))
        del whole[0]
        c.release(seq, old, 0)

    def fork(self, seq, new):
        """A new sequence `new` with the history of `seq`."""
        if seq not in self.whole or new in self.whole:
            raise ValueError(f"sequence {seq} must exist and {new} must not")
        if len(self.whole) == self.sequences:
            raise ValueError(f"there are {self.sequences} sequences already")
        c, done = self.cache, []
        try:
            for old, bind, release in ((self.whole[seq], c.bind, c.release),
                                       (self.packed[seq], c.bind_packed, c.release_packed)):
                copies = []
                for chunk, _ in old:
                    copies.append((chunk, bind(new, chunk, 0)))
                    done.append((release, chunk))
                if copies:
                    c.copy([s for _, s in old], [s for _, s in copies])
                (self.whole if old is self.whole[seq] else self.packed)[new] = copies
        except BaseException:
            for release, chunk in done:
                release(new, chunk, 0)
            self.whole.pop(new, None)
            self.packed.pop(new, None)
            raise

    def drop(self, seq):
        """Lets a sequence and its states go."""
        for chunk, _ in self.whole.pop(seq):
            self.cache.release(seq, chunk, 0)
        for chunk, _ in self.packed.pop(seq):
            self.cache.release_packed(seq, chunk, 0)

    def close(self):
        self.cache.close()

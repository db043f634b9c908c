"""Attention received per key (sva_attend_weights) against its formula in 64 bits.

Tolerance.  Every term exp(x) is positive, so an error of each term relative to
itself is one of the sum.  In the exponent (scale * s - lse), s is a sum of d
products in fp32, |ds| <= d 2^-24 sum |q||k|, and scale, lse and their log2(e)
multiples add four roundings of 2^-24 on values up to scale * sum |q||k| and
|lse|; ex2 is good to 2^-22, the sums over a Q tile's 128 queries and over the
tiles add one rounding a level: (tiles + 16) 2^-24.  So
  rel = 2^-24 ((d + 4) scale max(sum |q||k|) + 4 max|lse| + tiles + 16) + 2^-21,
and decay * prev adds two roundings.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def _pairs(d):
    return (d // 2 - 2 * (d // 6), d // 6, d // 6)


def _pack(keep):
    n = keep.shape[-1]
    words = -(-n // 32)
    k = torch.zeros(keep.shape[:-1] + (words * 32,), dtype=torch.bool, device=keep.device)
    k[..., :n] = keep
    v = (k.view(keep.shape[:-1] + (words, 32)).long() << torch.arange(32, device=keep.device)).sum(-1)
    return torch.where(v >= 2 ** 31, v - 2 ** 32, v).to(torch.int32)


class Case:
    """A cache with `states` written, nodes over them, their queries and the attention's log-sum-exps."""

    def __init__(self, sva, F, Hp, Wp, H, d, node_ctx, causal=False, hidden=(), spread=1.0, seed=1, spare=1):
        """node_ctx: per node ((seq, chunk, level), [context states]); hidden: (node, context index) pairs."""
        self.sva, self.T, self.H, self.d = sva, F * Hp * Wp, H, d
        self.frame = Hp * Wp
        self.causal, self.hidden, self.node_ctx = causal, set(hidden), node_ctx
        self.states = []
        for st, ctx in node_ctx:
            for s in [st] + ctx:
                if s not in self.states:
                    self.states.append(s)
        top = max(b for _, b, _ in self.states)
        self.cache = sva.Cache(sva.make_geometry(H, d, F, Hp, Wp, len(self.states) + spare, _pairs(d), F * (top + 2)))
        self.cache.set_workspace(torch.empty(self.cache.workspace_bytes(), dtype=torch.uint8, device="cuda"))
        g = torch.Generator(device="cuda").manual_seed(seed)
        T, n = self.T, len(node_ctx)
        self.slot = {s: self.cache.bind(*s) for s in self.states}
        for s, b in self.slot.items():
            k = torch.randn((1, T, H, d), generator=g, device="cuda") * spread
            self.cache.rope_kv_write([dict(seq=s[0], chunk=s[1], level=s[2], own_slot=b)], k.bfloat16(), k.bfloat16())
        self.q = torch.randn((n, T, H, d), generator=g, device="cuda").bfloat16()
        self.nodes = sva.make_nodes([
            dict(seq=st[0], chunk=st[1], level=st[2], own_slot=self.slot[st], ctx=[self.slot[c] for c in ctx],
                 visible=[0 if (i, j) in self.hidden else 1 for j in range(len(ctx))],
                 within=sva.WITHIN_FRAME_CAUSAL if causal else sva.WITHIN_BIDIRECTIONAL)
            for i, (st, ctx) in enumerate(node_ctx)])
        self.lse = torch.empty((n, H, T), device="cuda")
        self.shape = (len(self.states) + spare, H, T)
        self.g = g

    def attend(self, tile=None, own=None, hist=None):
        out = torch.empty_like(self.q)
        if tile is None and own is None and hist is None:
            self.cache.attend_nodes(self.nodes, self.q, out, self.lse)
        else:
            self.cache.attend_nodes_masked(self.nodes, self.q, out, self.lse, tile_mask=tile, own_mask=own, hist_mask=hist)
        return out

    def ref(self, prev=None, decay=1.0, tile=None, own=None, hist=None):
        """(sums, bound on the error, slots seen); masks as booleans."""
        T, d, scale = self.T, self.d, 1 / math.sqrt(self.d)
        w = torch.zeros(self.shape, dtype=torch.float64, device="cuda")
        seen, size, refs = set(), 0.0, 0
        nt = -(-T // 128)
        u = torch.arange(T, device="cuda")
        for i, (st, ctx) in enumerate(self.node_ctx):
            for j, s in enumerate([st] + ctx):
                if j and (i, j - 1) in self.hidden:
                    continue
                seen.add(self.slot[s])
                refs += 1
                keep = torch.ones((T, T), dtype=torch.bool, device="cuda")
                if j == 0 and self.causal:
                    keep &= (u[:, None] // self.frame) >= (u[None, :] // self.frame)
                if tile is not None:
                    t = tile[i, :, j * nt:(j + 1) * nt]
                    keep &= t.repeat_interleave(128, 0)[:T].repeat_interleave(128, 1)[:, :T]
                if j == 0 and own is not None:
                    keep &= own[i]
                if j and hist is not None:
                    keep &= hist[i, :, j - 1]
                k = self.cache.slot_pool()[self.slot[s], 0, :, :T]
                for h in range(self.H):
                    q = self.q[i, :, h].double()
                    x = (q @ k[h].double().t()) * scale - self.lse[i, h].double()[:, None]
                    x.masked_fill_(~keep | (self.lse[i, h] == -math.inf)[:, None], -math.inf)
                    w[self.slot[s], h] += torch.exp(x).sum(0)
                    ok = torch.isfinite(k[h].double()).all(-1)
                    size = max(size, float((q.abs() @ k[h][ok].double().abs().t()).max()) * scale) if ok.any() else size
        lse = self.lse[torch.isfinite(self.lse)]
        top = float(lse.abs().max()) if lse.numel() else 0.0
        rel = 2.0 ** -24 * ((d + 4) * size + 4 * top + refs * nt + 16) + 2.0 ** -21
        bound = w * rel
        if prev is not None:
            w = w + decay * prev.double()
            bound = bound + 2.0 ** -23 * w.abs()
        return w, bound, seen

    def check(self, prev=None, decay=1.0, tile=None, own=None, hist=None, lse=True):
        masks = dict(tile_mask=None if tile is None else _pack(tile), own_mask=None if own is None else _pack(own),
                     hist_mask=None if hist is None else _pack(hist))
        if lse:
            self.attend(masks["tile_mask"], masks["own_mask"], masks["hist_mask"])
        out = torch.full(self.shape, -7.0, device="cuda")
        self.cache.attend_weights(self.nodes, self.q, self.lse, out, prev=prev, decay=decay, **masks)
        assert self.cache.poll() == self.sva.OK
        want, bound, seen = self.ref(prev, decay, tile, own, hist)
        for s in range(self.shape[0]):
            if s not in seen:
                assert torch.all(out[s] == -7.0), f"slot {s} is not seen and was written"
                continue
            err = (out[s].double() - want[s]).abs()
            assert torch.all(err <= bound[s]), (f"slot {s}: off by up to {float(err.max()):.3e} "
                                                f"(bound there {float(bound[s][err == err.max()][0]):.3e})")
        return out

    def close(self):
        self.cache.close()


def _chain(n_nodes, W, seq=0, top=None):
    """Nodes (chunk b, level i) with the W chunks before them as clean context."""
    top = top or W + n_nodes
    return [((seq, top - i, 4), [(seq, top - i - r, 0) for r in range(1, min(W, top - i - 1) + 1)]) for i in range(n_nodes)]


@pytest.mark.parametrize("F,Hp,Wp,H,d,n,W", [
    (1, 1, 1, 1, 64, 1, 0),       # one token, one key
    (1, 1, 1, 3, 128, 2, 2),
    (1, 6, 7, 2, 64, 2, 1),       # 42 tokens: part of one tile
    (1, 8, 16, 1, 128, 1, 3),     # exactly one tile
    (3, 1, 43, 2, 64, 1, 2),      # 129: one key past a tile
    (1, 16, 16, 2, 128, 3, 2),    # exactly a pair of tiles
    (1, 7, 43, 3, 128, 2, 3),     # 301: three tiles, the last ragged
    (2, 13, 17, 16, 64, 2, 4),    # 442 tokens: more units than SMs
    (1, 20, 33, 12, 128, 4, 6),   # 660 tokens, uneven numbers of readers, several units a CTA
    (3, 23, 31, 1, 128, 1, 1),    # 2139 tokens of one head: a cluster shares a unit's queries
    (3, 23, 31, 1, 64, 2, 0),
])
def test_dense(sva_mod, F, Hp, Wp, H, d, n, W):
    c = Case(sva_mod, F, Hp, Wp, H, d, _chain(n, W))
    out = c.check()
    # every query's weights sum to one
    seen = sorted(c.slot[s] for s in c.states)
    total = out[seen].double().sum(dim=(0, 2))
    assert torch.allclose(total, torch.full_like(total, float(n * c.T)), rtol=1e-3)
    prev = torch.rand(c.shape, generator=c.g, device="cuda") * 3
    c.check(prev=prev, decay=0.5, lse=False)
    c.close()


def test_in_place_streams_and_repeats(sva_mod):
    c = Case(sva_mod, 1, 20, 33, 12, 128, _chain(4, 6))
    c.attend()
    first = torch.zeros(c.shape, device="cuda")
    c.cache.attend_weights(c.nodes, c.q, c.lse, first)
    again = torch.full(c.shape, 5.0, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c.cache.attend_weights(c.nodes, c.q, c.lse, again, stream=side)
    side.synchronize()
    seen = sorted(c.slot[s] for s in c.states)
    assert torch.equal(first[seen], again[seen])          # the same bits, whatever order the CTAs ran in
    acc = first.clone()
    for _ in range(2):                                     # accumulated in place
        c.cache.attend_weights(c.nodes, c.q, c.lse, acc, prev=acc, decay=1.0)
    assert torch.allclose(acc[seen], 3 * first[seen], rtol=1e-6)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        c.cache.attend_weights(c.nodes, c.q, c.lse, again)
    again.fill_(0)
    g.replay()
    assert torch.equal(first[seen], again[seen])
    c.close()


def test_nodes_and_contexts_to_the_limit(sva_mod):
    """64 nodes of one chunk over the same 16 states, and hidden contexts."""
    ctx = [(0, 16 - r, 0) for r in range(16)]
    nodes = [((0, 17, j), ctx) for j in range(64)]
    c = Case(sva_mod, 1, 5, 9, 1, 64, nodes, hidden={(0, 3), (7, 0), (63, 15)})
    c.check()
    c.close()


def test_two_streams_of_video_and_in_round_states(sva_mod):
    nodes = []
    for seq in (0, 5):
        nodes += [((seq, 4, 2), [(seq, 3, 1), (seq, 2, 0)]), ((seq, 3, 1), [(seq, 2, 0), (seq, 1, 0)])]
    c = Case(sva_mod, 1, 11, 13, 3, 64, nodes)
    c.check()
    c.close()


@pytest.mark.parametrize("F,Hp,Wp,H,d,n,W", [(3, 4, 8, 2, 64, 2, 1), (4, 5, 19, 3, 128, 1, 2), (5, 1, 100, 1, 64, 2, 0),
                                             (7, 20, 20, 1, 128, 1, 0)])
def test_frame_causal(sva_mod, F, Hp, Wp, H, d, n, W):
    c = Case(sva_mod, F, Hp, Wp, H, d, _chain(n, W), causal=True)
    c.check()
    c.close()


@pytest.mark.parametrize("d,causal,kinds", [(64, False, ("tile",)), (128, True, ("tile",)), (64, False, ("own",)),
                                            (128, False, ("hist",)), (128, True, ("own", "hist")),
                                            (64, True, ("tile", "own", "hist"))])
def test_masks(sva_mod, d, causal, kinds):
    """T = 330 (three tiles, 74 rows in the last): tiles and tokens at random, queries and keys with nothing."""
    c = Case(sva_mod, 3, 10, 11, 3, d, _chain(2, 2), causal=causal)
    T, n, nt = c.T, 2, 3
    tile = own = hist = None
    if "tile" in kinds:
        tile = torch.rand((n, nt, 3 * nt), generator=c.g, device="cuda") < 0.5
        tile[0, 1] = False                 # a query tile that sees nothing
        tile[1, :, 4] = False              # a key tile that nothing sees
    if "own" in kinds:
        own = torch.rand((n, T, T), generator=c.g, device="cuda") < 0.4
        own[:, 7], own[1, :, 9] = False, False
        own[0, :, 128:256] = True
    if "hist" in kinds:
        hist = torch.rand((n, T, 2, T), generator=c.g, device="cuda") < 0.4
        hist[:, 7], hist[0, 200:], hist[1, :, 1, 64:300] = False, False, False
    out = c.check(tile=tile, own=own, hist=hist)
    assert torch.all(out[out != -7.0] >= 0)
    prev = torch.rand(c.shape, generator=c.g, device="cuda")
    c.check(prev=prev, decay=1.0, tile=tile, own=own, hist=hist, lse=False)
    c.close()


def test_all_ones_masks_are_the_dense_launch(sva_mod):
    c = Case(sva_mod, 1, 10, 33, 2, 128, _chain(2, 2))
    dense = c.check()
    T = c.T
    ones = c.check(tile=torch.ones((2, 3, 9), dtype=torch.bool, device="cuda"),
                   own=torch.ones((2, T, T), dtype=torch.bool, device="cuda"),
                   hist=torch.ones((2, T, 2, T), dtype=torch.bool, device="cuda"), lse=False)
    assert torch.equal(dense, ones)
    c.close()


def test_masked_cluster_split(sva_mod):
    """Few units over many queries: the masked form shared by a cluster, with ranks that have nothing to do."""
    c = Case(sva_mod, 1, 40, 50, 1, 64, _chain(1, 0))
    T = c.T
    own = (torch.arange(T, device="cuda")[:, None] - torch.arange(T, device="cuda")[None, :]).abs() < 40
    tile = torch.zeros((1, 16, 16), dtype=torch.bool, device="cuda")
    tile[0, :9] = True
    c.check(own=own[None], tile=tile)
    c.close()


@pytest.mark.parametrize("d,causal,tokens", [(128, False, False), (64, True, False), (64, False, True), (128, True, True)])
def test_more_masked_units_than_sms(sva_mod, d, causal, tokens):
    """600 units that differ in work, some with none at all: each is summed once, whichever CTA takes it."""
    c = Case(sva_mod, 4, 5, 55, 20, d, _chain(2, 3), causal=causal)
    T, n, nt = c.T, 2, 9
    tile = torch.rand((n, nt, 4 * nt), generator=c.g, device="cuda") < torch.linspace(0.05, 1.0, 4 * nt, device="cuda")
    tile[:, :, 2:4] = False                 # the second pair of the own chunk's key tiles
    tile[:, :, nt:2 * nt] = False           # the first history state of either node
    own = hist = None
    if tokens:
        own = torch.rand((n, T, T), generator=c.g, device="cuda") < 0.5
        hist = torch.rand((n, T, 3, T), generator=c.g, device="cuda") < 0.5
        hist[:, 100:700, 1] = False
    first = c.check(tile=tile, own=own, hist=hist)
    masks = dict(tile_mask=_pack(tile), own_mask=_pack(own) if tokens else None, hist_mask=_pack(hist) if tokens else None)
    for _ in range(20):
        again = torch.full(c.shape, -7.0, device="cuda")
        c.cache.attend_weights(c.nodes, c.q, c.lse, again, **masks)
        assert torch.equal(again, first)
    assert c.cache.poll() == sva_mod.OK
    c.close()


def test_masked_units_in_a_graph(sva_mod):
    """A captured masked launch with more units than SMs gives the direct call's bits at every replay."""
    c = Case(sva_mod, 2, 14, 20, 24, 64, _chain(1, 3), causal=True)
    tile = torch.rand((1, 5, 20), generator=c.g, device="cuda") < 0.6
    direct = c.check(tile=tile)
    packed = _pack(tile)
    out = torch.full(c.shape, -7.0, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.cache.attend_weights(c.nodes, c.q, c.lse, out, tile_mask=packed)
    for _ in range(5):
        out.fill_(-7.0)
        graph.replay()
        assert torch.equal(out, direct)
    assert c.cache.poll() == sva_mod.OK
    c.close()


def test_hidden_keys_may_hold_anything(sva_mod):
    """NaN and infinities in keys that no query sees: zero for them, and the others as without."""
    c = Case(sva_mod, 1, 10, 33, 2, 128, _chain(1, 1))
    T = c.T
    hist = torch.ones((1, T, 1, T), dtype=torch.bool, device="cuda")
    gone = [0, 5, 127, 128, 329]
    hist[..., gone] = False
    k = c.cache.slot_pool()[c.slot[c.states[1]], 0]
    k[:, gone] = torch.tensor([math.nan, math.inf, -math.inf, math.nan, math.inf], device="cuda").bfloat16()[None, :, None]
    # log-sum-exps over what is visible, in 64 bits
    parts = []
    for j, s in enumerate(c.states):
        kk = c.cache.slot_pool()[c.slot[s], 0, :, :T].double()
        x = torch.einsum("uhd,hvd->huv", c.q[0].double(), kk) / math.sqrt(c.d)
        if j:
            x[..., gone] = -math.inf
        parts.append(x)
    c.lse.copy_(torch.logsumexp(torch.cat(parts, -1), -1)[None])
    out = c.check(hist=hist, lse=False)
    assert torch.all(out[c.slot[c.states[1]]][:, gone] == 0)
    c.close()


def test_queries_that_saw_nothing_add_nothing(sva_mod):
    """lse = -inf without any mask, and log-sum-exps far from the scores' (weights that vanish or are large)."""
    c = Case(sva_mod, 1, 6, 30, 2, 64, _chain(1, 1), spread=3.0)
    c.attend()
    c.lse[0, :, ::3] = -math.inf
    c.lse[0, :, 1::3] += 200.0
    c.lse[0, :, 2::3] -= 20.0
    c.check(lse=False)
    c.close()


def test_scanned_token_masks(sva_mod):
    """A launch long enough for the scan of its token masks: the same bits with it and without (no workspace)."""
    c = Case(sva_mod, 1, 39, 50, 12, 64, _chain(2, 3))      # 1950 tokens, 16 tiles
    T, n = c.T, 2
    u = torch.arange(T, device="cuda")
    own = ((u[:, None] - u[None, :]).abs() < 200)[None].expand(n, T, T).clone()
    hist = own[:, :, None].expand(n, T, 3, T).clone()
    hist[:, 128:256] = False               # a query tile without history
    hist[:, :, 1, :300] = False
    own[:, 7::97] = False
    hist[:, 7::97] = False                 # queries that see nothing
    words = dict(own_mask=_pack(own), hist_mask=_pack(hist))
    c.attend(own=words["own_mask"], hist=words["hist_mask"])
    out = torch.zeros(c.shape, device="cuda")
    c.cache.attend_weights(c.nodes, c.q, c.lse, out, **words)
    c.cache.set_workspace(None)
    plain = torch.zeros(c.shape, device="cuda")
    c.cache.attend_weights(c.nodes, c.q, c.lse, plain, **words)
    assert c.cache.poll() == sva_mod.OK
    assert torch.equal(out, plain)
    want, bound, seen = c.ref(own=own, hist=hist)
    for s in seen:
        assert torch.all((out[s].double() - want[s]).abs() <= bound[s])
    c.close()


def test_long_chunk_sums(sva_mod):
    """16384 queries into every key's sum, one head, both at a few keys checked in 64 bits."""
    c = Case(sva_mod, 1, 128, 128, 1, 64, _chain(1, 0), spare=0)
    c.attend()
    out = torch.empty(c.shape, device="cuda")
    c.cache.attend_weights(c.nodes, c.q, c.lse, out)
    at = torch.tensor([0, 1, 127, 128, 8191, 16000, 16383], device="cuda")
    k = c.cache.slot_pool()[0, 0, 0][at].double()
    q = c.q[0, :, 0].double()
    want = torch.exp((q @ k.t()) / 8.0 - c.lse[0, 0].double()[:, None]).sum(0)
    size = float((q.abs() @ k.abs().t()).max()) / 8.0
    rel = 2.0 ** -24 * (68 * size + 4 * float(c.lse.abs().max()) + 128 + 16) + 2.0 ** -21
    assert torch.all((out[0, 0][at].double() - want).abs() <= rel * want)
    assert abs(float(out.double().sum()) / 16384 - 1) < 1e-3
    c.close()


def test_timeout_is_reported_and_writes_nothing(sva_mod):
    """A withheld Q tile: the bounded waits end, the status says so, no unit is written; the next launch is whole."""
    for H, W, hw in ((12, 6, (20, 33)), (1, 0, (40, 50))):      # units in turn; a cluster a unit
        c = Case(sva_mod, 1, hw[0], hw[1], H, 64, _chain(1, W))
        good = c.check()
        out = torch.full(c.shape, -7.0, device="cuda")
        c.cache.debug_inject(2, 0.2)
        c.cache.attend_weights(c.nodes, c.q, c.lse, out)
        assert c.cache.poll() == sva_mod.ERR_DEVICE_TIMEOUT
        assert torch.all(out == -7.0)
        c.cache.debug_inject(0, 1.0)
        c.cache.attend_weights(c.nodes, c.q, c.lse, out)
        assert c.cache.poll() == sva_mod.OK
        assert torch.equal(out, good)
        c.close()


def test_refusals(sva_mod):
    sva = sva_mod
    c = Case(sva, 1, 6, 7, 2, 64, _chain(2, 1))
    c.attend()
    out = torch.full(c.shape, -7.0, device="cuda")

    def status(nodes=None, **kw):
        with pytest.raises(sva.SvaError) as e:
            c.cache.attend_weights(c.nodes if nodes is None else nodes, c.q, c.lse, kw.pop("out", out), **kw)
        return e.value.status

    def rejected(**kw):
        a = dict(q=c.q, lse=c.lse, out=out)
        a.update(kw)
        with pytest.raises(ValueError):
            c.cache.attend_weights(c.nodes, **a)

    assert status(decay=-0.1) == sva.ERR_INVALID_ARGUMENT
    assert status(decay=1.5) == sva.ERR_INVALID_ARGUMENT
    assert status(decay=math.nan) == sva.ERR_INVALID_ARGUMENT
    assert status(scale=0.0) == sva.ERR_INVALID_ARGUMENT
    assert status(scale=math.inf) == sva.ERR_INVALID_ARGUMENT
    (s0, x0), (s1, x1) = c.node_ctx
    e0 = dict(seq=0, chunk=s0[1], level=4, own_slot=c.slot[s0], ctx=[c.slot[x0[0]]])
    e1 = dict(seq=0, chunk=s1[1], level=4, own_slot=c.slot[s1], ctx=[c.slot[x1[0]]])
    assert status([dict(e0, ctx=[c.slot[s0]]), e1]) == sva.ERR_CAUSALITY
    assert status([dict(e0, ctx=e0["ctx"] * 2), e1]) == sva.ERR_INVALID_ARGUMENT
    assert status([dict(e0, own_slot=e1["own_slot"]), e1]) == sva.ERR_INVALID_ARGUMENT
    blank = c.cache.bind(0, 1 + max(b for _, b, _ in c.states), 0)
    assert status([dict(seq=0, chunk=1 + max(b for _, b, _ in c.states), level=0, own_slot=blank), e1]) == sva.ERR_NOT_RESIDENT
    words = torch.zeros((2, c.T, 1), dtype=torch.int32, device="cuda")
    assert status(own_mask=words) == sva.ERR_INVALID_ARGUMENT          # 42 tokens need two words
    rejected(q=c.q.float())
    rejected(q=c.q[:1])
    rejected(lse=c.lse.double())
    rejected(out=out[:1])
    rejected(out=out.transpose(1, 2).contiguous().transpose(1, 2))
    rejected(prev=out[:, :1])
    torch.cuda.synchronize()
    assert torch.all(out == -7.0)
    c.close()

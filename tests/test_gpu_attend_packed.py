"""Attention over packed slots (sva_attend_nodes_packed): against the formula in 64 bits over the values that the 4
bits stand for, and bit for bit the attention over the same states read back."""
import pytest
import torch

from paper_2609_22283_gb300.inputs import pack_bits
from tests._packed import assert_attention, attention, held, make_cache, random_kv, status, write

pytestmark = pytest.mark.gpu
NONE = torch.empty(0, dtype=torch.uint8, device="cuda") if torch.cuda.is_available() else None


class Layer:
    """A cache, one sequence: `kinds` says of each history state, oldest first, whether it is packed ("p") or whole
    ("w"); `nodes` of the newest chunks, each reading every state before it (the nodes' own ones included)."""

    def __init__(self, sva, F, Hp, Wp, H, d, kinds, nodes=1, causal=False, workspace=True, seed=0, hidden=()):
        W = len(kinds)
        self.kinds = kinds
        self.F, self.hw, self.T, self.H, self.d, self.n, self.W, self.causal = F, Hp * Wp, F * Hp * Wp, H, d, nodes, W, causal
        self.sva = sva
        c = self.c = make_cache(sva, F, Hp, Wp, H, d, 2 * W + nodes, max(kinds.count("p"), 1), workspace)
        g = self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.kv, ctx, back = [], [], []       # values by state; slots for the packed attention; read back
        for i, kind in enumerate(kinds):
            x = random_kv(c, g)
            s = write(c, (0, 1 + i, 0), x)
            if kind == "p":
                p = c.bind_packed(0, 1 + i, 0)
                c.pack([s], [p])
                c.release(0, 1 + i, 0)
                b = c.bind(0, 1 + i, 1)
                c.unpack([p], [b])
                ctx.append(p)
                back.append(b)
                x = held(x)
            else:
                ctx.append(s)
                back.append(s)
            self.kv.append(x)
        own = []
        for i in range(nodes):
            x = random_kv(c, g)
            own.append(write(c, (0, W + 1 + i, 0), x))
            self.kv.append(x)
        within = sva.WITHIN_FRAME_CAUSAL if causal else sva.WITHIN_BIDIRECTIONAL
        self.see, lists = [], ([], [])
        for i in range(nodes):
            states = list(range(W + i - 1, -1, -1))[:16]          # newest first
            vis = [0 if k in hidden else 1 for k in range(len(states))]
            self.see.append([W + i] + [k for k, v in zip(states, vis) if v])
            for out, slots in zip(lists, (ctx + own, back + own)):
                out.append(dict(seq=0, chunk=W + 1 + i, level=0, own_slot=own[i], within=within,
                                ctx=[slots[k] for k in states], visible=vis))
        self.states = [list(range(W + i - 1, -1, -1))[:16] for i in range(nodes)]
        self.nodes, self.nodes_back = sva.make_nodes(lists[0]), sva.make_nodes(lists[1])
        self.q = torch.randn((nodes, self.T, H, d), generator=g, device="cuda").bfloat16()

    def buffers(self):
        return (torch.full_like(self.q, float("nan")),
                torch.full((self.n, self.H, self.T), float("nan"), device="cuda"))

    def space(self, extra=0):
        """Rubbish, as much as all packed states need (extra: bytes more or less)."""
        c = self.c
        n = sum(kind == "p" for kind in self.kinds) * 2 * c.H * c.Tpad * c.d * 2 + extra
        return torch.randint(0, 256, (n,), dtype=torch.uint8, device="cuda")

    def run(self, **masks):
        out, lse = self.buffers()
        self.c.attend_nodes_packed(self.nodes, self.q, out, lse, **masks)
        assert self.c.poll() == self.sva.OK
        return out, lse

    def run_back(self, **masks):
        out, lse = self.buffers()
        self.c.attend_nodes_masked(self.nodes_back, self.q, out, lse, **masks)
        return out, lse

    def keep(self, i, tile=None, own=None, hist=None):
        """[T][keys] of node i over self.see[i]; tile [n][nt][(1 + ctx) nt], own [n][T][T], hist [n][T][ctx][T] bools."""
        T, nt = self.T, -(-self.T // 128)
        cols = []
        for k in self.see[i]:
            j = 0 if k == self.W + i else 1 + self.states[i].index(k)
            m = torch.ones((T, T), dtype=torch.bool, device="cuda")
            if tile is not None:
                m &= tile[i, :, j * nt:(j + 1) * nt].repeat_interleave(128, 0)[:T].repeat_interleave(128, 1)[:, :T]
            if j == 0 and own is not None:
                m &= own[i]
            if j and hist is not None:
                m &= hist[i, :, j - 1]
            if j == 0 and self.causal:
                f = torch.arange(T, device="cuda") // self.hw
                m &= f[:, None] >= f[None, :]
            cols.append(m)
        return torch.cat(cols, 1)

    def check(self, out, lse, heads=None, **bools):
        for i in range(self.n):
            keep = self.keep(i, **bools) if bools or self.causal else None
            for h in (range(self.H) if heads is None else heads):
                k, v = (torch.cat([self.kv[s][x, h].double() for s in self.see[i]]) for x in (0, 1))
                assert_attention(out[i, :, h], lse[i, h], attention(self.q[i, :, h], k, v, keep), f"node {i} head {h}")

    def close(self):
        self.c.close()


CASES = [
    # one token, one packed state; sixteen of them
    dict(F=1, Hp=1, Wp=1, H=1, d=64, kinds="p"),
    dict(F=1, Hp=1, Wp=1, H=3, d=128, kinds="p" * 16),
    # short of, at and past a tile; one and two query tiles
    dict(F=1, Hp=1, Wp=127, H=2, d=128, kinds="pp"),
    dict(F=1, Hp=8, Wp=16, H=2, d=64, kinds="pwp"),
    dict(F=1, Hp=3, Wp=43, H=2, d=128, kinds="wp"),
    dict(F=1, Hp=16, Wp=20, H=5, d=128, kinds="ppwppwpppppwpppp"),
    dict(F=1, Hp=16, Wp=20, H=4, d=64, kinds="ppwppwppp", nodes=3),
    # no workspace: no splits
    dict(F=1, Hp=16, Wp=20, H=2, d=128, kinds="pppp", workspace=False),
    dict(F=1, Hp=16, Wp=20, H=2, d=64, kinds="pppp", workspace=False),
    # frame-causal; states hidden by their node
    dict(F=3, Hp=9, Wp=17, H=3, d=128, kinds="pwpp", nodes=2, causal=True),
    dict(F=3, Hp=9, Wp=17, H=3, d=64, kinds="pwpp", nodes=2, causal=True, hidden=(1,)),
    dict(F=1, Hp=7, Wp=30, H=2, d=128, kinds="ppp", hidden=(0, 1, 2)),
    # full chunks whose query tiles see from a third to all of the own chunk: longest walks first
    dict(F=3, Hp=30, Wp=52, H=2, d=128, kinds="p", causal=True),
    dict(F=3, Hp=30, Wp=52, H=2, d=64, kinds="p", causal=True),
    # no history at all
    dict(F=1, Hp=9, Wp=15, H=2, d=128, kinds=""),
    # units split through the workspace: more of them than SMs, and a partial wave
    dict(F=3, Hp=20, Wp=26, H=12, d=128, kinds="pp", nodes=2),
    dict(F=3, Hp=20, Wp=26, H=14, d=64, kinds="pp", nodes=2),
]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_dense(sva_mod, case):
    """Against the formula, and the same bits as over the states read back (a node's slots in the same order, so the
    same plan, products and sums): unpacked by the units, beforehand, and as the call likes best."""
    a = Layer(sva_mod, seed=case, **CASES[case])
    out, lse = a.run(space=NONE)
    a.check(out, lse, heads=None if a.H <= 5 else (0, a.H - 1))
    for b_out, b_lse in (a.run_back(), a.run(space=a.space()), a.run(space=a.space(1 << 20)), a.run()):
        assert torch.equal(out, b_out) and torch.equal(lse, b_lse)
    a.close()


def _bools(a, g, what):
    T, nt, W = a.T, -(-a.T // 128), max(len(s) for s in a.states)
    rand = lambda *s: torch.rand(s, generator=g, device="cuda")  # noqa: E731
    b = {}
    if "tile" in what:
        b["tile"] = rand(a.n, nt, (1 + W) * nt) < 0.4
        b["tile"][:, 0] = False                # a query tile that attends nothing
    if "own" in what:
        b["own"] = rand(a.n, T, T) < 0.3
    if "hist" in what:
        b["hist"] = rand(a.n, T, W, T) < 0.3
        b["hist"][:, :, 0] = False             # a state that nobody sees
    for k in ("own", "hist"):
        if k in b:
            b[k][:, 5::41] = False             # queries that see none of it
    return b


def _words(a, b):
    out = {}
    for k, name in (("tile", "tile_mask"), ("own", "own_mask"), ("hist", "hist_mask")):
        if k in b:
            out[name] = pack_bits(b[k].cpu(), -(-b[k].shape[-1] // 32)).cuda()
    return out


@pytest.mark.parametrize("what", [("tile",), ("own",), ("hist",), ("own", "hist"), ("tile", "own", "hist")])
@pytest.mark.parametrize("case", [dict(F=1, Hp=16, Wp=20, H=2, d=128, kinds="pwpp", nodes=2),
                                  dict(F=2, Hp=11, Wp=17, H=2, d=64, kinds="ppw", causal=True),
                                  dict(F=1, Hp=1, Wp=40, H=2, d=64, kinds="pp"),
                                  dict(F=3, Hp=16, Wp=20, H=12, d=128, kinds="pp", nodes=2, workspace=True)])
def test_masks(sva_mod, what, case):
    a = Layer(sva_mod, seed=11, **case)
    b = _bools(a, torch.Generator(device="cuda").manual_seed(12), what)
    out, lse = a.run(space=NONE, **_words(a, b))
    a.check(out, lse, heads=(0, a.H - 1), **b)
    b_out, b_lse = a.run_back(**_words(a, b))
    if what != ("tile",):      # the same instance's arithmetic
        assert torch.equal(out, b_out) and torch.equal(lse, b_lse)
    out, lse = a.run(space=a.space(), **_words(a, b))
    assert torch.equal(out, b_out) and torch.equal(lse, b_lse)
    a.close()


def test_scanned_masks(sva_mod):
    """A launch long enough that its token masks are scanned first (12000 walks of a key tile)."""
    a = Layer(sva_mod, F=3, Hp=20, Wp=26, H=12, d=128, kinds="pwpp", nodes=3, seed=13)
    assert 3 * a.H * 7 * 4 * 13 >= 12000
    b = _bools(a, torch.Generator(device="cuda").manual_seed(14), ("own", "hist"))
    b["hist"][:, :512] = False
    for space in (NONE, a.space()):
        out, lse = a.run(space=space, **_words(a, b))
        a.check(out, lse, heads=(3,), **b)
    a.close()


def test_masked_values_do_not_leak(sva_mod):
    """NaN groups (a packed infinity) in keys and values that no query sees leave the others alone; seen, they are
    NaN in the output as they would be from a whole slot."""
    sva = sva_mod
    c = make_cache(sva, 1, 1, 200, 2, 64, 4, 2)
    g = torch.Generator(device="cuda").manual_seed(15)
    x, y, own = (random_kv(c, g) for _ in range(3))
    y[:, :, 3, 5] = float("inf")
    s = [write(c, (0, 1, 0), x), write(c, (0, 2, 0), y)]
    p = [c.bind_packed(0, 1, 0), c.bind_packed(0, 2, 0)]
    c.pack(s, p)
    o = write(c, (0, 3, 0), own)
    q = torch.randn((1, 200, 2, 64), generator=g, device="cuda").bfloat16()
    out, lse = torch.empty_like(q), torch.empty((1, 2, 200), device="cuda")
    node = dict(seq=0, chunk=3, level=0, own_slot=o, ctx=p)
    c.attend_nodes_packed([dict(node, visible=[1, 0])], q, out, lse)
    for h in range(2):
        k, v = (torch.cat([own[i, h].double(), held(x[i, h])]) for i in (0, 1))
        assert_attention(out[0, :, h], lse[0, h], attention(q[0, :, h], k, v))
    c.attend_nodes_packed([node], q, out, lse)
    assert out.isnan().all() and lse.isnan().all()
    c.close()


def test_without_packed_contexts(sva_mod):
    """Only whole states, or only hidden packed ones: the bits of the other entry points."""
    a = Layer(sva_mod, F=1, Hp=16, Wp=20, H=3, d=128, kinds="www", nodes=2, seed=16)
    out, lse = a.run()
    b_out, b_lse = a.buffers()
    a.c.attend_nodes(a.nodes_back, a.q, b_out, b_lse)
    assert torch.equal(out, b_out) and torch.equal(lse, b_lse)
    a.close()


def test_repeatable_in_graphs_and_streams(sva_mod):
    """The same bits launch after launch, in a graph whose packed states are packed anew in it, and on another stream;
    the split workspace's counters are left as they were."""
    for case in (dict(F=1, Hp=16, Wp=20, H=5, d=128, kinds="pppppppp"), dict(F=3, Hp=20, Wp=26, H=14, d=64, kinds="pp", nodes=2),
                 dict(F=3, Hp=20, Wp=26, H=12, d=128, kinds="pp", nodes=2)):
        a = Layer(sva_mod, seed=17, **case)
        out, lse = a.run()
        for _ in range(5):
            o, l = a.run()
            assert torch.equal(o, out) and torch.equal(l, lse)
        src = [a.c.lookup(0, 1 + i, 1) for i in range(a.W)]
        p = [a.c.lookup_packed(0, 1 + i, 0) for i in range(a.W)]
        o, l = a.buffers()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            a.c.pack(src, p)                   # what was read back, packed again: the same
            a.c.attend_nodes_packed(a.nodes, a.q, o, l)
        a.c.packed.fill_(255)      # (scales of NaN)
        for _ in range(3):
            o.zero_()
            graph.replay()
            assert torch.equal(o, out) and torch.equal(l, lse)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            a.c.packed.fill_(255)
            a.c.pack(src, p)
            o.zero_()
            a.c.attend_nodes_packed(a.nodes, a.q, o, l)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(o, out) and torch.equal(l, lse)
        assert a.c.poll() == sva_mod.OK
        del graph
        a.close()


@pytest.mark.parametrize("case", [dict(F=1, Hp=16, Wp=20, H=2, d=128, kinds="pp", workspace=False),
                                  dict(F=1, Hp=16, Wp=20, H=2, d=64, kinds="pp", workspace=False),
                                  dict(F=1, Hp=16, Wp=20, H=2, d=128, kinds="pppp"),
                                  dict(F=1, Hp=1, Wp=100, H=2, d=128, kinds="pp", workspace=False)])
def test_timeout(sva_mod, case):
    """A V tile that is withheld (of the own slot, or a packed one as the second tile) ends in the status and
    nothing worse, and the next launch gives the same bits as before."""
    a = Layer(sva_mod, seed=18, **case)
    out, lse = a.run()
    for space in (NONE, a.space()):
        a.c.debug_inject(1, 0.2)
        o, l = a.buffers()
        a.c.attend_nodes_packed(a.nodes, a.q, o, l, space=space)
        assert a.c.poll() == sva_mod.ERR_DEVICE_TIMEOUT
        a.c.debug_inject(0, 1.0)
        o, l = a.run(space=space)
        assert torch.equal(o, out) and torch.equal(l, lse)
    a.close()


def test_space(sva_mod):
    """A space that is short by a byte is not written; one that overlaps anything of the call or is not aligned is
    refused; the last key rows behind T are zeros whatever it held."""
    sva = sva_mod
    a = Layer(sva, F=1, Hp=9, Wp=15, H=2, d=64, kinds="ppw", seed=20)
    out, lse = a.run(space=NONE)
    short = a.space(-1)
    before = short.clone()
    o, l = a.run(space=short)
    assert torch.equal(o, out) and torch.equal(l, lse) and torch.equal(short, before)
    full = torch.full_like(a.space(), 255)          # bf16 NaN
    o, l = a.run(space=full)
    assert torch.equal(o, out) and torch.equal(l, lse)
    n = full.numel()
    need = torch.full((n + 512,), 255, dtype=torch.uint8, device="cuda")
    bad = sva.ERR_INVALID_ARGUMENT

    def call(space, q=a.q, out=out, **kw):
        return status(lambda: a.c.attend_nodes_packed(a.nodes, q, out, space=space, **kw))

    assert call(need[16:n + 16]) == bad
    whole = torch.empty(n + a.q.numel() * 2, dtype=torch.uint8, device="cuda")
    inside = whole[n - 256:n - 256 + a.q.numel() * 2].view(torch.bfloat16).view(a.q.shape)
    inside.copy_(a.q)
    kept = whole.clone()
    assert call(whole[:n], q=inside) == bad and "q" in sva.last_error()
    assert call(whole[:n], out=inside) == bad and "out" in sva.last_error()
    assert torch.equal(whole, kept)
    assert call(a.c.ws[256:256 + n]) == bad
    assert call(whole[:n], own_mask=whole[:4 * a.T * 5].view(torch.int32).view(1, a.T, 5)) == bad
    lib = sva.load()
    host = torch.empty(n + 256, dtype=torch.uint8)
    at = (host.data_ptr() + 255) // 256 * 256
    assert lib.sva_attend_nodes_packed(a.c.handle, a.nodes, 1, a.q.data_ptr(), out.data_ptr(), None, 0.125, None, at, n,
                                       0) == bad
    assert a.c.poll() == sva.OK
    a.close()


def test_advice(sva_mod):
    """Full chunks are unpacked first, small launches by their units, and nothing where nothing is packed or seen; the
    call takes what it is advised."""
    lib = sva_mod.load()
    for want, case in ((3, dict(F=3, Hp=30, Wp=52, H=4, d=128, kinds="pppw", nodes=2)), (0, dict(F=1, Hp=16, Wp=20, H=4, d=128, kinds="pp")),
                       (0, dict(F=3, Hp=30, Wp=52, H=2, d=64, kinds="ww")),
                       (0, dict(F=3, Hp=30, Wp=52, H=2, d=64, kinds="pp", hidden=(0, 1)))):
        a = Layer(sva_mod, seed=21, **case)
        c = a.c
        assert lib.sva_attend_packed_space(c.handle, a.nodes, a.n) == want * 2 * c.H * c.Tpad * c.d * 2
        out, lse = a.run()
        b_out, b_lse = a.run_back()
        assert torch.equal(out, b_out) and torch.equal(lse, b_lse)
        a.close()
    assert lib.sva_attend_packed_space(None, None, 1) == 0


def test_full_chunks(sva_mod):
    """4680 tokens, three packed states and a whole one, 12 heads: two of the heads against the formula."""
    a = Layer(sva_mod, F=3, Hp=30, Wp=52, H=12, d=128, kinds="pppw", seed=19)
    out, lse = a.run()
    a.check(out, lse, heads=(0, 11))
    b_out, b_lse = a.run_back()
    assert torch.equal(out, b_out) and torch.equal(lse, b_lse)
    a.close()


@pytest.mark.parametrize("d", [64, 128])
def test_longest_chunk(sva_mod, d):
    """65536 tokens, 512 tiles a state: queries of the first, a middle and the last tile against the formula."""
    a = Layer(sva_mod, F=1, Hp=256, Wp=256, H=1, d=d, kinds="p", seed=22)
    rows = torch.cat([torch.arange(r, r + 40, device="cuda") for r in (0, 32700, 65496)])
    k, v = (torch.cat([a.kv[s][x, 0].double() for s in a.see[0]]) for x in (0, 1))
    ref = attention(a.q[0, rows, 0], k, v)
    outs = [a.run(space=NONE), a.run(space=a.space())]
    for out, lse in outs:
        assert_attention(out[0, rows, 0], lse[0, 0, rows], ref)
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    a.close()


def test_most_nodes_and_contexts(sva_mod):
    """64 nodes of one token with sixteen contexts each, eighty distinct packed states among them: more than one
    launch unpacks at a time."""
    sva, H, d = sva_mod, 1, 64
    c = make_cache(sva, 1, 1, 1, H, d, 64 + 1, 80, chunks=200)
    g = torch.Generator(device="cuda").manual_seed(23)
    kv, packed = [], []
    for i in range(80):
        x = random_kv(c, g)
        s = write(c, (0, 1 + i, 0), x)
        packed.append(c.bind_packed(0, 1 + i, 0))
        c.pack([s], [packed[i]])
        c.release(0, 1 + i, 0)
        kv.append(held(x))
    nodes, own = [], []
    for i in range(64):
        x = random_kv(c, g)
        own.append(x)
        nodes.append(dict(seq=0, chunk=100 + i, level=0, own_slot=write(c, (0, 100 + i, 0), x),
                          ctx=[packed[(5 * i + k) % 80] for k in range(16)]))
    q = torch.randn((64, 1, H, d), generator=g, device="cuda").bfloat16()
    out, lse = torch.empty_like(q), torch.empty((64, H, 1), device="cuda")
    first = None
    for space in (NONE, torch.randint(0, 256, (80 * 2 * 128 * d * 2,), dtype=torch.uint8, device="cuda"), None):
        out.fill_(7.0)
        c.attend_nodes_packed(nodes, q, out, lse, space=space)
        first = out.clone() if first is None else first
        assert torch.equal(out, first)
        for i in range(64):
            k, v = (torch.cat([own[i][x, 0].double()] + [kv[(5 * i + j) % 80][x, 0] for j in range(16)]) for x in (0, 1))
            assert_attention(out[i, :, 0], lse[i, 0], attention(q[i, :, 0], k, v), f"node {i}")
    assert c.poll() == sva.OK
    c.close()

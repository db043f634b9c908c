"""Packed slots (sva_cache_pack, sva_cache_unpack) and copies of states (sva_cache_copy): values against the
definition, what may not change, and every refusal."""
import pytest
import torch

from tests._packed import held, make_cache, random_kv, status, write

pytestmark = pytest.mark.gpu

# (F, Hp, Wp, H, d): one token; one short of, at and past a tile; past a pair of tiles; a full chunk
SIZES = [(1, 1, 1, 1, 64), (1, 1, 1, 3, 128), (1, 1, 127, 2, 128), (1, 8, 16, 5, 64), (1, 3, 43, 2, 128),
         (2, 11, 13, 3, 64), (3, 30, 52, 2, 128)]


def _same(a, b):
    """Equal, NaN where NaN."""
    a, b = a.double(), b.double()
    return torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(1.5), b.nan_to_num(1.5))


@pytest.mark.parametrize("size", SIZES)
def test_round_trip(sva_mod, size):
    F, Hp, Wp, H, d = size
    n = 3
    c = make_cache(sva_mod, F, Hp, Wp, H, d, 2 * n, n + 1)
    g = torch.Generator(device="cuda").manual_seed(1)
    kv = [random_kv(c, g, 1.0) for _ in range(n)]
    kv[1][:, :, c.T // 2] = 0
    kv[2][0, 0, 0, :32] = 3.0 * 2.0 ** 100        # group by group: large, tiny, as it comes
    kv[2][1, H - 1, c.T - 1, 32:64] *= 2.0 ** -119
    src = [write(c, (0, 1 + i, 0), x) for i, x in enumerate(kv)]
    # a packed slot of a later level, out of order, the last one left alone
    packed = [c.bind_packed(0, 1 + i, 2) for i in (2, 0, 1)]
    packed = [packed[1], packed[2], packed[0]]
    assert sorted(packed) == [sva_mod.PACKED + i for i in range(n)]
    before = c.packed.clone()
    pool = c.slot_pool()
    whole = pool.clone()
    c.pack(src, packed)
    assert torch.equal(pool.view(torch.int16), whole.view(torch.int16))
    one = c.packed.numel() // (n + 1)
    assert torch.equal(c.packed[n * one:], before[n * one:])
    back = [c.bind(0, 1 + i, 1) for i in range(n)]
    kept = c.packed.clone()
    c.unpack(packed, back)
    assert torch.equal(c.packed, kept)
    for i in range(n):
        assert _same(pool[back[i], :, :, : c.T], held(kv[i])), i
        assert (pool[back[i], :, :, c.T:] == 0).all()
        assert torch.equal(pool[src[i]].view(torch.int16), whole[src[i]].view(torch.int16))
    # packed from what was read back: the same bytes
    c.pack(back, packed)
    assert torch.equal(c.packed, kept)
    assert c.poll() == sva_mod.OK
    c.close()


@pytest.mark.parametrize("d", [64, 128])
def test_every_number_and_every_special_value(sva_mod, d):
    """Every bf16 number against largest magnitudes of every mantissa: exact halves among them, subnormals, infinities
    and NaN, which take their group and nothing else with them."""
    Wp = 65536 // (d - d // 32)
    c = make_cache(sva_mod, 1, 1, Wp, 1, d, 2, 1)
    every = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    x = torch.zeros((Wp, d // 32, 32), dtype=torch.bfloat16)
    every = every[: x.numel() // 32 * 31]
    x.view(-1, 32)[: every.numel() // 31, 1:] = every[: every.numel() // 31 * 31].view(-1, 31)
    kv = torch.stack((x.flatten(-2), x.flatten(-2).flip(0)))[:, None].cuda()
    g = torch.Generator(device="cuda").manual_seed(2)
    # V: largest magnitudes of every mantissa, with elements that are small multiples of halves of their scale
    m = torch.randint(128, 256, (Wp, d // 32, 1), generator=g, device="cuda").double()
    s = held(m.expand(Wp, d // 32, 32).bfloat16())[..., :1] / 7
    half = torch.randint(-13, 14, (Wp, d // 32, 32), generator=g, device="cuda") / 2 * s
    half[..., 0] = m[..., 0]
    kv[1, 0] = half.flatten(-2).bfloat16()
    src = write(c, (0, 1, 0), kv)
    p, back = c.bind_packed(0, 1, 0), c.bind(0, 1, 1)
    c.pack([src], [p])
    c.unpack([p], [back])
    got, want = c.slot_pool()[back][:, :, : c.T], held(kv)
    assert _same(got, want)
    assert want[0].isnan().any() and (want[0] == 0).any()
    c.close()


def test_graph_other_stream_and_sources_twice(sva_mod):
    c = make_cache(sva_mod, 1, 9, 20, 3, 128, 6, 4)
    g = torch.Generator(device="cuda").manual_seed(3)
    kv = [random_kv(c, g) for _ in range(2)]
    a, b = (write(c, (0, 1 + i, 0), x) for i, x in enumerate(kv))
    p = [c.bind_packed(0, 5, i) for i in range(4)]
    back = [c.bind(0, 6, i) for i in range(4)]
    pool = c.slot_pool()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c.pack([a, b, a, a], p)               # one source three times
        c.unpack([p[1], p[0], p[0], p[3]], back)
    side.synchronize()
    want = [held(kv[k]) for k in (1, 0, 0, 0)]
    for s, w in zip(back, want):
        assert _same(pool[s, :, :, : c.T], w)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.pack([b, a], p[:2])
        c.unpack(p[:2], back[:2])
    for k in range(3):                        # the graph reads what the slots hold when it runs
        new = [random_kv(c, g) for _ in range(2)]
        pool[a, :, :, : c.T], pool[b, :, :, : c.T] = new
        graph.replay()
        assert _same(pool[back[0], :, :, : c.T], held(new[1])) and _same(pool[back[1], :, :, : c.T], held(new[0]))
    del graph
    c.close()


def test_refusals(sva_mod):
    sva = sva_mod
    c = make_cache(sva, 1, 5, 7, 2, 64, 4, 3)
    g = torch.Generator(device="cuda").manual_seed(4)
    a = write(c, (0, 5, 0), random_kv(c, g))
    blank = c.bind(0, 6, 0)                   # bound, not written
    p = c.bind_packed(0, 5, 0)
    later, early = c.bind_packed(0, 6, 0), c.bind_packed(0, 4, 0)
    assert status(lambda: c.bind_packed(0, 7, 0)) == sva.ERR_CAPACITY
    assert status(lambda: c.bind_packed(0, 5, 0)) == sva.ERR_INVALID_ARGUMENT
    assert status(lambda: c.bind_packed(0, 5, -1)) == sva.ERR_INVALID_ARGUMENT
    assert c.lookup_packed(0, 6, 0) == later and status(lambda: c.lookup_packed(0, 9, 0)) == sva.ERR_NOT_RESIDENT
    assert status(lambda: c.release_packed(0, 9, 0)) == sva.ERR_NOT_RESIDENT
    assert status(lambda: c.lookup(0, 4, 0)) == sva.ERR_NOT_RESIDENT       # tables of their own
    torch.cuda.synchronize()
    pool, bits = c.slot_pool().clone(), c.packed.clone()
    bad, gone, cap, causal = sva.ERR_INVALID_ARGUMENT, sva.ERR_NOT_RESIDENT, sva.ERR_CAPACITY, sva.ERR_CAUSALITY
    P = sva.PACKED
    for want, src, dst in [(bad, [], []), (cap, [a] * 65, [p] * 65), (gone, [blank], [p]), (bad, [a], [a]), (bad, [a], [blank]),
                           (bad, [-1], [p]), (bad, [4], [p]), (bad, [a], [P + 3]), (bad, [a], [P - 1]), (bad, [a], [-1]),
                           (bad, [a, a], [p, p]), (causal, [a], [early]), (gone, [P], [p]), (gone, [3], [p]),
                           (bad, [2 ** 31 - 1], [p]), (bad, [a], [2 ** 31 - 1])]:
        assert status(lambda: c.pack(src, dst)) == want, (src, dst)
    for want, src, dst in [(bad, [], []), (gone, [p], [blank]), (gone, [later], [blank])]:
        assert status(lambda: c.unpack(src, dst)) == want, (src, dst)
    with pytest.raises(ValueError):
        c.pack([a], [])
    torch.cuda.synchronize()
    assert torch.equal(pool.view(torch.int16), c.slot_pool().view(torch.int16)) and torch.equal(bits, c.packed)
    c.pack([a], [p])
    c.release_packed(0, 4, 0)
    other = c.bind_packed(1, 9, 0)
    assert status(lambda: c.pack([a], [other])) == causal                  # another sequence
    for want, src, dst in [(bad, [p], [p]), (bad, [p], [later]), (bad, [a], [blank]), (bad, [p, p], [blank, blank]),
                           (bad, [p], [3])]:
        assert status(lambda: c.unpack(src, dst)) == want, (src, dst)
    c.release(0, 6, 0)
    before = c.bind(0, 4, 3)
    assert status(lambda: c.unpack([p], [before])) == causal
    # a packed slot that was released and bound anew holds nothing
    c.release_packed(0, 5, 0)
    again = c.bind_packed(0, 5, 1)
    assert again == p and status(lambda: c.unpack([again], [c.bind(0, 8, 0)])) == gone
    # the other calls read no packed slots
    c.pack([a], [again])
    own = write(c, (0, 9, 0), random_kv(c, g))
    nodes = [dict(seq=0, chunk=9, level=0, own_slot=own, ctx=[again])]
    q = torch.randn((1, c.T, c.H, c.d), device="cuda").bfloat16()
    out = torch.full_like(q, 7.0)
    assert status(lambda: c.attend_nodes(nodes, q, out)) == bad and "attend_nodes_packed" in sva.last_error()
    assert status(lambda: c.attend_nodes_masked(nodes, q, out)) == bad
    w = torch.zeros((4, c.H, c.T), device="cuda")
    lse = torch.zeros((1, c.H, c.T), device="cuda")
    assert status(lambda: c.attend_weights(nodes, q, lse, w)) == bad
    index = torch.zeros((c.H, c.T), dtype=torch.int32, device="cuda")
    assert status(lambda: c.condense([again], own, w, index)) == bad
    assert status(lambda: c.rope_kv_write([dict(seq=0, chunk=5, level=1, own_slot=again)], q, q)) == bad
    # and the packed attention none as a node's own slot, nor one that was not packed, nor another sequence's
    call = lambda **kw: status(lambda: c.attend_nodes_packed([dict(nodes[0], **kw)], q, out))  # noqa: E731
    assert call(own_slot=again) == bad and call(ctx=[later]) == gone and call(ctx=[P + 3]) == bad
    assert call(ctx=[again, again]) == bad and call(ctx=[P - 1]) == bad and call(ctx=[other]) == gone
    c.release_packed(0, 6, 0)
    far = c.bind_packed(0, 12, 0)
    c.pack([own], [far])
    c.release_packed(0, 5, 1)
    again = c.bind_packed(0, 5, 0)
    c.pack([a], [again])
    assert call(ctx=[a, again]) == bad and call(ctx=[again, a]) == bad       # one state, whole and packed
    assert "same state" in sva.last_error()
    assert call(ctx=[far]) == causal
    torch.cuda.synchronize()
    assert (out == 7.0).all()
    # buffers
    small = torch.empty(sva.packed_bytes(c.g, 2), dtype=torch.uint8, device="cuda")
    assert status(lambda: c.set_packed(small, 2)) == bad                   # slots are bound
    assert status(lambda: c.set_packed(None)) == bad
    for s in ((0, 5, 0), (1, 9, 0), (0, 12, 0)):
        c.release_packed(*s)
    assert status(lambda: c.set_packed(small, 3)) == bad                   # too small
    assert status(lambda: c.set_packed(small, 0)) == bad
    assert status(lambda: c.set_packed(small[16:], 1)) == bad              # alignment
    assert status(lambda: c.set_packed(c.buf, 1)) == bad                   # the cache's own memory
    assert status(lambda: c.set_packed(c.ws[256:], 1)) == bad
    lib = sva.load()
    host = torch.empty(sva.packed_bytes(c.g, 1) + 256, dtype=torch.uint8)
    at = (host.data_ptr() + 255) // 256 * 256
    assert lib.sva_cache_set_packed(c.handle, at, sva.packed_bytes(c.g, 1), 1) == bad
    room = torch.empty(c.workspace_bytes(), dtype=torch.uint8, device="cuda")
    c.set_packed(room[-sva.packed_bytes(c.g, 1) // 256 * 256:], 1)
    assert status(lambda: c.set_workspace(room)) == bad
    c.set_packed(None)
    c.set_workspace(room)
    c.set_packed(small, 2)
    assert c.bind_packed(0, 1, 0) == P and c.bind_packed(0, 2, 0) == P + 1
    c.release_packed(0, 1, 0)
    c.release_packed(0, 2, 0)
    c.set_packed(None)
    assert status(lambda: c.bind_packed(0, 1, 0)) == sva.ERR_CAPACITY
    c.close()


@pytest.mark.parametrize("size", SIZES)
def test_copy(sva_mod, size):
    """Within a cache, with a source given twice, and into a larger one; slots and packed slots; nothing else moves."""
    F, Hp, Wp, H, d = size
    c = make_cache(sva_mod, F, Hp, Wp, H, d, 6, 3, chunks=20)
    big = make_cache(sva_mod, F, Hp, Wp, H, d, 9, 5, chunks=50)
    g = torch.Generator(device="cuda").manual_seed(5)
    kv = [random_kv(c, g) for _ in range(2)]
    kv[0].view(torch.int16)[0, 0, 0] = torch.arange(d, dtype=torch.int16, device="cuda") + 0x7F70   # NaN payloads too
    src = [write(c, (0, 1 + i, 0), x) for i, x in enumerate(kv)]
    to = [c.bind(1, 2, i) for i in range(3)]
    bits = lambda t: t.view(torch.int16)  # noqa: E731
    before = c.slot_pool().clone()
    c.copy([src[1], src[0], src[1]], [to[2], to[0], to[1]])
    pool = c.slot_pool()
    for s, k in ((to[2], 1), (to[0], 0), (to[1], 1), (src[0], 0), (src[1], 1)):
        assert torch.equal(bits(pool[s, :, :, : c.T].contiguous()), bits(kv[k])) and (pool[s, :, :, c.T:] == 0).all()
    spare = ({0, 1, 2, 3, 4, 5} - set(src) - set(to)).pop()
    assert torch.equal(bits(pool[spare]), bits(before[spare]))
    far = big.bind(7, 30, 3)
    blank = big.slot_pool().clone()
    c.copy([to[0]], [far], to=big)
    assert torch.equal(bits(big.slot_pool()[far, :, :, : c.T].contiguous()), bits(kv[0]))
    rest = [s for s in range(9) if s != far]
    assert torch.equal(bits(big.slot_pool()[rest]), bits(blank[rest]))
    # packed slots
    p = [c.bind_packed(0, 2, i) for i in range(3)]
    c.pack([src[1]], [p[1]])
    c.copy([p[1], p[1]], [p[2], p[0]])
    q = big.bind_packed(3, 9, 0)
    c.copy([p[0]], [q], to=big)
    one = c.packed.numel() // 3
    a = c.packed.view(3, one)
    assert torch.equal(a[0], a[1]) and torch.equal(a[2], a[1])
    assert torch.equal(big.packed.view(5, one)[q - sva_mod.PACKED], a[1])
    back = big.bind(3, 9, 1)
    big.unpack([q], [back])
    assert _same(big.slot_pool()[back, :, :, : c.T], held(kv[1]))
    c.close()
    big.close()


def test_copy_refusals(sva_mod):
    sva = sva_mod
    c = make_cache(sva, 1, 5, 7, 2, 64, 5, 2)
    g = torch.Generator(device="cuda").manual_seed(6)
    a = write(c, (0, 5, 0), random_kv(c, g))
    b, early = c.bind(1, 5, 0), c.bind(1, 4, 0)
    p, p2 = c.bind_packed(0, 5, 0), c.bind_packed(1, 6, 0)
    before = c.slot_pool().clone()
    bad, gone, cap, causal = sva.ERR_INVALID_ARGUMENT, sva.ERR_NOT_RESIDENT, sva.ERR_CAPACITY, sva.ERR_CAUSALITY
    for want, src, dst in [(bad, [], []), (cap, [a] * 65, [b] * 65), (gone, [b], [early]), (bad, [a], [a]), (causal, [a], [early]),
                           (bad, [a, a], [b, b]), (bad, [a], [4]), (bad, [a], [99]), (bad, [-1], [b]), (bad, [a], [p]),
                           (gone, [p], [p2])]:
        assert status(lambda: c.copy(src, dst)) == want, (src, dst)
    c.pack([a], [p])
    assert status(lambda: c.copy([p], [b])) == bad and status(lambda: c.copy([a, p], [b, p2])) == bad
    for kw in (dict(H=3), dict(d=128), dict(Wp=8), dict(F=5, Hp=1)):
        size = dict(dict(F=1, Hp=5, Wp=7, H=2, d=64), **kw)
        other = make_cache(sva, size["F"], size["Hp"], size["Wp"], size["H"], size["d"], 2, 0)
        t = other.bind(0, 5, 0)
        assert status(lambda: c.copy([a], [t], to=other)) == bad, kw
        other.close()
    geo = sva.make_geometry(2, 64, 1, 5, 7, 2, (12, 10, 10), 50, theta=5000.0)
    other = sva.Cache(geo)
    t = other.bind(0, 5, 0)
    assert status(lambda: c.copy([a], [t], to=other)) == bad
    other.close()
    twin = sva.Cache(c.g, buf=torch.empty(2 * c.nbytes, dtype=torch.uint8, device="cuda"))
    t = twin.bind(0, 5, 0)
    twin.set_packed(c.packed, 1)
    assert status(lambda: c.copy([a], [t], to=twin)) == bad and "share" in sva.last_error()
    twin.set_packed(None)
    c.copy([a], [t], to=twin)
    twin.close()
    torch.cuda.synchronize()
    assert torch.equal(before.view(torch.int16), c.slot_pool().view(torch.int16))
    c.close()


def test_past_32_bits(sva_mod):
    """Slots and packed slots whose bytes lie past 2^32, copied, packed and read back there."""
    c = make_cache(sva_mod, 1, 128, 128, 32, 128, 20, 70)       # 268 MB a slot, 75 MB a packed one
    assert c.nbytes // 20 * 18 > 1 << 32 and c.packed.numel() // 70 * 69 > 1 << 32
    g = torch.Generator(device="cuda").manual_seed(7)
    kv = random_kv(c, g)
    slots = [c.bind(0, 1, i) for i in range(20)]
    packed = [c.bind_packed(0, 1, i) for i in range(70)]
    blank = torch.zeros((1, c.T, c.H, c.d), dtype=torch.bfloat16, device="cuda")
    c.rope_kv_write([dict(seq=0, chunk=1, level=0, own_slot=slots[0])], blank, blank)
    pool = c.slot_pool()
    pool[slots[0], :, :, : c.T] = kv
    c.copy([slots[0]], [slots[19]])
    assert torch.equal(pool[19], pool[0])
    c.pack([slots[19]], [packed[69]])
    c.copy([packed[69]], [packed[1]])
    c.unpack([packed[69], packed[1]], [slots[18], slots[1]])
    assert torch.equal(pool[18], pool[1])
    for h in (0, 31):
        assert _same(pool[18, :, h], held(kv[:, h]))
    c.close()

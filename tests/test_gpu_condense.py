"""Condensing states by weight (sva_cache_condense): which tokens, in which order, copied bit for bit.

The selection is exact (whole numbers and copies), so every comparison is equality.  The expected
tokens come from a sort of (weight descending, candidate ascending) in Python numbers.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def _pairs(d):
    return (d // 2 - 2 * (d // 6), d // 6, d // 6)


def _cache(sva, F, Hp, Wp, H, d, n_src, spare=1, seed=2):
    """A cache of n_src written states (chunks 1..) in shuffled slots and a free destination; random bits in the pool."""
    T = F * Hp * Wp
    c = sva.Cache(sva.make_geometry(H, d, F, Hp, Wp, n_src + 1 + spare, _pairs(d), F * (n_src + 4)))
    g = torch.Generator(device="cuda").manual_seed(seed)
    order = torch.randperm(n_src, generator=torch.Generator().manual_seed(seed)).tolist()
    slot = {}
    blank = torch.zeros((1, T, H, d), dtype=torch.bfloat16, device="cuda")
    for i in order:
        slot[i] = c.bind(0, 1 + i, 0)
        c.rope_kv_write([dict(seq=0, chunk=1 + i, level=0, own_slot=slot[i])], blank, blank)
    dst = c.bind(0, n_src, 9)
    pool = c.slot_pool().view(torch.int16)
    pool[:, :, :, :T] = torch.randint(-2 ** 15, 2 ** 15, pool[:, :, :, :T].shape, generator=g, device="cuda", dtype=torch.int32).to(torch.int16)
    return c, [slot[i] for i in range(n_src)], dst, g


def _expected(w):
    """w [n * T] floats of one head, T kept -> ascending candidates."""
    def run(T):
        v = [(-math.inf if math.isnan(x) else x) for x in w.tolist()]
        return sorted(sorted(range(len(v)), key=lambda e: (-v[e], e))[:T])
    return run


def _check(c, src, dst, weight, T, H):
    before_pool, before_w = c.slot_pool().view(torch.int16).clone(), weight.clone()
    index = torch.full((H, T), -5, dtype=torch.int32, device="cuda")
    c.condense(src, dst, weight, index)
    assert c.poll() == 0
    pool = c.slot_pool().view(torch.int16)
    for h in range(H):
        cand = torch.cat([before_w[s, h] for s in src])
        want = _expected(cand.cpu())(T)
        assert index[h].tolist() == want, f"head {h}"
        at = torch.tensor(want, device="cuda")
        assert torch.equal(weight[dst, h].view(torch.int32), cand[at].view(torch.int32))
        for kv in (0, 1):
            rows = torch.cat([before_pool[s, kv, h, :T] for s in src])
            assert torch.equal(pool[dst, kv, h, :T], rows[at]), f"head {h} {'KV'[kv]}"
    rest = [s for s in range(pool.shape[0]) if s != dst]
    assert torch.equal(pool[rest], before_pool[rest]) and torch.equal(weight[rest].view(torch.int32), before_w[rest].view(torch.int32))
    assert torch.all(pool[dst, :, :, T:] == before_pool[dst, :, :, T:])
    return index


@pytest.mark.parametrize("F,Hp,Wp,H,d,n", [
    (1, 1, 1, 1, 64, 1), (1, 1, 1, 3, 128, 16), (1, 6, 7, 2, 64, 1), (1, 6, 7, 2, 128, 3), (1, 16, 20, 12, 128, 4),
    (1, 32, 32, 2, 64, 4),       # 4096 candidates: one CTA a head, and one more:
    (1, 1, 4097, 1, 64, 1),
    (3, 11, 29, 3, 64, 6), (1, 60, 61, 2, 128, 2), (3, 30, 52, 2, 128, 7), (1, 65, 67, 1, 64, 16)])
def test_random_weights(sva_mod, F, Hp, Wp, H, d, n):
    T = F * Hp * Wp
    c, src, dst, g = _cache(sva_mod, F, Hp, Wp, H, d, n)
    w = torch.exp(2 * torch.randn((n + 2, H, T), generator=g, device="cuda"))
    _check(c, src, dst, w, T, H)
    c.close()


@pytest.mark.parametrize("F,Hp,Wp,H,d,n", [(1, 8, 16, 3, 64, 16), (1, 3, 43, 3, 64, 15), (1, 8, 8, 3, 128, 16),
                                           (1, 5, 13, 3, 128, 16), (1, 1, 2, 40, 128, 2), (2, 3, 7, 12, 64, 5)])
def test_small_states(sva_mod, F, Hp, Wp, H, d, n):
    """Rows copied by the selection (up to 128 tokens of 64, 64 of 128) and by a launch of their own, ties among them."""
    T = F * Hp * Wp
    c, src, dst, g = _cache(sva_mod, F, Hp, Wp, H, d, n)
    w = torch.floor(3 * torch.rand((n + 2, H, T), generator=g, device="cuda"))
    _check(c, src, dst, w, T, H)
    c.close()


@pytest.mark.parametrize("kind", ["zeros", "equal", "few", "signs", "nan", "all nan", "inf", "close", "subnormal", "line"])
def test_ties_and_odd_values(sva_mod, kind):
    """Equal weights go to the lowest candidates, over CTA borders too (2214 candidates a CTA)."""
    F, Hp, Wp, H, d, n = 1, 27, 41, 2, 64, 8
    T = F * Hp * Wp
    c, src, dst, g = _cache(sva_mod, F, Hp, Wp, H, d, n)
    shape = (n + 2, H, T)
    w = torch.rand(shape, generator=g, device="cuda")
    u = torch.rand(shape, generator=g, device="cuda")
    if kind == "zeros":
        w[u < 0.95] = 0.0
    elif kind == "equal":
        w.fill_(0.25)
    elif kind == "few":
        w = torch.floor(w * 3)
    elif kind == "signs":
        w = torch.where(u < 0.4, torch.zeros_like(w), w - 0.9)
        w = torch.where(u < 0.2, -w.abs() * 0.0, w)      # -0 ties with 0
    elif kind == "nan":
        w[u < 0.9] = math.nan
        w[u < 0.3] = -math.inf
    elif kind == "all nan":
        w.fill_(math.nan)
    elif kind == "inf":
        w[u < 0.2] = math.inf
    elif kind == "close":
        w = 1.0 + torch.floor(u * 8) * 2.0 ** -23
    elif kind == "subnormal":
        w = torch.floor(u * 100) * 2.0 ** -149
    elif kind == "line":     # the T-th and (T + 1)-th candidates differ in the last bit only
        w.fill_(1.0)
        w[src[3]] = 1.0 + 2.0 ** -23
    _check(c, src, dst, w.contiguous(), T, H)
    c.close()


def test_long_range_is_read_again(sva_mod):
    """More candidates than a CTA holds: 16 states of 32768 tokens (65536 a CTA)."""
    T, n = 32768, 16
    c, src, dst, g = _cache(sva_mod, 2, 128, 128, 1, 64, n)
    w = torch.randint(0, 200000, (n + 2, 1, T), generator=g, device="cuda").float()
    _check(c, src, dst, w, T, 1)
    c.close()


def test_stream_graph_and_reuse(sva_mod):
    """On a side stream, from a graph, and again after the sources were freed and written anew."""
    F, Hp, Wp, H, d, n = 1, 27, 41, 3, 128, 5
    T = F * Hp * Wp
    c, src, dst, g = _cache(sva_mod, F, Hp, Wp, H, d, n)
    w = torch.rand((n + 2, H, T), generator=g, device="cuda")
    index = _check(c, src, dst, w, T, H)
    other = torch.zeros_like(index)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c.condense(src, dst, w, other, stream=side)
    side.synchronize()
    assert torch.equal(index, other)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.condense(src, dst, w, other)
    w[src] = torch.rand((n, H, T), generator=g, device="cuda")
    graph.replay()
    torch.cuda.synchronize()
    want = _check(c, src, dst, w, T, H)
    assert torch.equal(want, other)
    # a condensed state is a source like any other, and its slot's old tenant may go
    c.release(0, 1, 0)
    nxt = c.bind(0, n + 1, 9)
    assert nxt == src[0]
    _check(c, [dst] + src[1:], nxt, w, T, H)
    c.close()


def test_attention_over_a_condensed_state(sva_mod):
    """Tokens that nothing attended change nothing: attending over the condensed state gives the attention over both."""
    F, Hp, Wp, H, d = 1, 9, 14, 2, 64
    T = F * Hp * Wp
    c, src, dst, g = _cache(sva_mod, F, Hp, Wp, H, d, 2)
    pool = c.slot_pool()
    for s in src:
        pool[s, :, :, :T] = torch.randn((2, H, T, d), generator=g, device="cuda").bfloat16()
    half = torch.rand((H, 2 * T), generator=g, device="cuda").argsort(1)[:, :T]     # kept, head by head
    w = torch.zeros((4, H, T), device="cuda")
    flat = torch.zeros((H, 2 * T), device="cuda").scatter_(1, half, 1.0)
    w[src[0]], w[src[1]] = flat[:, :T], flat[:, T:]
    index = torch.empty((H, T), dtype=torch.int32, device="cuda")
    c.condense(src, dst, w, index)
    own = c.bind(0, 3, 1)
    blank = torch.zeros((1, T, H, d), dtype=torch.bfloat16, device="cuda")
    node = dict(seq=0, chunk=3, level=1, own_slot=own, ctx=[dst])
    c.rope_kv_write([node], blank, blank)
    q = torch.randn((1, T, H, d), generator=g, device="cuda").bfloat16()
    out = torch.empty_like(q)
    c.attend_nodes([node], q, out)
    for h in range(H):
        k = torch.cat([pool[s, 0, h, :T] for s in src]).double()[half[h]]
        v = torch.cat([pool[s, 1, h, :T] for s in src]).double()[half[h]]
        x = torch.cat([torch.zeros((T, T), device="cuda", dtype=torch.float64), q[0, :, h].double() @ k.t() / math.sqrt(d)], 1)
        p = torch.softmax(x, 1)[:, T:]
        # bf16 weights and output: 2^-8 of sum p |v| each
        assert torch.all((out[0, :, h].double() - p @ v).abs() <= 2.0 ** -7 * (p @ v.abs()) + 1e-3)
    c.close()


def test_refusals(sva_mod):
    sva = sva_mod
    F, Hp, Wp, H, d, n = 1, 6, 7, 2, 64, 3
    T = 42
    c, src, dst, g = _cache(sva, F, Hp, Wp, H, d, n, spare=3)
    w = torch.rand((n + 4, H, T), generator=g, device="cuda")
    index = torch.full((H, T), -5, dtype=torch.int32, device="cuda")
    before = c.slot_pool().view(torch.int16).clone()
    w0 = w.clone()

    def status(s, t, **kw):
        with pytest.raises(sva.SvaError) as e:
            c.condense(s, t, w, index, **kw)
        return e.value.status

    assert status([], dst) == sva.ERR_INVALID_ARGUMENT
    assert status(list(range(17)), dst) == sva.ERR_CAPACITY
    assert status([src[0], src[0]], dst) == sva.ERR_INVALID_ARGUMENT
    assert status([src[0], dst], dst) == sva.ERR_NOT_RESIDENT            # the destination, never written
    assert status([src[0], 99], dst) == sva.ERR_INVALID_ARGUMENT
    assert status([src[0], -1], dst) == sva.ERR_INVALID_ARGUMENT
    assert status(src, 99) == sva.ERR_INVALID_ARGUMENT
    assert status(src, n + 3) == sva.ERR_INVALID_ARGUMENT                # not bound
    empty = c.bind(0, 1, 5)
    assert status([src[0], empty], dst) == sva.ERR_NOT_RESIDENT
    early = c.bind(0, n - 1, 7)
    assert status(src, early) == sva.ERR_CAUSALITY                       # the last source is a later chunk
    alien = c.bind(4, n, 9)
    assert status(src, alien) == sva.ERR_CAUSALITY
    for bad in (dict(weight=w.double()), dict(weight=w[:2]), dict(index=index.long()), dict(index=index[:, :5])):
        a = dict(weight=w, index=index)
        a.update(bad)
        with pytest.raises(ValueError):
            c.condense(src, dst, **a)
    torch.cuda.synchronize()
    assert torch.all(index == -5) and torch.equal(w, w0) and torch.equal(c.slot_pool().view(torch.int16), before)
    # a refused destination did not become readable
    with pytest.raises(sva.SvaError) as e:
        c.condense([early], dst, w, index)
    assert e.value.status == sva.ERR_NOT_RESIDENT
    c.close()

"""RMSNorm of each head + 3D RoPE + cache write (sva_rope_kv_write_headnorm)
against the formulas in 64 bits.

Tolerance, per element of a rotated pair (a, b): the one bf16 rounding, at most
2^-8 of the value, plus the fp32 error in front of it.  Sum of squares, root,
gamma and rotation make about 16 roundings of 2^-24 on values of size |a| + |b|:
2^-20 (|a| + |b|) (and the smallest bf16 step, for values that underflow).
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

THETA = 10000.0


def _pairs(d):
    return (d // 2 - 2 * (d // 6), d // 6, d // 6)


def _geometry(sva, F, Hp, Wp, H, d, slots, max_frames=64):
    return sva.make_geometry(H, d, F, Hp, Wp, num_slots=slots, pairs=_pairs(d), max_frames=max_frames, theta=THETA)


def _ref(x, gamma, chunk, F, Hp, Wp, eps):
    """x [T][H][d] on the CPU -> (value, |a| + |b| of its pair), both [T][H][d] in 64 bits."""
    T, H, d = x.shape
    y = x.double()
    y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps)
    if gamma is not None:
        y = y * gamma.double().cpu()
    u = torch.arange(T)
    pos = (F * chunk + u // (Hp * Wp), u % (Hp * Wp) // Wp, u % Wp)
    ang = torch.cat([p.double()[:, None] * THETA ** (-torch.arange(n, dtype=torch.float64) / max(n, 1))
                     for p, n in zip(pos, _pairs(d))], dim=1)
    z = torch.view_as_complex(y.reshape(T, H, d // 2, 2).contiguous()) * torch.exp(1j * ang)[:, None]
    size = y.abs().reshape(T, H, d // 2, 2).sum(-1, keepdim=True).expand(T, H, d // 2, 2).reshape(T, H, d)
    return torch.view_as_real(z).reshape(T, H, d), size


def _assert_rotated(got, ref, size, what):
    err = (got.cpu().double() - ref).abs()
    bound = 2.0 ** -8 * ref.abs() + 2.0 ** -20 * size + 2.0 ** -133
    bad = ~(err <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((err - bound).max()):.3e}"


def _inputs(n, T, H, d, q, packed, seed=3):
    g = torch.Generator().manual_seed(seed)
    parts = 3 if q else 2
    x = torch.randn((n, T, parts, H, d), generator=g) * torch.exp(torch.randn((parts, H, d), generator=g))
    x[0, T // 2, :, H - 1] = 0.0
    x = x.to(torch.bfloat16).cuda()
    views = [x[:, :, i] for i in range(parts)]
    if not packed:
        views = [v.contiguous() for v in views]
    return (views[0] if q else None), views[-2], views[-1], g


# F, Hp, Wp, H, d, nodes, q, packed, gamma
CASES = [
    (1, 1, 1, 1, 64, 1, True, False, "shared"),      # one token, one narrow head: eight lanes of a warp
    (1, 1, 1, 1, 64, 5, True, True, "none"),
    (1, 1, 1, 1, 128, 3, False, False, "heads"),
    (1, 3, 1, 3, 64, 2, True, True, "heads"),        # 24 vectors a token: a half-used second step
    (2, 3, 7, 2, 64, 2, True, False, "shared"),
    (1, 6, 7, 5, 128, 1, True, True, "shared"),      # 42 tokens, 80 vectors
    (3, 5, 11, 7, 64, 3, False, True, "none"),       # 165 tokens, 56 vectors
    (1, 16, 20, 12, 128, 1, True, True, "heads"),
    (2, 9, 13, 13, 128, 2, True, False, "none"),
    (1, 20, 30, 40, 128, 1, False, False, "heads"),
    (1, 2, 2, 128, 128, 1, True, True, "shared"),    # the most heads
]


@pytest.mark.parametrize("F,Hp,Wp,H,d,n,has_q,packed,gamma", CASES)
def test_against_formula(sva_mod, F, Hp, Wp, H, d, n, has_q, packed, gamma):
    sva, T, eps = sva_mod, F * Hp * Wp, 1e-6
    cache = sva.Cache(_geometry(sva, F, Hp, Wp, H, d, n + 2))
    q, k, v, g = _inputs(n, T, H, d, has_q, packed)
    shape = {"shared": (d,), "heads": (H, d), "none": None}[gamma]
    gk = (torch.rand(shape, generator=g) + 0.5).cuda() if shape else None
    gq = (torch.rand(shape, generator=g) - 2.0).cuda() if shape and has_q else None
    pool = cache.slot_pool()
    pool.view(torch.int16)[:, :, :, :T] = 0x2A2A
    before = pool.clone()
    chunks = [3 + i for i in range(n)]
    nodes = [dict(seq=i % 2, chunk=c, level=1, own_slot=cache.bind(i % 2, c, 1)) for i, c in enumerate(chunks)]
    given = [t.clone() for t in (k, v)] + ([q.clone()] if has_q else [])
    q_out = torch.empty((n, T, H, d), dtype=torch.bfloat16, device="cuda") if has_q else None
    cache.rope_kv_write_headnorm(nodes, k, v, q, q_out, gk, gq, eps)
    for a, b in zip(given, [k, v] + ([q] if has_q else [])):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))       # inputs are only read
    written = set()
    for i, node in enumerate(nodes):
        s = node["own_slot"]
        written.add(s)
        ref, size = _ref(k[i].cpu(), gk, chunks[i], F, Hp, Wp, eps)
        _assert_rotated(pool[s, 0, :, :T].transpose(0, 1), ref, size, f"K of node {i}")
        assert torch.equal(pool[s, 1, :, :T].transpose(0, 1).contiguous().view(torch.int16),
                           v[i].contiguous().view(torch.int16))
        if has_q:
            ref, size = _ref(q[i].cpu(), gq, chunks[i], F, Hp, Wp, eps)
            _assert_rotated(q_out[i], ref, size, f"Q of node {i}")
    for s in range(n + 2):
        if s not in written:
            assert torch.equal(pool[s].view(torch.int16), before[s].view(torch.int16))
    assert torch.all(pool[:, :, :, T:] == 0)
    assert cache.poll() == sva.OK
    cache.close()


def test_in_place_strided_and_streams(sva_mod):
    """Dense q rotated in place gives the bits of q_out apart; k and v at strides of their own; a side stream."""
    sva, (F, Hp, Wp, H, d), n = sva_mod, (1, 7, 9, 6, 128), 2
    T = F * Hp * Wp
    cache = sva.Cache(_geometry(sva, F, Hp, Wp, H, d, n))
    q, k, v, g = _inputs(n, T, H, d, True, False)
    nodes = [dict(seq=0, chunk=2 + i, level=0, own_slot=cache.bind(0, 2 + i, 0)) for i in range(n)]
    q_out = torch.empty_like(q)
    cache.rope_kv_write_headnorm(nodes, k, v, q, q_out)
    want = cache.slot_pool().clone()
    wide_k = torch.zeros((n, T, 2 * H + 1, d), dtype=torch.bfloat16, device="cuda")
    wide_v = torch.zeros((n, T, H + 3, d), dtype=torch.bfloat16, device="cuda")
    wide_k[:, :, 1:H + 1], wide_v[:, :, 3:] = k, v
    cache.slot_pool()[:, :, :, :T] = 0
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    cache.rope_kv_write_headnorm(nodes, wide_k[:, :, 1:H + 1], wide_v[:, :, 3:], q, stream=side)
    side.synchronize()
    assert torch.equal(q.view(torch.int16), q_out.view(torch.int16))
    assert torch.equal(cache.slot_pool().view(torch.int16), want.view(torch.int16))
    cache.close()


def test_whole_row_norm_is_the_one_head_case(sva_mod):
    """With one head the norm over H*d is the norm of the head: same bits as sva_rope_kv_write_qknorm."""
    sva, (F, Hp, Wp, H, d) = sva_mod, (2, 5, 9, 1, 128)
    cache = sva.Cache(_geometry(sva, F, Hp, Wp, H, d, 1))
    q, k, v, g = _inputs(1, F * Hp * Wp, H, d, True, False)
    gk, gq = (torch.rand(d, generator=g) + 0.5).cuda(), (torch.rand(d, generator=g) + 0.5).cuda()
    nodes = [dict(seq=0, chunk=4, level=0, own_slot=cache.bind(0, 4, 0))]
    q2 = q.clone()
    cache.rope_kv_write_headnorm(nodes, k, v, q, None, gk, gq)
    a = cache.slot_pool().float()
    cache.rope_kv_write_qknorm(nodes, k, v, q2, gk, gq)
    b = cache.slot_pool().float()
    # the two sum the squares in different orders: a value may fall on the other side of a rounding
    assert float(((a - b).abs() > 2.0 ** -7 * b.abs()).float().mean()) == 0.0
    assert float((a != b).float().mean()) < 1e-3
    assert float((q.float() - q2.float()).abs().max()) <= 2.0 ** -7 * float(q2.float().abs().max())
    cache.close()


def test_attends_over_what_it_wrote(sva_mod):
    """The written state is resident and read by the attention like any other."""
    sva, (F, Hp, Wp, H, d) = sva_mod, (1, 5, 8, 2, 64)
    T = F * Hp * Wp
    cache = sva.Cache(_geometry(sva, F, Hp, Wp, H, d, 2))
    q, k, v, g = _inputs(1, T, H, d, True, True)
    node = dict(seq=0, chunk=1, level=0, own_slot=cache.bind(0, 1, 0))
    out, q_out = torch.empty((1, T, H, d), dtype=torch.bfloat16, device="cuda"), torch.empty((1, T, H, d), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(sva.SvaError) as e:
        cache.attend_nodes([node], out, out)
    assert e.value.status == sva.ERR_NOT_RESIDENT
    cache.rope_kv_write_headnorm([node], k, v, q, q_out)
    cache.attend_nodes([node], q_out, out)
    kk, vv = cache.slot_pool()[0, 0, :, :T].double(), cache.slot_pool()[0, 1, :, :T].double()
    p = torch.softmax(torch.einsum("uhd,hvd->huv", q_out[0].double(), kk) / math.sqrt(d), -1)
    ref = torch.einsum("huv,hvd->uhd", p, vv)
    # bf16 weights and output: 2^-8 of sum p |v| each, and as much again for fp32 sums
    bound = 2.0 ** -7 * torch.einsum("huv,hvd->uhd", p, vv.abs()) + 1e-3
    assert torch.all((out[0].double() - ref).abs() <= bound)
    cache.close()


def test_refusals(sva_mod):
    sva, (F, Hp, Wp, H, d) = sva_mod, (1, 4, 4, 2, 64)
    T = 16
    cache = sva.Cache(_geometry(sva, F, Hp, Wp, H, d, 2, max_frames=8))
    q, k, v, _ = _inputs(1, T, H, d, True, True)
    slot = cache.bind(0, 1, 0)
    node = dict(seq=0, chunk=1, level=0, own_slot=slot)
    q_out = torch.empty((1, T, H, d), dtype=torch.bfloat16, device="cuda")
    cache.slot_pool().view(torch.int16)[:, :, :, :T] = 0x1234
    before = cache.slot_pool().clone()
    gd, gh = torch.ones(d, device="cuda"), torch.ones((H, d), device="cuda")

    def status(*a, **kw):
        with pytest.raises(sva.SvaError) as e:
            cache.rope_kv_write_headnorm(*a, **kw)
        return e.value.status

    def rejected(*a, **kw):
        with pytest.raises(ValueError):
            cache.rope_kv_write_headnorm(*a, **kw)

    assert status([node], k, v, q, q_out, eps=0.0) == sva.ERR_INVALID_ARGUMENT
    assert status([node], k, v, q, q_out, eps=math.nan) == sva.ERR_INVALID_ARGUMENT
    assert status([node], k, v, q, q_out, gd, None) == sva.ERR_INVALID_ARGUMENT
    assert status([dict(node, own_slot=1)], k, v) == sva.ERR_INVALID_ARGUMENT
    assert status([dict(node, chunk=2)], k, v) == sva.ERR_INVALID_ARGUMENT
    far = cache.bind(0, 8, 0)
    assert status([dict(seq=0, chunk=8, level=0, own_slot=far)], k, v) == sva.ERR_CAPACITY
    two = torch.cat([k, k])
    assert status([node, node], two, two) == sva.ERR_INVALID_ARGUMENT      # one slot written twice
    rejected([node], k, v, q)                                               # packed q cannot be rotated in place
    rejected([node], k.float(), v)
    rejected([node], k[:, :8], v)
    rejected([node], k.transpose(2, 3).contiguous().transpose(2, 3), v)     # d not dense
    rejected([node], k, v, q, q_out, gh[:, :32].contiguous(), None)
    rejected([node], k, v, q, q_out, gd, gh)
    rejected([node], k, v, None, q_out)
    # through the C call: what the binding cannot express
    import ctypes
    lib = sva.load()
    arr = sva.make_nodes([node])

    def raw(kd, ks, qd=None, qs=0, out=None, heads=1, count=1):
        rk, rq = sva.sva_token_rows(kd, ks), sva.sva_token_rows(qd, qs)
        return lib.sva_rope_kv_write_headnorm(cache.handle, arr, count, ctypes.byref(rk), ctypes.byref(rk),
                                              ctypes.byref(rq) if qd else None, out, None, None, heads, 1e-6, None)

    kd = k.contiguous().data_ptr()
    assert raw(None, H * d) == sva.ERR_INVALID_ARGUMENT
    assert raw(kd + 2, H * d) == sva.ERR_INVALID_ARGUMENT
    assert raw(kd, H * d - 8) == sva.ERR_INVALID_ARGUMENT
    assert raw(kd, H * d + 4) == sva.ERR_INVALID_ARGUMENT
    assert raw(kd, -H * d) == sva.ERR_INVALID_ARGUMENT
    assert raw(kd, H * d, heads=3) == sva.ERR_INVALID_ARGUMENT
    assert raw(kd, H * d, count=0) == sva.ERR_INVALID_ARGUMENT
    assert raw(kd, H * d, count=65) == sva.ERR_CAPACITY
    assert raw(kd, H * d, qd=q_out.data_ptr(), qs=H * d) == sva.ERR_INVALID_ARGUMENT        # q without q_out
    assert raw(kd, H * d, out=q_out.data_ptr()) == sva.ERR_INVALID_ARGUMENT                 # q_out without q
    base = q.data_ptr()
    assert raw(k.data_ptr(), 3 * H * d, qd=base, qs=3 * H * d, out=base) == sva.ERR_INVALID_ARGUMENT   # in place, packed
    assert raw(q_out.data_ptr(), H * d, qd=base, qs=3 * H * d, out=q_out.data_ptr()) == sva.ERR_INVALID_ARGUMENT  # over k
    torch.cuda.synchronize()
    assert torch.equal(cache.slot_pool().view(torch.int16), before.view(torch.int16))       # nothing was launched
    cache.close()

"""Shared helpers of the tests of packed slots: what 4 bits hold, written from its definition in 64 bits, and caches
whose states are known."""
import math

import torch


def held(x):
    """The values that a packed slot holds for x [..., d] (bf16): groups of 32, scale max|x| / 7 to 5 significant
    bits (halves up), whole numbers x / scale (halves away from zero).  In 64 bits, by comparisons with the half-way
    marks instead of a division."""
    g = x.double().unflatten(-1, (-1, 32))
    a = g.abs().amax(-1, keepdim=True)
    lost = ~(a < 2.0 ** 124)
    small = a < 2.0 ** -120
    safe = torch.where(lost | small, 1.0, a)
    unit = torch.exp2(torch.floor(torch.log2(safe / 7)) - 4)     # one step of the fifth bit
    s = torch.floor(safe / 7 / unit + 0.5) * unit
    k = sum((2 * g.abs() >= (2 * j - 1) * s).double() for j in range(1, 8))
    v = torch.where(small, 0.0, torch.copysign(k, g) * s)
    return torch.where(lost, math.nan, v).flatten(-2)


def pairs(d):
    return (d // 2 - 2 * (d // 6), d // 6, d // 6)


def make_cache(sva, F, Hp, Wp, H, d, slots, packed, workspace=True, chunks=40):
    g = sva.make_geometry(H, d, F, Hp, Wp, num_slots=slots, pairs=pairs(d), max_frames=F * (chunks + 2))
    c = sva.Cache(g)
    if workspace:
        c.set_workspace(torch.empty(c.workspace_bytes(), dtype=torch.uint8, device="cuda"))
    if packed:
        # rubbish, as a caller's buffer has it
        c.set_packed(torch.randint(0, 256, (sva.packed_bytes(g, packed),), dtype=torch.uint8, device="cuda"), packed)
    return c


def write(c, state, kv):
    """Binds a slot to `state` and fills it with kv [2][H][T][d] as it is (no rotation)."""
    p = c.bind(*state)
    blank = torch.zeros((1, c.T, c.H, c.d), dtype=torch.bfloat16, device="cuda")
    c.rope_kv_write([dict(seq=state[0], chunk=state[1], level=state[2], own_slot=p)], blank, blank)
    c.slot_pool()[p, :, :, : c.T] = kv
    return p


def random_kv(c, gen, spread=0.5):
    scale = torch.exp(spread * torch.randn((2, c.H, 1, c.d), generator=gen, device="cuda"))
    return (torch.randn((2, c.H, c.T, c.d), generator=gen, device="cuda") * scale).bfloat16()


def status(fn):
    try:
        fn()
    except Exception as e:  # SvaError
        return getattr(e, "status", None)
    return 0


def attention(q, k, v, keep=None, scale=None):
    """out, lse, and the two parts of a tolerance: E_p|V| and the largest sum of |products| of a logit, in 64 bits.
    q [T][d], k, v [keys][d]; a query that keep leaves nothing gets 0 and -inf."""
    scale = 1 / math.sqrt(q.shape[1]) if scale is None else scale
    x = q.double() @ k.double().t() * scale
    big = (q.double().abs() @ k.double().abs().t()).amax() * scale
    if keep is not None:
        x = x.masked_fill(~keep, -math.inf)
    lse = torch.logsumexp(x, 1)
    p = torch.softmax(x, 1).nan_to_num(0.0)
    return p @ v.double(), lse, p @ v.double().abs(), big


def assert_attention(out, lse, ref, what=""):
    """out, lse of one (node, head) against attention(...).  A logit is off by at most (d + 16) 2^-24 of the sum of
    its |products| (fp32 sums of exact products, the scale's rounding), exponentials, the logarithm and the scale in
    base 2 by 2^-18 (1 + |lse|) together; that moves a weight by twice as much relative to it.  P and the output are
    each rounded to bf16 once: 2^-8."""
    o, l, ev, big = ref
    d = o.shape[1]
    t = (d + 16) * 2.0 ** -24 * big + 2.0 ** -18 * (1 + l.abs().nan_to_num(posinf=0.0))
    fine = torch.isfinite(l)
    assert torch.equal(fine, torch.isfinite(lse.double())), what
    assert ((lse.double() - l).abs()[fine] <= t[fine]).all(), (what, (lse.double() - l).abs()[fine].max())
    assert (out[~fine] == 0).all() and (lse[~fine] == -math.inf).all(), what
    bound = 2.0 ** -8 * o.abs() + (2.0 ** -8 * (1 + 2.0 ** -8) + 2 * t[:, None]) * ev + 1e-30
    bad = (out.double() - o).abs() > bound
    assert not bad[fine].any(), (what, int(bad.sum()), ((out.double() - o).abs() / bound).max())

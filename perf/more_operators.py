"""States held in 4 bits and states moved between slots, as measurable cases, in a plain form and in the library's.

A program that keeps a long history of a video holds its newer states whole (bf16) and its older ones
in 4 bits:

  park      puts whole states into packed slots (pack), and reads what these hold back into whole
            slots (unpack), which is where one sees the values that the 4 bits stand for;
  fetch     reads packed states back into whole slots (unpack), say before they are condensed;
  attend    attends over states of both kinds (attend_nodes_packed), with any of the attention's masks;
  copy      copies states to other slots, when a video branches (copy).

What 4 bits hold: each group of 32 neighbouring elements of a head's row has a scale s, its largest
magnitude / 7 rounded to 5 significant bits (halves up), and each element a whole number from -7 to 7,
x / s rounded to the nearest (halves away from zero).  A group with nothing of 2^-120 or more is
zeros.  Every value, number times scale, is a bf16 number.

The sizes are those of the repository's workloads (chunks of 3 latent frames of 30 x 52 patches, 12
or 40 heads of 128; tiny test chunks) and generic ones between them.
"""
from __future__ import annotations

import math

import torch

own = False      # False: the plain forms below; True: the library's calls

LEVELS = 4       # denoising levels of the pipelines (level 0 = clean)
GROUP = 32       # elements that share a scale
DEV = "cuda"


def _case(name=None, **kw):
    """A case with every field set.

    kind       "park", "fetch", "copy", "attend"
    F,Hp,Wp    latent frames of a chunk, patch rows and columns of a frame;  H,d: heads, head dimension
    n          park, fetch, copy: states
    streams    independent videos, `nodes` nodes (consecutive levels of one pipeline round) in each
    W          history chunks a node reads;  policy "clean", "same" or "prog"
    recent     history chunks that are held whole: older ones are packed, the round's own never
    causal     frame-causal inside the own chunk
    mask       "", "tiles" (each block of `span` query tiles keeps its own chunk and a share `keep`
               of the history's 128-key tiles), "local" (token masks: a query sees keys within
               `span` patch rows and columns), "random" (token masks: half of the keys); under the
               token masks a few queries see nothing at all
    """
    c = dict(kind="attend", F=3, Hp=30, Wp=52, H=12, d=128, n=1, streams=1, nodes=1, W=3, policy="clean", recent=0,
             causal=False, mask="", span=0, keep=1.0)
    c.update(kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # Four single-frame low-resolution states of an interactive session: latency.
        _case("park small", kind="park", F=1, Hp=16, Wp=20, n=4),
        # The history window of the 12-head model, six full-size states.
        _case("park window", kind="park", n=6),
        # One full-size state of the 12-head model, brought back alone.
        _case("fetch chunk", kind="fetch"),
        # Seven full-size states of the 40-head model.
        _case("fetch large", kind="fetch", H=40, n=7),
        # A small session branches: four states to slots of another sequence.
        _case("copy small", kind="copy", F=1, Hp=16, Wp=20, n=4),
        # A full-size window branches.
        _case("copy window", kind="copy", n=6),
        # The repository's tiny workload: two nodes of 64 tokens, two heads of 64.
        _case("attend tiny", F=1, Hp=8, Wp=8, H=2, d=64, nodes=2, W=2, policy="prog"),
        # Few queries over the longest history: one small frame, 40 heads, sixteen packed states.
        _case("attend long", F=1, Hp=16, Wp=20, H=40, W=16),
        # One denoising update on clean history, a full-size chunk over 18720 keys, three of four states packed.
        _case("attend serial"),
        # A pipeline round: four nodes over 32760 keys each, the newest clean state whole.
        _case("attend round", nodes=4, W=6, policy="prog", recent=1),
        # 64-wide heads, mid-size chunks, two nodes with clean history.
        _case("attend narrow", Hp=20, Wp=36, H=16, d=64, nodes=2, W=4),
        # Token masks: spatially local attention, some queries with nothing to see.
        _case("attend local", mask="local", span=6),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = max(work(c)["flops"] for c in listed())
    while True:
        kind = rng.choice(["park", "fetch", "copy", "attend", "attend", "attend"])
        c = _case(kind=kind, F=rng.randint(1, 4), Hp=_log(rng, 1, 40), Wp=_log(rng, 1, 60), H=_log(rng, 1, 40),
                  d=rng.choice([64, 128, 128]))
        if kind == "attend":
            c.update(streams=rng.choice([1, 1, 1, 2]), nodes=rng.randint(1, 4), W=rng.randint(1, 16),
                     policy=rng.choice(["clean", "same", "prog"]), recent=rng.choice([0, 0, 1, 2]),
                     causal=rng.random() < 0.25, mask=rng.choice(["", "", "", "tiles", "local", "random"]))
            if c["mask"] == "tiles":
                c["span"], c["keep"] = rng.choice([1, 2, 2, 4]), round(rng.uniform(0.1, 0.9), 2)
            if c["mask"] == "local":
                c["span"] = rng.randint(2, 10)
            if c["mask"] in ("local", "random"):
                c["streams"] = 1
            if (1 + c["W"]) * -(-_tokens(c) // 128) > 4096 and c["mask"]:
                continue
        else:
            c["n"] = _log(rng, 1, 16)
        if work(c)["flops"] <= most and work(c)["bytes"] <= 1.2e9:
            return c


# ------------------------------------------------------------------ the round

def _tokens(c):
    return c["F"] * c["Hp"] * c["Wp"]


def _pairs(d):
    hw = d // 6
    return (d // 2 - 2 * hw, hw, hw)


def _round(c):
    """[(node, its history states)] in order, states as (seq, chunk, level)."""
    last = c["W"] + c["nodes"]
    phi = {"clean": lambda j, r: 0, "same": lambda j, r: j, "prog": lambda j, r: max(j - r, 0)}[c["policy"]]
    out = []
    for s in range(c["streams"]):
        for i in range(c["nodes"]):
            b, j = last - i, LEVELS - i
            out.append(((s, b, j), [(s, b - r, phi(j, r)) for r in range(1, min(c["W"], b - 1) + 1)]))
    return out


def _states(c):
    """The states that are whole (the nodes' own ones first), the packed ones after them, and how many are whole."""
    if c["kind"] != "attend":
        return [(0, 1 + i, 0) for i in range(c["n"])], c["n"]
    own_states = [n for n, _ in _round(c)]
    seen = set(own_states)
    other = []
    for _, ctx in _round(c):
        for s in ctx:
            if s not in seen:
                seen.add(s)
                other.append(s)
    line = c["W"] - c["recent"]
    whole = own_states + [s for s in other if s[1] > line]
    return whole + [s for s in other if s[1] <= line], len(whole)


def _pack_bits(keep):
    """bool [..., n] -> int32 [..., ceil(n / 32)], bit k % 32 of word k // 32."""
    n = keep.shape[-1]
    words = -(-n // 32)
    k = torch.zeros(keep.shape[:-1] + (words * 32,), dtype=torch.bool, device=keep.device)
    k[..., :n] = keep
    v = (k.view(keep.shape[:-1] + (words, 32)).long() << torch.arange(32, device=keep.device)).sum(-1)
    return torch.where(v >= 2 ** 31, v - 2 ** 32, v).to(torch.int32)


def _unpack_bits(words, n):
    b = (words.unsqueeze(-1) >> torch.arange(32, device=words.device, dtype=torch.int32)) & 1
    return b.reshape(words.shape[:-1] + (-1,))[..., :n].bool()


def _near(n, span):
    i = torch.arange(n)
    return (i[:, None] - i[None, :]).abs() <= span


class _State:
    pass


def _inputs(c, seed):
    """What the call takes, from the seed alone: tensors on the GPU.  kv: the states' K and V [2][H][T][d],
    as the cache holds them (the packed ones before they are packed)."""
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    T, H, d = _tokens(c), c["H"], c["d"]
    i = _State()
    i.states, i.whole = _states(c)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV)

    # channels of different sizes, as projections have them, and a row that is all zeros
    scale = torch.exp(0.4 * normal(2, H, 1, d))
    i.kv = torch.empty((len(i.states), 2, H, T, d), dtype=torch.bfloat16, device=DEV)
    for kv in i.kv:
        kv.copy_(normal(2, H, T, d) * scale)
    i.kv[:, :, 0, T // 2] = 0
    if c["kind"] != "attend":
        i.order = torch.randperm(c["n"], generator=g, device=DEV)
        return i
    n, W, nt = len(_round(c)), c["W"], -(-T // 128)
    i.q = normal(n, T, H, d).to(torch.bfloat16)
    i.tile = i.tok_own = i.tok_hist = None
    if c["mask"] == "tiles":
        keep = torch.rand((n, -(-nt // c["span"]), (1 + W) * nt), generator=g, device=DEV) < c["keep"]
        keep = keep.repeat_interleave(c["span"], dim=1)[:, :nt]
        keep[:, :, :nt] = True
        i.tile = _pack_bits(keep)
    elif c["mask"]:
        if c["mask"] == "local":
            h, w = _near(c["Hp"], c["span"]).to(DEV), _near(c["Wp"], c["span"]).to(DEV)
            m = (h[:, None, :, None] & w[None, :, None, :]).reshape(c["Hp"] * c["Wp"], -1).repeat(c["F"], c["F"])
            m = _pack_bits(m)
            i.tok_own = m.expand(n, T, -1).contiguous()
            i.tok_hist = m[None, :, None].expand(n, T, W, -1).contiguous()
        else:
            def bits(*shape):
                return torch.randint(-2 ** 31, 2 ** 31, shape, generator=g, device=DEV, dtype=torch.int64).to(torch.int32)
            i.tok_own, i.tok_hist = bits(n, T, -(-T // 32)), bits(n, T, W, -(-T // 32))
        i.tok_own[:, 7::997] = 0      # queries that see nothing
        i.tok_hist[:, 7::997] = 0
    return i


def _keep(c, i, n, states):
    """bool [T][states * T]: which keys of its first `states` states (its own first) node n's queries see; None: all."""
    T, nt = _tokens(c), -(-_tokens(c) // 128)
    keep = None
    if i.tile is not None:
        k = _unpack_bits(i.tile[n], states * nt).repeat_interleave(128, 0)[:T].view(T, states, nt)
        keep = k.repeat_interleave(128, 2)[:, :, :T].reshape(T, states * T)
    elif i.tok_own is not None:
        k = torch.cat((i.tok_own[n][:, None], i.tok_hist[n, :, :states - 1]), dim=1)
        keep = _unpack_bits(k, T).reshape(T, states * T)
    if c["causal"]:
        f = torch.arange(T, device=DEV) // (c["Hp"] * c["Wp"])
        past = torch.ones((T, states * T), dtype=torch.bool, device=DEV)
        past[:, :T] = f[:, None] >= f[None, :]
        keep = past if keep is None else keep & past
    return keep


def prepare(case, seed):
    """A layer's cache with its history, the round's node table, the inputs and the output buffers."""
    c, s = case, _inputs(case, seed)
    s.c = c
    T, H, d = _tokens(c), c["H"], c["d"]
    if not own:
        if c["kind"] == "copy":      # a pool of slots: the states in order, and as many free slots
            s.pool = torch.cat((s.kv, torch.zeros_like(s.kv)))
            s.src, s.dst = s.order, torch.arange(c["n"], 2 * c["n"], device=DEV)
        elif c["kind"] == "fetch":
            s.codes, s.scales = _quantised(s.kv)
        elif c["kind"] == "attend":
            s.codes, s.scales = _quantised(s.kv[s.whole:])
            s.at = [[s.states.index(t) for t in [st] + ctx] for st, ctx in _round(c)]
        return s
    from paper_2609_22283_gb300 import sva
    top = max(b for _, b, _ in s.states)
    packed_n = len(s.states) - s.whole if c["kind"] == "attend" else (0 if c["kind"] == "copy" else len(s.states))
    slots = s.whole + 1 if c["kind"] == "attend" else 2 * len(s.states)
    geo = sva.make_geometry(H, d, c["F"], c["Hp"], c["Wp"], num_slots=slots, pairs=_pairs(d),
                            max_frames=c["F"] * (top + 2))
    s.cache = sva.Cache(geo, device=torch.device(DEV))
    s.cache.set_workspace(torch.empty(s.cache.workspace_bytes(), dtype=torch.uint8, device=DEV))
    if packed_n:
        s.cache.set_packed(torch.empty(sva.packed_bytes(geo, packed_n), dtype=torch.uint8, device=DEV), packed_n)
    pool = s.cache.slot_pool()
    blank = torch.zeros((1, T, H, d), dtype=torch.bfloat16, device=DEV)

    def hold(k):      # state k in a slot, as an earlier run left it: marked written, then its very values restored
        q, b, j = s.states[k]
        p = s.cache.bind(q, b, j)
        s.cache.rope_kv_write([dict(seq=q, chunk=b, level=j, own_slot=p)], blank, blank)
        pool[p, :, :, :T] = s.kv[k]
        return p

    def park(k, p):
        x = s.cache.bind_packed(*s.states[k])
        s.cache.pack([p], [x])
        return x

    if c["kind"] == "attend":
        at = {}
        for k, st in enumerate(s.states):
            at[st] = hold(k)
            if k >= s.whole:
                at[st], p = park(k, at[st]), at[st]
                s.cache.release(*st)
        within = sva.WITHIN_FRAME_CAUSAL if c["causal"] else sva.WITHIN_BIDIRECTIONAL
        s.nodes = sva.make_nodes([dict(seq=st[0], chunk=st[1], level=st[2], own_slot=at[st], ctx=[at[t] for t in ctx],
                                       within=within) for st, ctx in _round(c)])
        s.out = torch.empty_like(s.q)
        s.lse = torch.empty((len(_round(c)), H, T), device=DEV)
        return s
    s.slots = [hold(k) for k in range(c["n"])]
    if c["kind"] == "copy":      # the same states of another sequence
        s.src = [s.slots[k] for k in s.order.tolist()]
        s.to = [s.cache.bind(1, s.states[k][1], 0) for k in s.order.tolist()]
    else:                        # where they are read back to
        s.packed = [s.cache.bind_packed(*st) if c["kind"] == "park" else park(k, s.slots[k])
                    for k, st in enumerate(s.states)]
        s.to = [s.cache.bind(q, b, LEVELS + 1) for q, b, _ in s.states]
    s.outs = [pool[p, :, :, :T] for p in s.to]
    return s


def run(state):
    s, c = state, state.c
    if own:
        if c["kind"] == "attend":
            s.cache.attend_nodes_packed(s.nodes, s.q, s.out, s.lse, tile_mask=s.tile, own_mask=s.tok_own,
                                        hist_mask=s.tok_hist)
            return [s.out, s.lse]
        if c["kind"] == "copy":
            s.cache.copy(s.src, s.to)
            return s.outs
        if c["kind"] == "park":
            s.cache.pack(s.slots, s.packed)
        s.cache.unpack(s.packed, s.to)
        return s.outs
    if c["kind"] == "attend":
        return _plain_attend(s, c)
    if c["kind"] == "copy":
        s.pool[s.dst] = s.pool[s.src]
        return list(s.pool[c["n"]:])
    return list(_values(*(_quantised(s.kv) if c["kind"] == "park" else (s.codes, s.scales))).to(torch.bfloat16))


# ------------------------------------------------------------------ the plain forms

def _quantised(x):
    """bf16 [..., d] -> whole numbers (int8) [..., d / 32][32] and scales (fp32) [..., d / 32][1].  In 32 bits: a
    bf16 number by 7, or by a scale of 5 bits, is either half-way between two results or further from it than
    2^-13 of the result."""
    x = x.unflatten(-1, (-1, GROUP)).float()
    a = x.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(a / 7)
    s = torch.ldexp(torch.floor(m * 32 + 0.5), e - 5)
    s = torch.where(a < 2.0 ** -120, 0.0, s)
    k = torch.where(s > 0, torch.floor(x.abs() / s + 0.5) * torch.sign(x), 0.0)
    return k.to(torch.int8), s


def _values(codes, scales):
    return (codes * scales).flatten(-2)


def _plain_attend(s, c):
    T, H, d = _tokens(c), c["H"], c["d"]
    kv = torch.cat((s.kv[:s.whole].float(), _values(s.codes, s.scales)))
    out = torch.empty_like(s.q)
    lse = torch.empty((len(s.at), H, T), device=DEV)
    for n, at in enumerate(s.at):
        k, v = kv[at].permute(1, 2, 0, 3, 4).reshape(2, H, len(at) * T, d)
        x = (s.q[n].float().transpose(0, 1) @ k.transpose(1, 2)).mul_(1 / math.sqrt(d))
        keep = _keep(c, s, n, len(at))
        if keep is not None:
            x.masked_fill_(~keep, -math.inf)
        m = x.amax(-1, keepdim=True).clamp_(min=-3e38)      # a query that sees nothing: 0, and -inf
        p = x.sub_(m).exp_()
        z = p.sum(-1, keepdim=True)
        out[n] = ((p @ v) / z.clamp(min=1e-30)).transpose(0, 1)
        lse[n] = (m + z.log())[..., 0]
    return [out, lse]


# ------------------------------------------------------------------ work

def _visible(c):
    """(query, key) pairs that may attend, over all nodes and one head."""
    T, F, hw = _tokens(c), c["F"], c["Hp"] * c["Wp"]
    near = 1.0
    if c["mask"] == "random":
        near = 0.5
    elif c["mask"] == "local":
        near = float(_near(c["Hp"], c["span"]).double().mean() * _near(c["Wp"], c["span"]).double().mean())
    keep = c["keep"] if c["mask"] == "tiles" else 1.0
    inside = (hw * hw * F * (F + 1) / 2 if c["causal"] else T * T) * near
    return sum(inside + len(ctx) * T * T * near * keep for _, ctx in _round(c))


def work(case):
    c = case
    T, H, d = _tokens(c), c["H"], c["d"]
    whole, packed = 2 * 2.0 * T * H * d, 2 * (0.5 + 2.0 / GROUP) * T * H * d      # bytes of a state
    if c["kind"] == "park":      # read, held, read back, written
        return {"bytes": c["n"] * 2 * (whole + packed), "flops": 4.0 * c["n"] * 2 * T * H * d}
    if c["kind"] == "fetch":
        return {"bytes": c["n"] * (whole + packed), "flops": 1.0 * c["n"] * 2 * T * H * d}
    if c["kind"] == "copy":
        return {"bytes": c["n"] * 2 * whole, "flops": 0.0}
    states, n_whole = _states(c)
    nodes = len(_round(c))
    by = n_whole * whole + (len(states) - n_whole) * packed + nodes * T * H * (4.0 * d + 4)
    if c["mask"] in ("local", "random"):
        by += nodes * T * T / 8 + sum(T * T * len(ctx) / 8 for _, ctx in _round(c))
    return {"bytes": by, "flops": 4.0 * _visible(c) * H * d}


# ------------------------------------------------------------------ in 64 bits

def _held(x):
    """What 4 bits hold of x, in 64 bits: the scale by its own exponent, each number by the half-way marks below it."""
    x = x.double().unflatten(-1, (-1, GROUP))
    a = x.abs().amax(-1, keepdim=True)
    step = torch.exp2(torch.floor(torch.log2(torch.where(a > 0, a, 1.0) / 7)) - 4)
    s = torch.floor(a / 7 / step + 0.5) * step * (a >= 2.0 ** -120)
    k = sum((2 * x.abs() >= (2 * j - 1) * s).double() for j in range(1, 8)) * (s > 0)
    return (torch.copysign(k, x) * s).flatten(-2)


def exact(case, seed):
    c, i = case, _inputs(case, seed)
    T, H, d = _tokens(c), c["H"], c["d"]
    if c["kind"] == "copy":
        return [i.kv[k].double() for k in i.order.tolist()]
    if c["kind"] != "attend":
        return [_held(kv) for kv in i.kv]
    if work(c)["flops"] > 4e12:
        return None
    at = [[i.states.index(t) for t in [st] + ctx] for st, ctx in _round(c)]
    out = torch.zeros((len(at), T, H, d), dtype=torch.float64, device=DEV)
    lse = torch.zeros((len(at), H, T), dtype=torch.float64, device=DEV)
    for n, see in enumerate(at):
        keep = _keep(c, i, n, len(see))
        for h in range(H):
            k, v = (torch.cat([i.kv[t, x, h].double() if t < i.whole else _held(i.kv[t, x, h]) for t in see])
                    for x in (0, 1))
            for r in range(0, T, 2048):
                x = torch.einsum("ud,vd->uv", i.q[n, r:r + 2048, h].double(), k) / math.sqrt(d)
                if keep is not None:
                    x[~keep[r:r + 2048]] = -math.inf
                lse[n, h, r:r + 2048] = torch.logsumexp(x, dim=1)
                p = torch.softmax(x, dim=1).nan_to_num_(0.0)      # a row of -inf has no softmax
                out[n, r:r + 2048, h] = p @ v
    return [out, lse]

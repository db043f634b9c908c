"""The cache operators of a long stream, as measurable cases, in a plain form and in the library's.

A program that streams video for longer than its cache lasts does, per layer and round:

  write     normalises each head's queries and keys, rotates them at their (t, h, w) positions and
            puts K' and V into the new states' slots (rope_kv_write_headnorm).  q, k and v lie
            where the projection left them: in tensors of their own, or side by side in one;
  weights   after the attention (whose log-sum-exps it has), adds up how much attention each cached
            key got from the round's queries (attend_weights), with the attention's own masks;
  condense  now and then keeps, of several old states, the tokens that got the most attention, head
            by head, in one state, and lets the others go (condense).

The sizes are those of the repository's workloads (chunks of 3 latent frames of 30 x 52 patches, 12
or 40 heads of 128; tiny test chunks) and generic ones between them.
"""
from __future__ import annotations

import math

import torch

own = False      # False: the plain forms below; True: the library's calls

LEVELS = 4       # denoising levels of the pipelines (level 0 = clean)
EPS = 1e-6
THETA = 10000.0
DEV = "cuda"


def _case(name=None, **kw):
    """A case with every field set.

    kind       "write", "weights", "condense"
    F,Hp,Wp    latent frames of a chunk, patch rows and columns of a frame;  H,d: heads, head dimension
    streams    independent videos, `nodes` nodes (consecutive levels of one pipeline round) in each
    W          history chunks a node reads;  policy "clean", "same" or "prog"
    causal     frame-causal inside the own chunk
    mask       "", "tiles" (each block of `span` query tiles keeps its own chunk and a share `keep`
               of the history's 128-key tiles), "local" (token masks: a query sees keys within
               `span` patch rows and columns), "random" (token masks: half of the keys); under the
               token masks a few queries see nothing at all
    decay      of the weights before: 0 means there are none yet
    q          write: queries too;  packed: q, k, v side by side per token
    gamma      write: "shared" (one [d] vector), "heads" ([H][d]) or "none"
    src        condense: states that become one;  zeros: share of their tokens that nothing attended
    """
    c = dict(kind="weights", F=3, Hp=30, Wp=52, H=12, d=128, streams=1, nodes=1, W=3, policy="prog", causal=False,
             mask="", span=0, keep=1.0, decay=0.9, q=True, packed=True, gamma="shared", src=4, zeros=0.1)
    c.update(kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # A single-frame low-resolution chunk of an interactive session: latency.
        _case("write small", kind="write", F=1, Hp=16, Wp=20),
        # One full-size chunk of the 12-head model, q, k and v side by side as one projection left them.
        _case("write chunk", kind="write"),
        # A pipeline round of four such chunks from tensors of their own, norm weights for each head.
        _case("write round", kind="write", nodes=4, packed=False, gamma="heads"),
        # The clean-state refresh of a 40-head model: keys and values only.
        _case("write refresh", kind="write", H=40, q=False),
        # The repository's tiny workload: two nodes of 64 tokens, two heads of 64.
        _case("weights tiny", F=1, Hp=8, Wp=8, H=2, d=64, nodes=2, W=2, decay=0.0),
        # One denoising update on clean history, a full-size chunk over 18720 keys.
        _case("weights serial", policy="clean"),
        # A pipeline round: four nodes over 32760 keys each.
        _case("weights round", nodes=4, W=6),
        # 64-wide heads, mid-size chunks, two nodes with same-level history.
        _case("weights narrow", Hp=20, Wp=36, H=16, d=64, nodes=2, W=4, policy="same"),
        # Token masks: spatially local attention, some queries with nothing to see.
        _case("weights local", mask="local", span=6),
        # Four small states into one: latency.
        _case("condense small", kind="condense", F=1, Hp=16, Wp=20),
        # Six full-size states of the 12-head model into one.
        _case("condense chunks", kind="condense", src=6),
        # Seven states of the 40-head model, most tokens of which nothing attended (ties at zero).
        _case("condense large", kind="condense", H=40, src=7, zeros=0.9),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = max(work(c)["flops"] for c in listed())
    while True:
        kind = rng.choice(["write", "weights", "weights", "condense"])
        c = _case(kind=kind, F=rng.randint(1, 4), Hp=_log(rng, 1, 40), Wp=_log(rng, 1, 60), H=_log(rng, 1, 40),
                  d=rng.choice([64, 128, 128]))
        if kind == "write":
            c.update(streams=rng.choice([1, 1, 2]), nodes=rng.randint(1, 4), q=rng.random() < 0.7,
                     packed=rng.random() < 0.5, gamma=rng.choice(["shared", "heads", "none"]))
        elif kind == "condense":
            c.update(src=rng.randint(1, 16), zeros=rng.choice([0.0, 0.1, 0.5, 0.95]))
        else:
            c.update(streams=rng.choice([1, 1, 1, 2]), nodes=rng.randint(1, 4), W=rng.randint(0, 6),
                     policy=rng.choice(["clean", "same", "prog"]), causal=rng.random() < 0.25,
                     mask=rng.choice(["", "", "", "tiles", "local", "random"]), decay=rng.choice([0.0, 0.5, 1.0]))
            if c["mask"] == "tiles":
                c["span"], c["keep"] = rng.choice([1, 2, 2, 4]), round(rng.uniform(0.1, 0.9), 2)
            if c["mask"] == "local":
                c["span"] = rng.randint(2, 10)
            if c["mask"] in ("local", "random"):
                c["streams"] = 1
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
    """The nodes' own states, then the other states they read."""
    if c["kind"] == "condense":
        return [(0, 1 + i, 0) for i in range(c["src"])]
    own_states = [n for n, _ in _round(c)]
    other = []
    if c["kind"] == "weights":
        for _, ctx in _round(c):
            other += [s for s in ctx if s not in own_states and s not in other]
    return own_states + other


def _pack(keep):
    """bool [..., n] -> int32 [..., ceil(n / 32)], bit k % 32 of word k // 32."""
    n = keep.shape[-1]
    words = -(-n // 32)
    k = torch.zeros(keep.shape[:-1] + (words * 32,), dtype=torch.bool, device=keep.device)
    k[..., :n] = keep
    v = (k.view(keep.shape[:-1] + (words, 32)).long() << torch.arange(32, device=keep.device)).sum(-1)
    return torch.where(v >= 2 ** 31, v - 2 ** 32, v).to(torch.int32)


def _unpack(words, n):
    b = (words.unsqueeze(-1) >> torch.arange(32, device=words.device, dtype=torch.int32)) & 1
    return b.reshape(words.shape[:-1] + (-1,))[..., :n].bool()


def _near(n, span):
    i = torch.arange(n)
    return (i[:, None] - i[None, :]).abs() <= span


class _State:
    pass


def _inputs(c, seed):
    """What the call takes, from the seed alone: tensors on the GPU."""
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    T, H, d = _tokens(c), c["H"], c["d"]
    i = _State()

    def normal(*shape, dtype=torch.bfloat16):
        return torch.randn(shape, generator=g, device=DEV).to(dtype)

    def uniform(*shape):
        return torch.rand(shape, generator=g, device=DEV)

    i.states = _states(c)
    if c["kind"] == "write":
        n, parts = len(i.states), 3 if c["q"] else 2
        # channels of very different sizes, as projections have them
        scale = torch.exp(torch.randn((parts, H, d), generator=g, device=DEV))
        x = torch.randn((n, T, parts, H, d), generator=g, device=DEV) * scale
        x[:, T // 2, :, 0] = 0        # a head that is all zeros
        x = x.to(torch.bfloat16)
        views = [x[:, :, p] for p in range(parts)]
        if not c["packed"]:
            views = [v.contiguous() for v in views]
        i.k, i.v = views[-2], views[-1]
        i.q = views[0] if c["q"] else None
        shape = {"shared": (d,), "heads": (H, d), "none": None}[c["gamma"]]
        i.gk = uniform(*shape) + 0.5 if shape else None
        i.gq = uniform(*shape) + 0.5 if shape and c["q"] else None
        return i
    i.k, i.v = normal(len(i.states), H, T, d), normal(len(i.states), H, T, d)    # as the cache holds them
    if c["kind"] == "condense":
        w = torch.exp(2 * torch.randn((c["src"], H, T), generator=g, device=DEV))
        w[uniform(c["src"], H, T) < c["zeros"]] = 0.0
        i.weight = w
        return i
    n = len(_round(c))
    i.q = normal(n, T, H, d)
    i.prev = torch.exp(torch.randn((len(i.states), H, T), generator=g, device=DEV)) if c["decay"] else None
    i.tile = i.tok_own = i.tok_hist = None
    W, nt = max(c["W"], 1), -(-T // 128)
    if c["mask"] == "tiles":
        keep = uniform(n, -(-nt // c["span"]), (1 + c["W"]) * nt) < c["keep"]
        keep = keep.repeat_interleave(c["span"], dim=1)[:, :nt]
        keep[:, :, :nt] = True
        i.tile = _pack(keep)
    elif c["mask"]:
        if c["mask"] == "local":
            h, w = _near(c["Hp"], c["span"]).to(DEV), _near(c["Wp"], c["span"]).to(DEV)
            m = (h[:, None, :, None] & w[None, :, None, :]).reshape(c["Hp"] * c["Wp"], -1).repeat(c["F"], c["F"])
            m = _pack(m)
            i.tok_own = m.expand(n, T, -1).contiguous()
            i.tok_hist = m[None, :, None].expand(n, T, W, -1).contiguous()
        else:
            def bits(*shape):
                return torch.randint(-2 ** 31, 2 ** 31, shape, generator=g, device=DEV, dtype=torch.int64).to(torch.int32)
            i.tok_own, i.tok_hist = bits(n, T, -(-T // 32)), bits(n, T, W, -(-T // 32))
        i.tok_own[:, 7::997] = 0      # queries that see nothing
        i.tok_hist[:, 7::997] = 0
    return i


def _keep(c, i, n, j, dev=DEV):
    """bool [T][T]: which keys of its state j (0 its own) node n's queries see; None: all."""
    T, nt = _tokens(c), -(-_tokens(c) // 128)
    keep = None
    if c["causal"] and j == 0:
        f = torch.arange(T, device=dev) // (c["Hp"] * c["Wp"])
        keep = f[:, None] >= f[None, :]
    more = None
    if i.tile is not None:
        t = _unpack(i.tile[n], (1 + c["W"]) * nt)[:, j * nt:(j + 1) * nt]
        more = t.repeat_interleave(128, 0)[:T].repeat_interleave(128, 1)[:, :T]
    elif i.tok_own is not None:
        more = _unpack(i.tok_own[n] if j == 0 else i.tok_hist[n, :, j - 1], T)
    if keep is None or more is None:
        return more if keep is None else keep
    return keep & more


def _log_sums(c, i):
    """The attention's log-sum-exps [n][H][T], as the program has them from its attention call."""
    T, H, d = _tokens(c), c["H"], c["d"]
    rnd = _round(c)
    lse = torch.empty((len(rnd), H, T), device=DEV)
    for n, (st, ctx) in enumerate(rnd):
        see = [i.states.index(s) for s in [st] + ctx]
        keep = [_keep(c, i, n, j) for j in range(len(see))]
        for h in range(H):
            q = i.q[n, :, h].float() / math.sqrt(d)
            parts = []
            for s, m in zip(see, keep):
                x = q @ i.k[s, h].float().t()
                if m is not None:
                    x.masked_fill_(~m, -math.inf)
                parts.append(torch.logsumexp(x, dim=1))
            lse[n, h] = torch.logsumexp(torch.stack(parts), dim=0)
    return lse


def _angles(c, chunk):
    """Rotation angles [T][d/2] of a chunk's tokens, in 64 bits."""
    u = torch.arange(_tokens(c), device=DEV)
    hw = c["Hp"] * c["Wp"]
    at = (c["F"] * chunk + u // hw, u % hw // c["Wp"], u % c["Wp"])
    return torch.cat([pos.double()[:, None] * THETA ** (-torch.arange(p, device=DEV, dtype=torch.float64) / max(p, 1))
                      for pos, p in zip(at, _pairs(c["d"]))], dim=1)


def prepare(case, seed):
    """A layer's cache with its history, the round's node table, the inputs and the output buffers."""
    c, s = case, _inputs(case, seed)
    s.c = c
    T, H, d = _tokens(c), c["H"], c["d"]
    if c["kind"] == "weights":
        s.lse = _log_sums(c, s)
    if not own:
        if c["kind"] == "write":
            a = torch.stack([_angles(c, b) for _, b, _ in s.states])[:, :, None]      # [n][T][1][d/2]
            s.cos, s.sin = torch.cos(a).float(), torch.sin(a).float()
        return s
    from paper_2609_22283_gb300 import sva
    top = max(b for _, b, _ in s.states)
    extra = 1 if c["kind"] == "condense" else 0
    geo = sva.make_geometry(H, d, c["F"], c["Hp"], c["Wp"], num_slots=len(s.states) + extra, pairs=_pairs(d),
                            max_frames=c["F"] * (top + 2), theta=THETA)
    s.cache = sva.Cache(geo, device=torch.device(DEV))
    s.cache.set_workspace(torch.empty(s.cache.workspace_bytes(), dtype=torch.uint8, device=DEV))
    slot = [s.cache.bind(*st) for st in s.states]
    pool = s.cache.slot_pool()
    at = {st: p for st, p in zip(s.states, slot)}
    if c["kind"] == "write":
        s.nodes = sva.make_nodes([dict(seq=q, chunk=b, level=j, own_slot=at[(q, b, j)]) for q, b, j in s.states])
        s.q_out = torch.empty((len(s.states), T, H, d), dtype=torch.bfloat16, device=DEV) if c["q"] else None
        s.written = [pool[p][:, :, :T] for p in slot]
        return s
    # the history as an earlier run left it: states marked written, then their very values restored
    blank = torch.zeros((1, T, H, d), dtype=torch.bfloat16, device=DEV)
    for (q, b, j), p in at.items():
        s.cache.rope_kv_write([dict(seq=q, chunk=b, level=j, own_slot=p)], blank, blank)
    for n, p in enumerate(slot):
        pool[p, 0, :, :T], pool[p, 1, :, :T] = s.k[n], s.v[n]
    order = torch.tensor(slot, device=DEV)
    if c["kind"] == "condense":
        s.src, s.dst = slot, s.cache.bind(0, top, LEVELS + 1)
        w = torch.zeros((len(slot) + 1, H, T), device=DEV)
        w[order] = s.weight
        s.weight = w
        s.index = torch.empty((H, T), dtype=torch.int32, device=DEV)
        s.kept = [pool[s.dst][:, :, :T], s.weight[s.dst], s.index]
        return s
    within = sva.WITHIN_FRAME_CAUSAL if c["causal"] else sva.WITHIN_BIDIRECTIONAL
    s.nodes = sva.make_nodes([dict(seq=st[0], chunk=st[1], level=st[2], own_slot=at[st], ctx=[at[t] for t in ctx],
                                   within=within) for st, ctx in _round(c)])
    if s.prev is not None:
        w = torch.empty((len(slot), H, T), device=DEV)
        w[order] = s.prev
        s.prev = w
    s.out = torch.empty((len(slot), H, T), device=DEV)
    s.outs = [s.out[p] for p in slot]
    return s


def run(state):
    s, c = state, state.c
    if own:
        if c["kind"] == "write":
            s.cache.rope_kv_write_headnorm(s.nodes, s.k, s.v, s.q, s.q_out, s.gk, s.gq, EPS)
            return s.written + ([s.q_out] if c["q"] else [])
        if c["kind"] == "condense":
            s.cache.condense(s.src, s.dst, s.weight, s.index)
            return s.kept
        s.cache.attend_weights(s.nodes, s.q, s.lse, s.out, prev=s.prev, decay=c["decay"], tile_mask=s.tile,
                               own_mask=s.tok_own, hist_mask=s.tok_hist if c["W"] else None)
        return s.outs
    return {"write": _plain_write, "weights": _plain_weights, "condense": _plain_condense}[c["kind"]](s, c)


# ------------------------------------------------------------------ the plain forms

def _plain_write(s, c):
    def turned(x, gamma):
        y = x.float()
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS)
        if gamma is not None:
            y = y * gamma
        a, b = y[..., 0::2], y[..., 1::2]
        return torch.stack((a * s.cos - b * s.sin, a * s.sin + b * s.cos), dim=-1).flatten(-2).to(torch.bfloat16)

    k = turned(s.k, s.gk)
    out = [torch.stack((k[n].transpose(0, 1), s.v[n].transpose(0, 1))) for n in range(k.shape[0])]
    return out + ([turned(s.q, s.gq)] if c["q"] else [])


def _plain_weights(s, c):
    scale = 1.0 / math.sqrt(c["d"])
    out = s.prev * c["decay"] if s.prev is not None else torch.zeros(s.k.shape[:3], device=DEV)
    for n, (st, ctx) in enumerate(_round(c)):
        lse = torch.where(s.lse[n] == -math.inf, math.inf, s.lse[n])      # a query that saw nothing adds nothing
        for j, t in enumerate([st] + ctx):
            m, at = _keep(c, s, n, j), s.states.index(t)
            for h in range(c["H"]):
                p = torch.exp((s.q[n, :, h].float() @ s.k[at, h].float().t()) * scale - lse[h][:, None])
                out[at, h] += (p if m is None else p * m).sum(0)
    return [out[i] for i in range(out.shape[0])]


def _plain_condense(s, c):
    T, H, d, n = _tokens(c), c["H"], c["d"], c["src"]
    w = s.weight.transpose(0, 1).reshape(H, n * T)
    best = torch.sort(w, dim=1, descending=True, stable=True).indices[:, :T]
    best = torch.sort(best, dim=1).values
    at = best[:, :, None].expand(H, T, d)
    kv = [x.transpose(0, 1).reshape(H, n * T, d).gather(1, at) for x in (s.k, s.v)]
    return [torch.stack(kv), w.gather(1, best), best.to(torch.int32)]


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
    T, H, d, n = _tokens(c), c["H"], c["d"], len(_states(c))
    if c["kind"] == "write":
        parts = 3 if c["q"] else 2
        return {"bytes": 2.0 * 2 * parts * n * T * H * d, "flops": (7.0 * (parts - 1)) * n * T * H * d}
    if c["kind"] == "condense":
        return {"bytes": 4.0 * n * T * H + 2 * (2 * 2.0 * T * H * d) + 8.0 * T * H, "flops": 1.0 * n * T * H}
    nodes = len(_round(c))
    by = 2.0 * nodes * T * H * d + 4.0 * nodes * H * T + 2.0 * n * T * H * d + 4.0 * n * H * T * (2 if c["decay"] else 1)
    if c["mask"] in ("local", "random"):
        by += nodes * T * T / 8 + sum(T * T * len(ctx) / 8 for _, ctx in _round(c))
    return {"bytes": by, "flops": 2.0 * _visible(c) * H * d}


# ------------------------------------------------------------------ in 64 bits

def exact(case, seed):
    c, i = case, _inputs(case, seed)
    T, H, d = _tokens(c), c["H"], c["d"]
    if c["kind"] == "write":
        def turned(x, gamma, chunk):      # complex numbers: pair (x, y) is x + iy
            y = x.double()
            y = y / torch.sqrt((y ** 2).sum(-1, keepdim=True) / d + EPS)
            y = y if gamma is None else y * gamma.double()
            z = torch.view_as_complex(y.reshape(T, H, d // 2, 2)) * torch.exp(1j * _angles(c, chunk))[:, None]
            return torch.view_as_real(z).reshape(T, H, d)

        got = [torch.stack((turned(i.k[n], i.gk, b).permute(1, 0, 2), i.v[n].double().permute(1, 0, 2)))
               for n, (_, b, _) in enumerate(i.states)]
        if c["q"]:
            got.append(torch.stack([turned(i.q[n], i.gq, b) for n, (_, b, _) in enumerate(i.states)]))
        return got
    if c["kind"] == "condense":
        # the T-th largest value, all above it, then the first ones equal to it
        kv, ws, at = [], [], []
        for h in range(H):
            w = i.weight[:, h].reshape(-1)
            line = torch.kthvalue(w, w.numel() - T + 1).values
            above, level = w > line, w == line
            take = above | (level & (torch.cumsum(level, 0) <= T - above.sum()))
            e = torch.nonzero(take)[:, 0]
            at.append(e.to(torch.int32)), ws.append(w[e].double())
            kv.append(torch.stack([x[:, h].reshape(-1, d)[e].double() for x in (i.k, i.v)]))
        return [torch.stack(kv, dim=1), torch.stack(ws), torch.stack(at)]
    if work(c)["flops"] > 4e12:
        return None
    lse = _log_sums(c, i).double()
    got = [torch.zeros((H, T), dtype=torch.float64, device=DEV) for _ in i.states]
    for n, (st, ctx) in enumerate(_round(c)):
        for j, t in enumerate([st] + ctx):
            m, to = _keep(c, i, n, j), got[i.states.index(t)]
            for h in range(H):
                k = i.k[i.states.index(t), h].double()
                for r in range(0, T, 2048):
                    x = torch.einsum("ud,vd->uv", i.q[n, r:r + 2048, h].double(), k) / math.sqrt(d)
                    x -= lse[n, h, r:r + 2048, None]
                    x.exp_()
                    gone = lse[n, h, r:r + 2048, None] == -math.inf
                    x.masked_fill_(gone if m is None else gone | ~m[r:r + 2048], 0.0)
                    to[h] += x.sum(0)
    if i.prev is not None:
        got = [g + c["decay"] * i.prev[n].double() for n, g in enumerate(got)]
    return got

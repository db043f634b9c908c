"""A layer over a video longer than its cache (stream.Stream): every call of the chain together, against
what the cache holds and where it came from."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def _pairs(d):
    return (d // 2 - 2 * (d // 6), d // 6, d // 6)


def test_stream_outgrows_its_cache(sva_mod):
    from paper_2609_22283_gb300.stream import Stream

    F, Hp, Wp, H, d, window, recent, chunks = 1, 9, 17, 2, 64, 3, 2, 11
    T = F * Hp * Wp
    st = Stream(H, d, F, Hp, Wp, _pairs(d), max_frames=F * (chunks + 2), window=window, recent=recent, decay=0.9)
    c = st.cache
    g = torch.Generator(device="cuda").manual_seed(4)
    gk, gq = torch.rand((H, d), generator=g, device="cuda") + 0.5, torch.rand((H, d), generator=g, device="cuda") + 0.5
    origin, rows, weight = {}, {}, {}    # slot -> [H][T] ids; id -> its K' and V rows; slot -> [H][T] in 64 bits
    pool = c.slot_pool()
    most = 0
    for chunk in range(1, chunks + 1):
        for level in (2, 0):
            qkv = torch.randn((1, T, 3, H, d), generator=g, device="cuda").bfloat16()
            q, k, v = qkv[:, :, 0], qkv[:, :, 1], qkv[:, :, 2]
            out = torch.empty((1, T, H, d), dtype=torch.bfloat16, device="cuda")
            ctx = st.context()
            assert len(ctx) == len(st.clean) + (1 if st.condensed else 0)
            before = {s: w.clone() for s, w in weight.items()}
            free = set(range(window + 3)) - set(ctx)
            held, kept = list(st.clean), st.condensed
            st.update(chunk, level, q, k, v, out, gk, gq)
            if level == 0:
                own = dict(st.clean)[chunk]
            else:     # the slot that was free and lowest on the stack: its K' is the one just written
                cand = [s for s in free if torch.equal(pool[s, 1, :, :T].transpose(0, 1), v[0])]
                assert len(cand) == 1
                own = cand[0]
            # the attention over exactly the context and the own chunk
            see = ctx + [own]
            y = q.double()
            y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + 1e-6) * gq.double()
            u = torch.arange(T, device="cuda")
            pos = (F * chunk + u // (Hp * Wp), u % (Hp * Wp) // Wp, u % Wp)
            ang = torch.cat([p.double()[:, None] * 10000.0 ** (-torch.arange(n, device="cuda", dtype=torch.float64) / n)
                             for p, n in zip(pos, _pairs(d))], 1)
            z = torch.view_as_complex(y.reshape(T, H, d // 2, 2)) * torch.exp(1j * ang)[:, None]
            qr = torch.view_as_real(z).reshape(T, H, d).bfloat16().double()
            if level == 0 and st.condensed != kept:
                # condensed after the update: the sources' slots are still as they were
                assert st.condensed[1] not in see
            for h in range(H):
                kk = torch.cat([pool[s, 0, h, :T] for s in see]).double()
                vv = torch.cat([pool[s, 1, h, :T] for s in see]).double()
                p = torch.softmax(qr[:, h] @ kk.t() / math.sqrt(d), 1)
                # bf16 rotation of q (a value on the other side of a rounding moves a logit by 2^-8 of a
                # term), bf16 weights and output
                bound = 2.0 ** -6 * (p @ vv.abs()) + 2e-3
                assert torch.all((out[0, :, h].double() - p @ vv).abs() <= bound)
                got = p.sum(0)
                for i, s in enumerate(see):
                    w = weight.setdefault(s, torch.zeros((H, T), dtype=torch.float64, device="cuda"))
                    w[h] = got[i * T:(i + 1) * T] + (0.9 * before[s][h] if s in ctx else 0.0)
            for s in see:
                assert torch.allclose(st.weight[s].double(), weight[s], rtol=2e-2, atol=1e-3), (chunk, level, s)
                weight[s] = st.weight[s].double()      # the rounding of q above does not add up over the chunks
            if level:
                weight.pop(own)
                continue
            origin[own] = (chunk * T + u)[None].expand(H, T).clone()
            for t in range(T):
                rows[chunk * T + t] = pool[own, :, :, t].clone()      # [2][H][d]
            if st.condensed != kept:
                src = ([kept[1]] if kept else []) + [s for _, s in held[:len(held) + 1 - recent]]
                ids = torch.cat([origin[s] for s in src], 1)
                ws = torch.cat([st.weight[s] for s in src], 1)
                dst = st.condensed[1]
                origin[dst] = ids.gather(1, st.index.long())
                weight[dst] = st.weight[dst].double()
                for h in range(H):
                    kept_w, all_w = ws[h][st.index[h].long()], ws[h]
                    assert torch.equal(st.weight[dst, h], kept_w)
                    assert kept_w.min() >= torch.sort(all_w, descending=True).values[T - 1]
                    for t in range(0, T, 13):
                        assert torch.equal(pool[dst, :, h, t], rows[int(origin[dst][h, t])][:, h])
                for s in src:
                    origin.pop(s), weight.pop(s)
            most = max(most, len(st.context()))
    assert c.poll() == sva_mod.OK
    assert st.condensed is not None and most == window + 1
    # every condensed token came from a chunk up to the state's own, none twice
    ids = origin[st.condensed[1]]
    assert int(ids.max()) // T <= st.condensed[0]
    for h in range(H):
        assert len(torch.unique(ids[h])) == T
    st.close()


def test_stream_refuses_bad_windows(sva_mod):
    from paper_2609_22283_gb300.stream import Stream
    for window, recent in ((3, 0), (3, 4), (15, 2)):
        with pytest.raises(ValueError):
            Stream(2, 64, 1, 2, 2, _pairs(64), 16, window=window, recent=recent)

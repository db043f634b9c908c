"""PackedStream: a layer over a long window in 4 bits, and branches of a video: its book of slots on the CPU with a
cache that only keeps the tables, and every call of the chain together on the GPU against the formula."""
import pytest
import torch

from tests._packed import assert_attention, attention, held, pairs

F, HP, WP, H, D = 1, 5, 27, 2, 64
T = F * HP * WP


class FakeCache:
    """The two tables of slots and the calls; call number `fail_at` raises."""

    def __init__(self, geometry, device=None):
        self.buf = torch.empty(0)
        self.free, self.bound = list(range(geometry.num_slots))[::-1], {}
        self.packed_free, self.packed_bound = [], {}
        self.calls, self.fail_at = [], None

    def workspace_bytes(self):
        return 0

    def set_workspace(self, ws):
        pass

    def set_packed(self, buf, n):
        self.packed_free = list(range(n))[::-1]

    @staticmethod
    def _take(free, bound, state):
        if state in bound or not free:
            raise RuntimeError(f"cannot bind {state}")
        bound[state] = free.pop()
        return bound[state]

    def bind(self, *state):
        return self._take(self.free, self.bound, state)

    def bind_packed(self, *state):
        return 1000 + self._take(self.packed_free, self.packed_bound, state)

    def release(self, *state):
        self.free.append(self.bound.pop(state))

    def release_packed(self, *state):
        self.packed_free.append(self.packed_bound.pop(state))

    def _call(self, *what):
        self.calls.append(what)
        if self.fail_at is not None and len(self.calls) > self.fail_at:
            raise RuntimeError(what[0])

    def rope_kv_write_headnorm(self, *a, **kw):
        self._call("write")

    def attend_nodes_packed(self, nodes, *a, **kw):
        self._call("attend", list(nodes[0].ctx_slot[:nodes[0].n_ctx]))

    def pack(self, slots, packed):
        self._call("pack", slots, packed)

    def copy(self, src, dst):
        self._call("copy", src, dst)


@pytest.fixture
def fake(monkeypatch):
    from paper_2609_22283_gb300 import stream as module
    monkeypatch.setattr(module.sva, "Cache", FakeCache)
    monkeypatch.setattr(module.sva, "packed_bytes", lambda g, n: 16 * n)
    return lambda **kw: module.PackedStream(H, D, F, HP, WP, pairs(D), 64, device="cpu", **kw)


X = torch.empty((1, T, H, D), dtype=torch.bfloat16)


@pytest.mark.parametrize("window,recent", [(1, 0), (1, 1), (3, 0), (3, 1), (4, 4), (16, 2)])
def test_window(fake, window, recent):
    """After any number of chunks the newest `recent` are whole, those before them packed, up to the window, and a
    context lists them oldest first; nothing else is bound."""
    st = fake(window=window, recent=recent)
    c = st.cache
    for chunk in range(1, 2 * window + 6):
        for level in (3, 0):
            st.update(chunk, level, X, X, X, X)
        keep = list(range(max(1, chunk - window + 1), chunk + 1))
        whole, packed = keep[len(keep) - min(recent, len(keep)):], keep[:len(keep) - min(recent, len(keep))]
        assert c.bound == {(0, b, 0): s for b, s in st.whole[0]} and [b for b, _ in st.whole[0]] == whole
        assert {k: 1000 + s for k, s in c.packed_bound.items()} == {(0, b, 0): s for b, s in st.packed[0]}
        assert [b for b, _ in st.packed[0]] == packed and len(st.context()) == min(chunk, window)


@pytest.mark.parametrize("fail", range(2))
def test_failed_update_leaves_nothing(fake, fail):
    st = fake(window=3, recent=1)
    c = st.cache
    for chunk in range(1, 6):
        st.update(chunk, 0, X, X, X, X)
    before = (dict(c.bound), dict(c.packed_bound), st.context())
    for level in (0, 2) * 4:
        c.fail_at = len(c.calls) + fail
        with pytest.raises(RuntimeError, match=("write", "attend")[fail]):
            st.update(6, level, X, X, X, X)
    assert before == (c.bound, c.packed_bound, st.context())
    c.fail_at = None
    st.update(6, 0, X, X, X, X)


def test_branches(fake):
    st = fake(window=4, recent=2, sequences=2)
    c = st.cache
    for chunk in range(1, 7):
        st.update(chunk, 0, X, X, X, X)
    free = (len(c.free), len(c.packed_free))
    for fail in (0, 1):      # either copy fails: nothing of the branch is left
        c.fail_at = len(c.calls) + fail
        with pytest.raises(RuntimeError, match="copy"):
            st.fork(0, 5)
        assert (len(c.free), len(c.packed_free)) == free and list(st.whole) == list(st.packed) == [0]
    c.fail_at = None
    with pytest.raises(ValueError):
        st.fork(1, 2)
    st.fork(0, 5)
    assert [b for b, _ in st.whole[5]] == [5, 6] and [b for b, _ in st.packed[5]] == [3, 4]
    assert not set(st.context(0)) & set(st.context(5))
    for new in (5, 0, 7):    # exists, exists, one too many
        with pytest.raises(ValueError):
            st.fork(0, new)
    for chunk in range(7, 12):
        st.update(chunk, 2, X, X, X, X, seq=5)
        st.update(chunk, 0, X, X, X, X, seq=5)
        st.update(chunk, 0, X, X, X, X, seq=0)
    assert [b for b, _ in st.whole[5]] == [10, 11] and [b for b, _ in st.packed[0]] == [8, 9]
    st.drop(0)
    st.fork(5, 6)
    st.drop(5), st.drop(6)
    assert not c.bound and not c.packed_bound


def test_arguments(fake):
    for kw in (dict(window=0), dict(window=17), dict(window=3, recent=4), dict(recent=-1), dict(sequences=0)):
        with pytest.raises(ValueError):
            fake(**kw)


@pytest.mark.gpu
def test_on_the_gpu(sva_mod):
    """Two sequences that branch, window 5 of which 2 whole: every update's attention over the states as they are
    held, a packed one's values those of the state that was written."""
    from paper_2609_22283_gb300 import sva
    from paper_2609_22283_gb300.stream import PackedStream

    st = PackedStream(H, D, F, HP, WP, pairs(D), max_frames=40, window=5, recent=2, sequences=2)
    other = sva.Cache(sva.make_geometry(H, D, F, HP, WP, 1, pairs(D), 40))     # for the rotated queries alone
    g = torch.Generator(device="cuda").manual_seed(8)
    gk, gq = torch.rand((H, D), generator=g, device="cuda") + 0.5, torch.rand((H, D), generator=g, device="cuda") + 0.5
    pool = st.cache.slot_pool()
    written = {0: {}}       # sequence -> chunk -> K', V as written
    out, rotated = torch.empty((1, T, H, D), dtype=torch.bfloat16, device="cuda"), torch.empty((1, T, H, D), dtype=torch.bfloat16, device="cuda")

    def update(seq, chunk, level):
        qkv = torch.randn((1, T, 3, H, D), generator=g, device="cuda").bfloat16()
        q, k, v = qkv.unbind(2)
        s = other.bind(seq, chunk, level)
        other.rope_kv_write_headnorm([dict(seq=seq, chunk=chunk, level=level, own_slot=s)], k, v, q, rotated, gk, gq)
        own = other.slot_pool()[s, :, :, :T].clone()
        other.release(seq, chunk, level)
        packed, whole = [b for b, _ in st.packed[seq]], [b for b, _ in st.whole[seq]]
        assert len(whole) <= 2 and len(packed) <= 3 and packed + whole == sorted(packed + whole)
        kv = [held(written[seq][b]) for b in packed] + [written[seq][b].double() for b in whole] + [own.double()]
        st.update(chunk, level, q, k, v, out, gk, gq, seq=seq)
        for h in range(H):
            k, v = (torch.cat([x[i, h] for x in kv]) for i in (0, 1))
            ref = attention(rotated[0, :, h], k, v)
            assert_attention(out[0, :, h], ref[1].float(), ref, f"{seq} {chunk} {level}")
        if level == 0:
            written[seq][chunk] = own
            for b, s in st.whole[seq]:
                assert torch.equal(pool[s, :, :, :T], written[seq][b])

    for chunk in range(1, 9):
        update(0, chunk, 2)
        update(0, chunk, 0)
    st.fork(0, 3)
    written[3] = dict(written[0])
    for chunk in range(9, 14):
        update(3, chunk, 0)
        update(0, chunk, 1)
        update(0, chunk, 0)
    st.drop(0)
    st.fork(3, 4)
    written[4] = dict(written[3])
    update(4, 14, 0)
    update(3, 14, 0)
    assert st.cache.poll() == sva_mod.OK
    st.close()
    other.close()

"""An update of stream.Stream that raises leaves the cache as it was: its slot is free again, and the same update
can be made once more."""
import pytest
import torch

F, HP, WP, H, D = 1, 3, 5, 2, 64
T = F * HP * WP
PAIRS = (D // 2 - 2 * (D // 6), D // 6, D // 6)


class FakeCache:
    """Keeps the book of slots that Cache keeps and records its calls; call number `fail_at` raises."""

    def __init__(self, geometry, device=None):
        self.buf = torch.empty(0)
        self.H, self.T = H, T
        self.free, self.bound = list(range(geometry.num_slots))[::-1], {}
        self.calls, self.fail_at = [], None

    def workspace_bytes(self):
        return 0

    def set_workspace(self, ws):
        pass

    def bind(self, *state):
        if state in self.bound or not self.free:
            raise RuntimeError(f"cannot bind {state}")
        self.bound[state] = self.free.pop()
        return self.bound[state]

    def release(self, *state):
        self.free.append(self.bound.pop(state))

    def _call(self, name):
        self.calls.append(name)
        if self.fail_at is not None and len(self.calls) > self.fail_at:
            raise RuntimeError(name)

    def rope_kv_write_headnorm(self, *a, **kw):
        self._call("write")

    def attend_nodes(self, *a, **kw):
        self._call("attend")

    def attend_weights(self, *a, **kw):
        self._call("weights")

    def condense(self, *a, **kw):
        self._call("condense")


@pytest.fixture
def stream(monkeypatch):
    from paper_2609_22283_gb300 import stream as module
    monkeypatch.setattr(module.sva, "Cache", FakeCache)
    return module.Stream(H, D, F, HP, WP, PAIRS, 64, window=3, recent=2, device="cpu")


@pytest.mark.parametrize("level", [0, 2])
@pytest.mark.parametrize("fail_at", [0, 1, 2])
def test_slot_is_free_again(stream, level, fail_at):
    c = stream.cache
    x = torch.empty((1, T, H, D), dtype=torch.bfloat16)
    stream.update(1, 0, x, x, x, x)
    before, free = dict(c.bound), sorted(c.free)
    c.fail_at = len(c.calls) + fail_at
    for _ in range(8):           # more often than there are slots
        with pytest.raises(RuntimeError, match=("write", "attend", "weights")[fail_at]):
            stream.update(2, level, x, x, x, x)
        c.fail_at = len(c.calls) + fail_at
    assert c.bound == before and sorted(c.free) == free and len(stream.clean) == 1
    c.fail_at = None
    stream.update(2, level, x, x, x, x)
    assert len(stream.clean) == (2 if level == 0 else 1)


@pytest.mark.gpu
def test_refused_updates(sva_mod):
    """Wrong shapes, a chunk outside the rotation table and one that is not after the condensed state."""
    from paper_2609_22283_gb300.stream import Stream
    st = Stream(H, D, F, HP, WP, PAIRS, max_frames=8, window=3, recent=2)
    g = torch.Generator(device="cuda").manual_seed(9)
    qkv = torch.randn((7, 1, T, 3, H, D), generator=g, device="cuda").bfloat16()
    out = torch.empty((1, T, H, D), dtype=torch.bfloat16, device="cuda")

    def update(chunk, level=0, **kw):
        q, k, v = (qkv[chunk % 7, :, :, i] for i in range(3))
        a = dict(q=q, k=k, v=v, out=out)
        a.update(kw)
        st.update(chunk, level, **a)

    for chunk in range(1, 5):
        update(chunk)
    assert st.condensed is not None
    context, slots = st.context(), list(st.clean)
    weight = st.weight.clone()
    for _ in range(3):
        for bad in (dict(k=out[:, :3]), dict(out=out.float()), dict(out=out[:, :3])):
            with pytest.raises(ValueError):
                update(5, **bad)
        with pytest.raises(sva_mod.SvaError) as e:
            update(9)
        assert e.value.status == sva_mod.ERR_CAPACITY
        with pytest.raises(sva_mod.SvaError) as e:
            update(2, level=3)
        assert e.value.status == sva_mod.ERR_CAUSALITY
    assert st.context() == context and list(st.clean) == slots
    assert torch.equal(st.weight[context], weight[context])
    update(5)
    assert [b for b, _ in st.clean][-1] == 5
    assert st.cache.poll() == sva_mod.OK
    st.close()

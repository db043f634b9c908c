"""PackedStream when the state that leaves the newest ones cannot be packed, on the CPU with the cache that only keeps
the tables: the update leaves no trace and is made again, and no other sequence notices."""
import pytest

from tests.test_packed_stream import X, fake  # noqa: F401  (a fixture)


def _books(st):
    c = st.cache
    return (dict(c.bound), dict(c.packed_bound), {q: list(s) for q, s in st.whole.items()},
            {q: list(s) for q, s in st.packed.items()})


@pytest.mark.parametrize("fails", ["pack", "bind_packed"])
@pytest.mark.parametrize("window,recent", [(1, 0), (3, 1), (3, 2), (16, 0)])
def test_an_update_whose_parking_fails_is_made_again(fake, monkeypatch, fails, window, recent):  # noqa: F811
    st = fake(window=window, recent=recent)
    twin = fake(window=window, recent=recent)
    c = st.cache
    for chunk in range(1, 2 * window + 4):
        for _ in range(2):
            if chunk <= recent:      # nothing is parked yet
                break
            before = _books(st)
            with monkeypatch.context() as m:
                def fail(*a):
                    raise RuntimeError("no " + fails)
                m.setattr(c, fails, fail)
                with pytest.raises(RuntimeError, match="no " + fails):
                    st.update(chunk, 0, X, X, X, X)
            assert _books(st) == before
        for s in (st, twin):
            s.update(chunk, 2, X, X, X, X)
            s.update(chunk, 0, X, X, X, X)
        assert {k: [b for b, _ in v] for k, v in st.whole.items()} == {k: [b for b, _ in v] for k, v in twin.whole.items()}
        assert {k: [b for b, _ in v] for k, v in st.packed.items()} == {k: [b for b, _ in v] for k, v in twin.packed.items()}
    assert len(st.context()) == window


def test_other_sequences_go_on(fake, monkeypatch):  # noqa: F811
    """All sequences full: one whose state cannot be parked does not take the slot that the others' updates need."""
    st = fake(window=4, recent=2, sequences=2)
    c = st.cache
    for chunk in range(1, 8):
        st.update(chunk, 0, X, X, X, X)
    st.fork(0, 1)
    before = _books(st)
    with monkeypatch.context() as m:
        def fail(*a):
            raise RuntimeError("no pack")
        m.setattr(c, "pack", fail)
        with pytest.raises(RuntimeError, match="no pack"):
            st.update(8, 0, X, X, X, X, seq=0)
        assert _books(st) == before
        st.update(8, 3, X, X, X, X, seq=1)
    for seq in (1, 0):
        st.update(8, 0, X, X, X, X, seq=seq)
        assert [b for b, _ in st.packed[seq]] == [5, 6] and [b for b, _ in st.whole[seq]] == [7, 8]
    st.drop(0)
    st.fork(1, 2)
    st.drop(1), st.drop(2)
    assert not c.bound and not c.packed_bound

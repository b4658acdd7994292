"""runtime.KVCache's own bookkeeping, on the CPU: the entry points that it calls are stood in for by recorders."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

HQ, HKV, DH, PAGE = 4, 2, 32, 16
WIDTH = (HQ + 2 * HKV) * DH


class Recorder:
    """In the binding's place: names and arguments of the calls; `refuse` makes the next call of that name fail."""

    def __init__(self, error):
        self.calls, self.refuse, self.error = [], None, error

    def make_kv_cache(self, *a):
        return "struct"

    def brl_attention_cached_workspace_bytes(self, *a):
        return 64

    def __getattr__(self, name):
        def call(*a):
            if self.refuse == name:
                self.refuse = None
                raise self.error
            self.calls.append((name, a))
        return call

    def named(self, name):
        return [a for n, a in self.calls if n == name]


@pytest.fixture
def holder(monkeypatch):
    from paper_2604_24273_amd import runtime as R
    fake = Recorder(ValueError("refused"))
    monkeypatch.setattr(R, "B", fake)
    monkeypatch.setattr(R, "DEV", "cpu")

    def make(states=2, max_tokens=64, **kw):
        return R.KVCache(states, HQ, HKV, DH, max_tokens, 1e4, page_tokens=PAGE, **kw)

    return make, fake


def rows(n):
    return torch.zeros(n, WIDTH)


def book(kv):
    """Everything that the holder keeps, on the host and for the device; pages as who owns how many."""
    return (kv.lens_host.tolist(), kv.seen.tolist(), [list(p) for p in kv.pages], sorted(kv.free), kv.lens.tolist(), kv.table.tolist())


def test_a_refused_append_changes_nothing(holder):
    make, fake = holder
    kv = make()
    for before in ([], [20, 3]):                                          # nothing held yet; something appended
        if before:
            kv.append(rows(sum(before)), before)
        was, last = book(kv), kv._last
        fake.refuse = "attention_cache_append"
        with pytest.raises(ValueError, match="refused"):
            kv.append(rows(21), [18, 3])
        assert book(kv) == was and kv._last is last
        if before:
            kv.attend()                                                   # of the tokens appended before
            assert fake.named("attention_cached_forward")[-1][3] == sum(before)
        else:
            with pytest.raises(ValueError, match="append"):
                kv.attend()
    kv.append(rows(21), [18, 3])                                          # the same once more
    assert kv.lens_host.tolist() == [38, 6] and kv.seen.tolist() == [38, 6] and kv.lens.tolist() == [38, 6]
    assert [len(p) for p in kv.pages] == [3, 1] and len(kv.free) == 8 - 4


def test_the_attention_of_an_append_is_added_up_once(holder):
    """Attending again (another mask, a call that was refused) gives outputs, but no slot its weight a second time."""
    make, fake = holder
    kv = make(track_weights=True)
    for new in ([5, 2], [1, 0]):
        kv.append(rows(sum(new)), new)
        fake.refuse = "attention_cached_forward"
        with pytest.raises(ValueError, match="refused"):
            kv.attend()
        begin = len(fake.named("attention_cached_forward"))
        kv.attend()
        kv.attend(torch.ones(sum(new), 1, dtype=torch.int32))
        fake.refuse = "attention_cache_append"
        with pytest.raises(ValueError, match="refused"):
            kv.append(rows(1), [1, 0])
        kv.attend()
        calls = fake.named("attention_cached_forward")[begin:]
        assert [c[14] is not None for c in calls] == [True, False, False]


def test_a_state_goes_on_behind_the_tokens_that_it_keeps(holder):
    """The next token's position is behind the last one kept, also where the kept ones are no whole path from the first."""
    make, fake = holder
    kv = make(states=4)
    position = lambda: fake.named("attention_cache_append")[-1][8].tolist()  # noqa: E731
    kv.append(rows(8), [2, 2, 2, 2])
    kv.append(rows(11), [3, 4, 4, 0], [0, 1, 2, 0, 0, 1, 2, 0, 1, 2, 3])
    kv.keep_branch([[0, 2], [1, 2, 3], [], []])                           # its middle dropped; a path; nothing; nothing new
    assert kv.lens_host.tolist() == [4, 5, 2, 2]
    kv.append(rows(5), [2, 1, 1, 1])
    assert position() == [5, 6, 5, 2, 2]
    kv.keep_branch([[1], [0], [0], []])
    kv.append(rows(4), [1, 1, 1, 1])
    assert position() == [7, 6, 3, 2]

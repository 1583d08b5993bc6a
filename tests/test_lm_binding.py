"""The Python binding's own checks of the cache plan, whose sizes it takes from the tensors (on the host: a refused call reaches nothing)."""
import pytest
import torch


def _tensors(**other):
    t = dict(cached=torch.zeros(3, dtype=torch.int32), fresh=torch.zeros(3, dtype=torch.int32), free_pages=torch.zeros(5, dtype=torch.int32),
             table=torch.zeros((3, 4), dtype=torch.int32), starts=torch.zeros(4, dtype=torch.int32), slots=torch.zeros(9, dtype=torch.int64), counts=torch.zeros(2, dtype=torch.int32))
    t.update(other)
    return [t[k] for k in ("cached", "fresh")] + [16] + [t[k] for k in ("free_pages", "table", "starts", "slots", "counts")]


@pytest.fixture
def plan(monkeypatch):
    """The binding over a library that takes note of the call instead of making it."""
    import paper_2011_10680_amd.binding as b
    calls = []

    class Library:
        def hawq_cache_plan(self, *a):
            calls.append(a)
            return 0
    monkeypatch.setattr(b, "load_library", Library)
    return lambda *t: b.hawq_cache_plan(*t, stream=0), calls


def test_sound_tensors_pass(plan):
    call, calls = plan
    call(*_tensors())
    assert calls[0][:5] == (3, 16, 4, 5, 9)
    call(*_tensors(starts=torch.zeros(9, dtype=torch.int32), counts=torch.zeros(7, dtype=torch.int32)))
    none = torch.zeros(0, dtype=torch.int32)
    call(*_tensors(cached=none, fresh=none, table=torch.zeros((0, 4), dtype=torch.int32), free_pages=none, slots=torch.zeros(0, dtype=torch.int64)))
    assert len(calls) == 3


@pytest.mark.parametrize("other", [
    dict(table=torch.zeros((3, 9), dtype=torch.int32)[:, :4]), dict(table=torch.zeros((4, 3), dtype=torch.int32).t()), dict(table=torch.zeros((2, 4), dtype=torch.int32)),
    dict(table=torch.zeros(12, dtype=torch.int32)), dict(fresh=torch.zeros(2, dtype=torch.int32)), dict(cached=torch.zeros(6, dtype=torch.int32)[::2]),
    dict(starts=torch.zeros(3, dtype=torch.int32)), dict(counts=torch.zeros(1, dtype=torch.int32)), dict(slots=torch.zeros(18, dtype=torch.int64)[::2]),
    dict(free_pages=torch.zeros(10, dtype=torch.int32)[::2])])
def test_sizes_and_strides_that_the_call_would_misread(plan, other):
    from paper_2011_10680_amd import HawqError
    call, calls = plan
    with pytest.raises(HawqError):
        call(*_tensors(**other))
    assert not calls


@pytest.mark.parametrize("name", ["cached", "fresh", "free_pages", "table", "starts", "slots", "counts"])
def test_types_that_the_call_would_misread(plan, name):
    from paper_2011_10680_amd import HawqError
    call, calls = plan
    for dt in (torch.int32 if name == "slots" else torch.int64, torch.float32):
        shape = dict(table=(3, 4), starts=(4,), counts=(2,), slots=(9,), free_pages=(5,)).get(name, (3,))
        with pytest.raises(HawqError):
            call(*_tensors(**{name: torch.zeros(shape, dtype=dt)}))
    assert not calls

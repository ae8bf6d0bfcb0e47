"""The asynchronous engine advances one request: a second one is refused where it would be made."""
import pytest

from paper_2506_19830_b200.async_cycle import AsyncCycleEngine


def engine():
    eng = object.__new__(AsyncCycleEngine)  # (its host side; the pages themselves are on a device)
    eng.pages, eng.length, eng.free = [[3, 1]], [20], [2, 0]
    return eng


def test_a_fork_is_refused_and_leaves_the_engine_as_it_was():
    eng = engine()
    with pytest.raises(NotImplementedError, match="one request"):
        eng.fork(0)
    assert eng.pages == [[3, 1]] and eng.length == [20] and eng.free == [2, 0]

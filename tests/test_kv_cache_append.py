"""FqKvCache.append: what a refused call leaves behind, and what it does on the host (no GPU needed; the calls are plain copies, as in test_kv_cache_fork.py)."""
import sys

import pytest

from paper_2402_17985_amd import binding, kv_cache
from tests.test_kv_cache_fork import Model, copies  # noqa: F401


def test_a_refused_copy_loses_no_past(copies, monkeypatch):  # noqa: F811
    """Page copies are refused where the cache is not on the current device.  The sequences still share what they shared; the same append goes through later."""
    m = Model(12, 4)
    m.append([100, 0, 0, 0])
    m.fork(0, [1, 2])
    before = ([list(h) for h in m.cache.held], list(m.cache._users), list(m.cache._free), m.cache.page_table.clone())
    with monkeypatch.context() as c:
        def refuse(*_, **__):
            raise ValueError("not on the current device")
        c.setattr(binding, "fq_kv_copy_pages", refuse)
        rows = m.cache.k_cache[:3, :, 0]
        with pytest.raises(ValueError, match="current device"):
            m.cache.append(None, rows, rows, [1, 1, 1, 0])
    assert before[:3] == (m.cache.held, m.cache._users, m.cache._free) and (before[3] == m.cache.page_table).all()
    m.check()
    m.append([1, 1, 1, 0])
    m.check()
    assert len(copies) == 1 and len(copies[0][0]) == 2


def lines_of(call):
    """Lines that a call runs in the cache's own file."""
    count = 0

    def local(frame, event, _):
        nonlocal count
        count += event == "line"
        return local

    before = sys.gettrace()
    sys.settrace(lambda frame, event, _: local if frame.f_code.co_filename == kv_cache.__file__ else None)
    try:
        call()
    finally:
        sys.settrace(before)
    return count


@pytest.mark.parametrize("grow", [False, True])
def test_an_append_without_forks_does_not_look_for_shared_pages(copies, grow):  # noqa: F811
    """It runs once for every layer and token.  A cache that cannot fork takes 10 lines a sequence (15 for one that takes a page)."""
    counts = []
    for batch in (16, 80):
        m = Model(4 * batch, batch)
        m.append([64 if grow else 10] * batch)
        counts.append(lines_of(lambda: m.append([1] * batch)))
        m.check()
    assert counts[1] - counts[0] <= (15 if grow else 10) * 64


def test_one_write_to_the_table(copies, monkeypatch):  # noqa: F811
    """However many sequences take pages of their own or grow: a write for each is a launch for each."""
    m = Model(40, 8)
    m.append([100] + [0] * 7)
    m.fork(0, [1, 2, 3, 4, 5])
    m.append([0] * 6 + [63, 63])
    sent = []
    make = m.cache._i32
    monkeypatch.setattr(m.cache, "_i32", lambda values: sent.append(values) or make(values))
    m.append([1, 1, 100, 0, 5, 1, 2, 2])
    m.check()
    assert len(sent) == 5                      # source and target pages of the copies, the table's changes, offsets and lengths

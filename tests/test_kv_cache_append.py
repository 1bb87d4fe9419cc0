"""FqKvCache.append: what a refused call leaves behind (no GPU needed; the calls are plain copies, as in test_kv_cache_fork.py)."""
import pytest

from paper_2402_17985_amd import binding
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

"""FqKvCache's bookkeeping around the calls, with the calls themselves replaced (no GPU needed)."""
import pytest
import torch

import paper_2402_17985_amd as fq
from paper_2402_17985_amd import binding


@pytest.fixture
def calls(monkeypatch):
    """What reaches the binding, in order; tensors are kept alive as a stream that has not run yet would need them."""
    seen = []
    monkeypatch.setattr(binding, "fq_kv_append", lambda *a, **k: seen.append(("append", a, k)))
    monkeypatch.setattr(binding, "fq_attn_cache", lambda *a, **k: seen.append(("attend", a, k)))
    return seen


def _cache(batch=2, max_len=4096):
    return fq.FqKvCache(2 * batch * max_len // 64, batch, max_len, 1, 64, device="cpu")


def _rows(n, heads=1):
    return torch.zeros((n, heads, 64), dtype=torch.bfloat16)


def test_attentions_under_way_at_once_have_workspaces_of_their_own(calls):
    """Two streams may be at it together, and a larger call may follow one that has not run yet."""
    c = _cache()
    c.append(None, _rows(3000), _rows(3000), [3000, 0])
    for n in (1, 1, 2):
        c.attend(_rows(n), [n, 0], 0.125)
    spaces = [a[-1] for kind, a, _ in calls if kind == "attend"]
    assert len(spaces) == 3 and all(s.numel() > 16 for s in spaces)
    ends = sorted((s.data_ptr(), s.data_ptr() + s.numel()) for s in spaces)
    assert all(a[1] <= b[0] for a, b in zip(ends, ends[1:]))


@pytest.mark.parametrize("new", [[3, -1], [-2, 4], [-1, -1]])
def test_counts_below_zero_are_refused(calls, new):
    """They would make offsets that fall, which the kernels cut, and lengths that the pages do not hold."""
    c = _cache()
    c.append(None, _rows(130), _rows(130), [70, 60])
    before = (list(c.lengths), [list(h) for h in c.held])
    with pytest.raises(ValueError, match="negative"):
        c.append(None, _rows(max(0, sum(new))), _rows(max(0, sum(new))), new)
    with pytest.raises(ValueError, match="negative"):
        c.attend(_rows(max(0, sum(new))), new, 0.125)
    assert (c.lengths, c.held) == before and len(calls) == 1


def test_calls_get_offsets_lengths_and_bounds(calls):
    c = _cache()
    c.append(None, _rows(130), _rows(130), [70, 60])
    c.append(None, _rows(1), _rows(1), [0, 1])
    c.attend(_rows(3), [2, 1], 0.125)
    (_, a, _), (_, b, _), (_, d, _) = calls
    assert [t.tolist() for t in a[3:5]] == [[0, 70, 130], [0, 0]] and a[5] == 70
    assert [t.tolist() for t in b[3:5]] == [[0, 0, 1], [70, 60]] and b[5] == 1
    assert [t.tolist() for t in d[1:3]] == [[0, 2, 3], [70, 61]] and d[3:5] == (2, 70)

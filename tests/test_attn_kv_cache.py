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

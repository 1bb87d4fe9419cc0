"""What the binding of fq_rms_norm_quant hands to the library (no GPU needed: the tensors are the host's, and the library is replaced)."""
from types import SimpleNamespace

import pytest
import torch

from paper_2402_17985_amd import binding


@pytest.fixture
def calls(monkeypatch):
    seen = []
    monkeypatch.setattr(binding, "_get_device", lambda: -1)
    monkeypatch.setattr(binding, "_stream_on", lambda stream, here: None)
    monkeypatch.setattr(binding, "_lib", SimpleNamespace(fq_rms_norm_quant=lambda *a: seen.append(a)))
    return seen


def norm(**k):
    x, i = torch.zeros(4, 64), torch.arange(64, dtype=torch.int32)
    binding.fq_rms_norm_quant(**{**dict(X=x, gamma=x[0], eps=1e-5, src_idx=i, rep=i, Xq_out=torch.zeros(4, 64, dtype=torch.int8), s_x_out=torch.zeros(1),
                                        workspace=torch.zeros(1 << 16, dtype=torch.uint8)), **k})


def test_a_bound_without_a_value_is_refused(calls):
    """Its address is null, which would ask for a dynamic scale."""
    with pytest.raises(ValueError, match="absmax_in"):
        norm(absmax_in=torch.zeros(0))
    assert not calls
    for shape in ((), (1,), (2,)):
        bound = torch.zeros(shape)
        norm(absmax_in=bound)
        assert calls[-1][20] == bound.data_ptr() != 0
    norm()
    assert calls[-1][20] is None

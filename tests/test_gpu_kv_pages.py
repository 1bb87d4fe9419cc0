"""fq_kv_copy_pages: bytes of pages and scales."""
import numpy as np
import pytest
import torch

import paper_2402_17985_amd as fq
from oracle import step as S
from tests import step_util as T

pytestmark = pytest.mark.gpu


def pool(rng, pages, heads, page, dim):
    k = rng.integers(-128, 128, (pages, heads, page, dim)).astype(np.int8)
    v = rng.integers(-128, 128, (pages, heads, dim, page)).astype(np.int8)
    return [k, v] + [rng.standard_normal((pages, heads)).astype(np.float32) for _ in range(2)]


@pytest.mark.parametrize("heads", [1, 3, 8, 40])
@pytest.mark.parametrize("page", [64, 128])
@pytest.mark.parametrize("dim", [64, 80, 96, 128])
def test_pages(heads, page, dim):
    rng = np.random.default_rng(heads + page + dim)
    arrays = pool(rng, 21, heads, page, dim)
    dev = [torch.from_numpy(a.copy()).to(T.DEV) for a in arrays]
    order = rng.permutation(21).astype(np.int32)
    src, dst = order[:8].copy(), order[8:16].copy()
    src[3] = src[0]                                                   # one page copied twice
    src[5], dst[6], src[7], dst[7] = 21, -1, 2**31 - 1, -2**31         # no such pages
    dst[4] = src[4]                                                   # itself
    S.copy_pages(arrays, src, dst)
    fq.fq_kv_copy_pages(*dev, torch.from_numpy(src).to(T.DEV), torch.from_numpy(dst).to(T.DEV))
    for a, d in zip(arrays, dev):
        assert np.array_equal(a, d.cpu().numpy())


def test_no_pages():
    dev = [torch.from_numpy(a).to(T.DEV) for a in pool(np.random.default_rng(0), 2, 1, 64, 64)]
    none = torch.empty(0, dtype=torch.int32, device=T.DEV)
    fq.fq_kv_copy_pages(*dev, none, none)


def test_many_pages_of_one_head():
    rng = np.random.default_rng(1)
    arrays = pool(rng, 5000, 1, 64, 64)
    dev = [torch.from_numpy(a.copy()).to(T.DEV) for a in arrays]
    order = rng.permutation(5000).astype(np.int32)
    src, dst = order[:2400].copy(), order[2500:4900].copy()
    S.copy_pages(arrays, src, dst)
    fq.fq_kv_copy_pages(*dev, torch.from_numpy(src).to(T.DEV), torch.from_numpy(dst).to(T.DEV))
    for a, d in zip(arrays, dev):
        assert np.array_equal(a, d.cpu().numpy())


def test_pages_beyond_4_gib():
    """Byte offsets that 32 bits cannot hold."""
    pages, heads, page, dim = 9000, 64, 64, 128        # 4.7 GB each
    k, v = (torch.zeros(s, dtype=torch.int8, device=T.DEV) for s in ((pages, heads, page, dim), (pages, heads, dim, page)))
    ks, vs = (torch.zeros(pages, heads, device=T.DEV) for _ in range(2))
    k[8999], v[8999], ks[8999], vs[8999] = 3, 4, 5.0, 6.0
    k[1], v[1], ks[1], vs[1] = 7, 8, 9.0, 10.0
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device=T.DEV)  # noqa: E731
    fq.fq_kv_copy_pages(k, v, ks, vs, i32(8999, 1), i32(0, 8998))
    for t, (a, b) in ((k, (3, 7)), (v, (4, 8)), (ks, (5, 9)), (vs, (6, 10))):
        assert (t[0] == a).all() and (t[8998] == b).all() and (t[1] == b).all() and not t[2].any()

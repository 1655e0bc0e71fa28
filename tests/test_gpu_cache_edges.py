"""Token-cache operators on the GPU where their input is broken, unequal or out of the ordinary: pages outside the pool,
lengths beyond the table, unequal batches, rare layouts, and what the operators refuse."""
import math

import pytest
import torch

from .test_gpu_cache import BF16, F16, UNIT, Case

pytestmark = pytest.mark.gpu

OUTSIDE = (-1, -(1 << 31), (1 << 31) - 1)   # page ids that no pool has; -1 is what a search pads its answer with


class Holes(Case):
    """A case whose table names no page of the pool in some places: tokens that belong to such a place take no part."""

    def __init__(self, lens, news, share=0.3, **kw):
        super().__init__(lens, news, **kw)
        self.whole, pages = self.table.clone(), self.k.shape[0]
        self.gone = torch.rand(self.table.shape, generator=self.g, device="cuda") < share
        ids = torch.tensor(OUTSIDE + (pages,), dtype=torch.int32, device="cuda")
        pick = torch.randint(0, len(ids), self.table.shape, generator=self.g, device="cuda")
        self.table = torch.where(self.gone & (self.whole >= 0), ids[pick], self.whole)
        self.cache.status, self.found = (lambda: 0), self.cache.status    # (the checks of Case want none set)

    def where(self, b, n, first=0):
        j = torch.arange(first, n, device="cuda")
        return (self.whole if hasattr(self, "whole") else self.table)[b].long()[j // self.page], j % self.page

    def valid(self, b):
        return ~self.gone[b][torch.arange(self.lens[b], device="cuda") // self.page]

    def seen(self, b, causal=True, window=0):
        return super().seen(b, causal, window) & self.valid(b)[None]


def pad_heads(c, extra):
    """The case on a pool whose heads lie `extra` entries further apart than they are long."""
    from paper_2608_21163_b200.cache import TokenCache
    k, v = (torch.full((*x.shape[:3], x.shape[3] + extra), math.nan, device="cuda", dtype=x.dtype) for x in (c.k, c.v))
    k[..., : c.dim], v[..., : c.dim] = c.k, c.v
    c.k, c.v = k[..., : c.dim], v[..., : c.dim]
    status = c.cache.status
    c.cache = TokenCache(c.k, c.v, c.weights, q_heads=c.qh, max_batch=max(1, len(c.lens)), max_tokens=max(1, c.total))
    if isinstance(c, Holes):
        c.cache.status, c.found = status, c.cache.status
    return c


# ---- pages outside the pool

HOLES = [
    # lens, news: the streaming kernels, then those on the tensor cores
    ([300, 17, 130, 1], [1, 1, 1, 1]), ([90, 400], [3, 4]), ([5000], [1]), ([700, 90], [200, 60]), ([1500], [300]), ([40], [40]),
]


@pytest.mark.parametrize("lens,news", HOLES)
@pytest.mark.parametrize("dtype,dim,page,share", [(BF16, 64, 1, 0.3), (F16, 128, 3, 0.2), (BF16, 96, 16, 0.5), (BF16, 128, 48, 0.3), (F16, 40, 128, 0.5), (BF16, 64, 4, 1.0)])
def test_attend_leaves_out_tokens_without_a_page(lens, news, dtype, dim, page, share):
    c = Holes(lens, news, share, qh=8, kvh=2, dim=dim, page=page, dtype=dtype)
    c.check_attend()
    assert c.found() == (1 if bool(torch.cat([~c.valid(b) for b in range(len(lens))]).any()) else 0)
    c.check_attend(scale=-0.2)
    c.check_attend(scale=0.0)


@pytest.mark.parametrize("window", [1, 60, 200])
@pytest.mark.parametrize("lens,news", [([300, 64], [4, 1]), ([700, 130], [200, 130])])
def test_attend_window_with_tokens_without_a_page(lens, news, window):
    Holes(lens, news, 0.4, qh=4, kvh=2, dim=64, page=16).check_attend(window=window)


def test_attend_all_with_tokens_without_a_page():
    Holes([300, 64, 9], [4, 1, 9], 0.4, qh=4, kvh=1, dim=64, page=5, heads_first=True).check_attend(causal=False)
    Holes([300, 640], [150, 64], 0.4, qh=4, kvh=1, dim=128, page=5, heads_first=True).check_attend(causal=False)


@pytest.mark.parametrize("qh,new", [(1, 1), (4, 40)])
def test_a_padded_list_of_rows_is_its_rows(qh, new):
    """A search pads its answer with an id that no row has; the padding must change neither output nor sum."""
    k = 50
    c = Case([k] * 3, [new] * 3, qh=qh, kvh=1, dim=64, page=1)
    want, lse = c.cache.attend(c.q, c.table, c.kv_lens, cu_new=c.cu, causal=False)
    padded = torch.cat([c.table, torch.full((3, 14), -1, dtype=torch.int32, device="cuda")], 1)
    got, padded_lse = c.cache.attend(c.q, padded, torch.full_like(c.kv_lens, k + 14), cu_new=c.cu, causal=False)
    assert torch.equal(got, want) and torch.equal(padded_lse, lse)
    assert c.cache.status() == 1


@pytest.mark.parametrize("lens,news", HOLES)
@pytest.mark.parametrize("dim,page,groups", [(64, 1, 1), (128, 16, 2), (96, 5, 2)])
def test_weigh_with_tokens_without_a_page(lens, news, dim, page, groups):
    Holes(lens, news, 0.3, qh=8, kvh=2, dim=dim, page=page, groups=groups).check_weigh()

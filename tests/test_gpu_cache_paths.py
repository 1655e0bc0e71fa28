"""Token-cache operators on the GPU where a call takes a path of its own: unequal batches, layouts without a tile load or with
loads of one row, long lists whose keys the blocks do not hold, and the precision of the probabilities."""
import math

import pytest
import torch

from .test_gpu_cache import BF16, F16, UNIT, Case, kept_ref
from .test_gpu_cache_edges import Holes, pad_heads

pytestmark = pytest.mark.gpu


# ---- batches of unequal sequences

@pytest.mark.parametrize("lens,news", [
    ([128] * 127 + [16384], [1] * 128), ([16384] + [128] * 127, [1] * 128), ([3] * 200 + [9000], [1] * 201),    # one long cache
    ([1500] * 60 + [3000], [1] * 60 + [512]), ([3000] + [1500] * 63, [440] + [1] * 63), ([700] * 20 + [2500], [1] * 20 + [900]),   # one long chunk
    ([0, 5000, 1, 40, 0, 9, 2600], [0, 700, 1, 40, 0, 1, 2])])
@pytest.mark.parametrize("dim", [64, 128])
def test_unequal_sequences(lens, news, dim):
    c = Case(lens, news, qh=8, kvh=2, dim=dim, page=16)
    c.check_attend()
    c.check_weigh()
    c.check_attend(window=300)
    c.check_weigh(window=300, decay=0.5)


@pytest.mark.parametrize("lens,news", [([40000], [1]), ([9000, 100], [3, 8]), ([6000, 900], [700, 900]), ([20000], [40])])
def test_equal_calls_give_equal_bits(lens, news):
    """Parts of a sequence are joined in their order, whichever block arrives last."""
    c = Case(lens, news, qh=8, kvh=2, dim=64, page=16)
    want, lse = c.cache.attend(c.q, c.table, c.kv_lens, cu_new=c.cu)
    for _ in range(20):
        got, again = c.cache.attend(c.q, c.table, c.kv_lens, cu_new=c.cu)
        assert torch.equal(got, want) and torch.equal(again, lse)


# ---- layouts

@pytest.mark.parametrize("page", [1, 2, 4, 6])
@pytest.mark.parametrize("dim,extra,dtype", [(120, 8, BF16), (64, 8, F16), (40, 24, BF16)])
@pytest.mark.parametrize("lens,news", [([700, 90], [200, 60]), ([300, 17], [1, 1])])
def test_heads_further_apart_than_they_are_long(page, dim, extra, dtype, lens, news):
    """Small pages of a pool that is no plain list of rows: tile loads of one, two or four rows."""
    c = pad_heads(Case(lens, news, qh=4, kvh=2, dim=dim, page=page, dtype=dtype), extra)
    c.check_attend()
    c.check_weigh()
    pad_heads(Holes(lens, news, 0.3, qh=4, kvh=2, dim=dim, page=page, dtype=dtype), extra).check_attend()


@pytest.mark.parametrize("lens,news", [([700, 90], [200, 60]), ([300, 17], [1, 1])])
def test_heads_that_share_their_rows(lens, news):
    """A pool expanded over its heads has a stride of 0, which no tile load describes: the streaming kernels take such a call."""
    from paper_2608_21163_b200.cache import TokenCache
    c = Case(lens, news, qh=4, kvh=2, dim=64, page=16)
    c.k[:, :, 1], c.v[:, :, 1] = c.k[:, :, 0], c.v[:, :, 0]
    k, v = (x[:, :, :1].contiguous().expand(-1, -1, 2, -1) for x in (c.k, c.v))
    c.cache = TokenCache(k, v, c.weights, q_heads=4, max_batch=2, max_tokens=c.total)
    c.check_attend()
    c.check_weigh()


@pytest.mark.parametrize("lens,news", [([300, 40], [1, 1]), ([500], [30])])
def test_more_query_heads_than_a_tile_has_rows(lens, news):
    c = Case(lens, news, qh=130, kvh=1, dim=64, page=16)
    c.check_attend()
    c.check_weigh()


@pytest.mark.parametrize("inplace", [True, False])
def test_evict_lists_that_the_blocks_do_not_hold(inplace):
    """One block a list (there are more lists than half the SMs) of more tokens than its shared memory has keys for."""
    lens, keep, groups, page = [26000, 24600] + [25500 + i for i in range(18)], 5000, 4, 64
    c = Case(lens, [0] * len(lens), kvh=groups, qh=groups, dim=8, page=page, groups=groups, spare=3 + len(lens) * -(-keep // page))
    w = torch.rand(c.weights.shape, generator=c.g, device="cuda")
    c.weights.copy_(torch.where(w < 0.9, (w * 64).floor() / 64, w))
    into = None if inplace else c.spare.nonzero().flatten()[: len(lens) * -(-keep // page)].view(len(lens), -1).to(torch.int32)
    k0, w0 = c.k.clone(), c.weights.clone()
    kept, new = c.cache.evict(c.table, c.kv_lens, keep, sinks=7, recent=300, into=into)
    assert new.tolist() == [keep] * len(lens)
    dest = c.table if inplace else into
    for b in (0, 1, 9, len(lens) - 1):
        p, s = c.where(b, lens[b])
        for g in range(groups):
            ref = kept_ref(w0[p, g, s], lens[b], keep, 7, 300)
            assert kept[b, g].tolist() == ref
            j, i = torch.tensor(ref, device="cuda"), torch.arange(keep, device="cuda")
            dp, ds = dest[b].long()[i // page], i % page
            assert torch.equal(c.k[dp, ds, g], k0[p[j], s[j], g]) and torch.equal(c.weights[dp, g, ds], w0[p[j], g, s[j]])
    assert c.cache.status() == 0


# ---- precision

@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("news", [[1, 1], [8, 8]])     # tiles of 16 rows and of 32
def test_the_streaming_kernel_keeps_what_a_probability_loses(dtype, news):
    """Neighbouring keys have almost equal scores and opposite values, so an output is small beside its terms.  Probabilities
    that meet the values as two 16-bit numbers leave the output's own rounding; rounded to one they would not."""
    n, u = 32, UNIT[dtype]
    c = Case([n, n], news, qh=4, kvh=1, dim=64, page=16, dtype=dtype)
    c.q.mul_(0.1)
    for b in range(2):
        p, s = c.where(b, n)
        k, v = torch.randn((n // 2, 64), generator=c.g, device="cuda"), torch.rand((n // 2, 64), generator=c.g, device="cuda") + 0.5
        c.k[p, s, 0] = torch.stack([k, k * (1 + 2.0 ** -6)], 1).flatten(0, 1).to(dtype)
        c.v[p, s, 0] = torch.stack([v, -v], 1).flatten(0, 1).to(dtype)
    out, _ = c.cache.attend(c.q, c.table, c.kv_lens, cu_new=c.cu, causal=False)
    ref, _, mag, most = c.reference(c.dim ** -0.5, causal=False)
    e = c.score_bound(most)
    # a probability keeps all but u^2 of itself (in float16 to a multiple of 2^-24 beside a largest of 2^7, n of them on values
    # below 1.6), its score is off by e, products and sums by a unit a step
    bound = (1.05 * u * u + 2 * e + 2 * n * 2.0 ** -23) * mag + 1.05 * u * ref.abs() + (n * 2.0 ** -31 * 1.6 + 2.0 ** -25 if dtype == F16 else 0.0)
    assert bool((out.double() - ref).abs().le(bound).all()), float(((out.double() - ref).abs() / bound).max())
    # the same with probabilities of one 16-bit number breaks the bound (in bfloat16, whose rounding is far above the others)
    if dtype == BF16:
        worst, t = 0.0, 0
        for b, m in enumerate(news):
            k, v = c.rows(b)
            for h in range(4):
                x = c.q[t : t + m, h].double() @ k[:, 0].T * c.dim ** -0.5
                p = (x - x.amax(1, keepdim=True)).exp()
                once = (p.to(dtype).double() @ v[:, 0]) / p.sum(1, keepdim=True)
                worst = max(worst, float(((once - ref[t : t + m, h]).abs() / bound[t : t + m, h]).max()))
            t += m
        assert worst > 2.0
    assert c.cache.status() == 0

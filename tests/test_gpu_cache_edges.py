"""Token-cache operators on the GPU where their input is broken, unequal or out of the ordinary: pages outside the pool,
lengths beyond the table, unequal batches, rare layouts, and what the operators refuse."""
import math

import pytest
import torch

from paper_2608_21163_b200.binding import GrandError

from .test_gpu_cache import BF16, F16, UNIT, Case, rope_ref_differentiable

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


def kept_with_gaps(w, valid, keep, sinks, recent):
    n, valid = len(valid), valid.tolist()
    if n <= keep:
        return [j for j in range(n) if valid[j]]
    rank = [(-math.inf if x != x else x) for x in w.tolist()]
    fixed = [j for j in (*range(sinks), *range(n - recent, n)) if valid[j]]
    free = sorted((j for j in range(sinks, n - recent) if valid[j]), key=lambda j: (-rank[j], j))
    return sorted(fixed + free[: keep - len(fixed)])


@pytest.mark.parametrize("inplace", [True, False])
@pytest.mark.parametrize("lens,keep,sinks,recent,page,kvh,dim,groups,share", [
    ([300, 40, 257, 0], 64, 4, 16, 16, 2, 64, 2, 0.3), ([300, 64, 257], 64, 40, 24, 1, 2, 40, 1, 0.3), ([300, 1], 64, 0, 0, 16, 1, 64, 1, 0.9),
    ([300, 20], 32, 32, 0, 5, 2, 64, 2, 0.4), ([9000, 30, 8200], 3000, 16, 100, 7, 1, 8, 1, 0.3), ([20000], 19000, 0, 500, 16, 1, 8, 1, 0.3),
    ([500, 300], 64, 4, 16, 16, 2, 64, 1, 1.0)])
def test_evict_with_tokens_without_a_page(inplace, lens, keep, sinks, recent, page, kvh, dim, groups, share):
    c = Holes(lens, [0] * len(lens), share, kvh=kvh, qh=kvh, dim=dim, page=page, groups=groups, spare=3 + len(lens) * -(-keep // page))
    w = torch.rand(c.weights.shape, generator=c.g, device="cuda")
    w = torch.where(w < 0.5, (w * 8).floor() / 8, w)
    w[w > 0.99] = math.nan
    c.weights.copy_(w)
    into = None
    if not inplace:
        into = c.spare.nonzero().flatten()[: len(lens) * -(-keep // page)].view(len(lens), -1).to(torch.int32)
    k0, v0, w0 = c.k.clone(), c.v.clone(), c.weights.clone()
    want_k, want_v, want_w = k0.clone(), v0.clone(), w0.clone()
    kept, new = c.cache.evict(c.table, c.kv_lens, keep, sinks=sinks, recent=recent, into=into)
    for b, n in enumerate(lens):
        p, s = c.where(b, n)
        for g in range(groups):
            ref = kept_with_gaps(w0[p, g, s], c.valid(b), keep, sinks, recent)
            assert kept[b, g].tolist() == ref + [-1] * (keep - len(ref)) and int(new[b]) == len(ref)
            j, i = torch.tensor(ref, device="cuda", dtype=torch.long), torch.arange(len(ref), device="cuda")
            dp, ds = (c.table if inplace else into)[b].long()[i // page], i % page
            there = (dp >= 0) & (dp < c.k.shape[0])      # a slot in a page outside the pool takes nothing
            j, dp, ds = j[there], dp[there], ds[there]
            want_w[dp, g, ds] = w0[p[j], g, s[j]]
            for h in range(kvh) if groups == 1 else [g]:
                want_k[dp, ds, h], want_v[dp, ds, h] = k0[p[j], s[j], h], v0[p[j], s[j], h]
    for got, want in ((c.k, want_k), (c.v, want_v), (c.weights, want_w)):
        assert torch.equal(got.nan_to_num(77.0), want.nan_to_num(77.0))
    assert c.found() == 1


# ---- lengths and bounds that do not fit

@pytest.mark.parametrize("lens,cu,written", [
    # written: slots of either sequence and the rows that they get
    ([65, 40], None, ({}, {39: 1})),                                               # one slot past the table
    ([66, 40], [0, 5, 8], ({61: 0, 62: 1, 63: 2}, {37: 5, 38: 6, 39: 7})),         # the last two of five past it
    ([1 << 30, 40], [0, 5, 8], ({}, {37: 5, 38: 6, 39: 7})),
    ([-3, 40], [0, 5, 8], ({}, {37: 5, 38: 6, 39: 7})),
    ([64, 40], [0, 5, 12], ({59 + i: i for i in range(5)}, {})),                   # bounds past the rows of the call
    ([64, 40], [-2, 5, 8], ({}, {37: 5, 38: 6, 39: 7})),
    ([64, 40], [0, 6, 2], ({58 + i: i for i in range(6)}, {})),                    # bounds that descend
])
def test_append_writes_no_other_tokens_slot(lens, cu, written):
    c = Case([64, 48], [1, 1] if cu is None else [5, 3], qh=4, kvh=2, dim=64, page=16)
    c.weights.fill_(3.0)
    k, v = (torch.randn((c.total, 2, 64), generator=c.g, device="cuda").to(BF16) for _ in range(2))
    want_k, want_v, want_w = c.k.clone(), c.v.clone(), c.weights.clone()
    for b in range(2):
        for slot, row in written[b].items():
            p, s = int(c.table[b, slot // 16]), slot % 16
            want_k[p, s], want_v[p, s], want_w[p, :, s] = k[row], v[row], 0.0
    c.cache.append(None, k, v, None, None, c.table, torch.tensor(lens, dtype=torch.int32, device="cuda"),
                   cu_new=None if cu is None else torch.tensor(cu, dtype=torch.int32, device="cuda"))
    for got, want in ((c.k, want_k), (c.v, want_v), (c.weights, want_w)):
        assert torch.equal(got.nan_to_num(77.0), want.nan_to_num(77.0))
    assert c.cache.status() == 4


def test_evict_refuses_to_write_the_lengths_that_it_reads():
    import ctypes as C
    c = Case([100, 50], [1, 1], qh=4, kvh=2, dim=64)
    hold = c.cache._sequences(c.table, c.kv_lens, None, 2)
    kept, after = torch.zeros((2, 2, 20), dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    both = torch.tensor([100, 50, 0, 0], dtype=torch.int32, device="cuda")

    def evict(lens, out):
        c.cache._seqs.kv_lens = lens.data_ptr()
        stream = torch.cuda.current_stream().cuda_stream
        return c.cache.lib.grand_cache_evict(c.cache.h, c.cache._pool_at, c.cache._seqs_at, 20, 0, 0, None, 0, 0, kept.data_ptr(), out.data_ptr(), C.c_void_p(stream))

    assert evict(both, both) == -1 and b"lens_out" in c.cache.lib.grand_cache_last_error(c.cache.h)
    assert evict(both, both[1:]) == -1 and evict(both[1:], both) == -1
    assert evict(both, both[2:]) == 0 and both.tolist() == [100, 50, 20, 20]
    assert evict(both, after[1:]) == 0 and after.tolist() == [0, 20, 20, 0]
    del hold


# ---- arguments that do not fit

def test_tensors_elsewhere_are_refused():
    """Every tensor has to be on the pool's device: a pointer to host memory must never reach a kernel."""
    from paper_2608_21163_b200.cache import rope, rope_frequencies, rope_table
    c = Case([100, 50], [1, 1], qh=4, kvh=2, dim=64)
    k, table, at = c.q[:, :2].contiguous(), rope_table(128, rope_frequencies(64)), torch.tensor([99, 49], dtype=torch.int32, device="cuda")
    spare = c.spare.nonzero().flatten()[:2].view(2, 1).to(torch.int32)
    _, lse = c.cache.attend(c.q, c.table, c.kv_lens, cu_new=c.cu)
    calls = {
        "append": (c.cache.append, dict(q=c.q, k=k, v=k, table=table, positions=at, page_table=c.table, kv_lens=c.kv_lens, cu_new=c.cu, q_out=torch.empty_like(c.q))),
        "attend": (c.cache.attend, dict(q=c.q, page_table=c.table, kv_lens=c.kv_lens, cu_new=c.cu, out=torch.empty_like(c.q), lse=torch.empty_like(lse))),
        "weigh": (c.cache.weigh, dict(q=c.q, lse=lse, page_table=c.table, kv_lens=c.kv_lens, cu_new=c.cu)),
        "evict": (c.cache.evict, dict(page_table=c.table, kv_lens=c.kv_lens, keep=16, into=spare)),
        "rope": (rope, dict(x=c.q, table=table, positions=at, out=torch.empty_like(c.q)))}
    for name, (call, kw) in calls.items():
        for arg, t in kw.items():
            if isinstance(t, torch.Tensor):
                with pytest.raises(ValueError):
                    call(**{**kw, arg: t.cpu()})
        call(**kw)
    with pytest.raises(ValueError):
        rope_table_on_host = table.cpu()
        rope(c.q.cpu(), rope_table_on_host, at.cpu())


@pytest.mark.parametrize("number", [-1, 1 << 32, (1 << 32) + 5])
def test_numbers_that_32_bits_do_not_hold_are_refused(number):
    from paper_2608_21163_b200.cache import TokenCache
    c = Case([100, 50], [1, 1], qh=4, kvh=2, dim=64)
    for call in (lambda: c.cache.attend(c.q, c.table, c.kv_lens, window=number),
                 lambda: c.cache.weigh(c.q, torch.zeros(2, 4, device="cuda"), c.table, c.kv_lens, window=number),
                 lambda: c.cache.evict(c.table, c.kv_lens, number), lambda: c.cache.evict(c.table, c.kv_lens, 16, sinks=number),
                 lambda: c.cache.evict(c.table, c.kv_lens, 16, recent=number), lambda: TokenCache(c.k, c.v, q_heads=number),
                 lambda: TokenCache(c.k, c.v, max_batch=number), lambda: TokenCache(c.k, c.v, max_tokens=number)):
        with pytest.raises(ValueError):
            call()
    # the largest window that fits is as good as none
    want, _ = c.cache.attend(c.q, c.table, c.kv_lens)
    assert torch.equal(c.cache.attend(c.q, c.table, c.kv_lens, window=(1 << 32) - 1)[0], want)


def test_the_ids_of_a_search_are_a_page_table():
    """uint32, as they come, padding included, and non-contiguous too."""
    c = Case([30] * 3, [1] * 3, qh=2, kvh=1, dim=64, page=1)
    want, lse = c.cache.attend(c.q, c.table, c.kv_lens)
    ids = c.table.view(torch.uint32)
    padded = torch.full((3, 40), 0xFFFFFFFF, dtype=torch.int64, device="cuda").to(torch.uint32)
    padded.view(torch.int32)[:, :30] = c.table
    spread = padded.view(torch.int32).repeat_interleave(2, 1).view(torch.uint32)[:, ::2]
    for table, n in ((ids, 30), (padded, 40), (spread, 40)):
        got, got_lse = c.cache.attend(c.q, table, torch.full_like(c.kv_lens, n))
        assert torch.equal(got, want) and torch.equal(got_lse, lse)
    c.weights.zero_()
    assert torch.equal(c.cache.evict(ids, c.kv_lens, 10, into=c.table[:, :10].clone().view(torch.uint32))[0].cpu(), torch.arange(10, dtype=torch.int32).expand(3, 1, 10))


# ---- gradients

@pytest.mark.parametrize("dtype", [BF16, F16, torch.float32])
@pytest.mark.parametrize("inter,inverse,dim,rot", [(False, False, 48, 32), (True, False, 64, 64), (False, True, 64, 64), (True, True, 40, 6)])
def test_rope_takes_part_in_a_backward_pass(dtype, inter, inverse, dim, rot):
    from paper_2608_21163_b200.cache import rope, rope_frequencies, rope_table
    g = torch.Generator(device="cuda"); g.manual_seed(7)
    table = rope_table(100, rope_frequencies(rot), magnitude=1.2)
    pos = torch.randint(0, 100, (9,), generator=g, device="cuda", dtype=torch.int32)
    x, up = (torch.randn((9, 3, dim), generator=g, device="cuda").to(dtype) for _ in range(2))
    wide = torch.randn((9, 5, dim + 8), generator=g, device="cuda").to(dtype).requires_grad_()   # a view of it goes in
    leaf = x.clone().requires_grad_()
    for param, part in ((leaf, leaf), (wide, wide[:, 1:4, :dim])):
        y = rope(part, table, pos, interleaved=inter, inverse=inverse)
        assert torch.equal(y.detach(), rope(part.detach(), table, pos, interleaved=inter, inverse=inverse))
        (grad,) = torch.autograd.grad(y, param, up)
        d = part.detach().double().requires_grad_()
        t = table.clone()
        if inverse:
            t[:, rot // 2 :] *= -1
        (want,) = torch.autograd.grad(rope_ref_differentiable(d, t, pos, inter), d, up.double())
        grad = grad if param is leaf else grad[:, 1:4, :dim]
        size = float(up.abs().max()) * 1.2 * 2
        bound = UNIT[dtype] * 1.01 * want.abs() + 3 * 2.0 ** -24 * size + (2.0 ** -25 if dtype == F16 else 0.0)
        assert bool((grad.double() - want).abs().le(bound).all())
    # through a sum, whose gradient has no strides; and a gradient of a gradient
    (grad,) = torch.autograd.grad(rope(leaf, table, pos, interleaved=inter, inverse=inverse).sum(), leaf)
    assert torch.equal(grad, rope(torch.ones_like(x), table, pos, interleaved=inter, inverse=not inverse))
    v = up.clone().requires_grad_()
    (grad,) = torch.autograd.grad(rope(leaf, table, pos, interleaved=inter, inverse=inverse), leaf, v, create_graph=True)
    (again,) = torch.autograd.grad(grad, v, x)
    assert torch.equal(again, rope(x, table, pos, interleaved=inter, inverse=inverse))


def test_what_has_no_gradient_says_so():
    from paper_2608_21163_b200.cache import rope, rope_frequencies, rope_table
    c = Case([100, 50], [1, 1], qh=4, kvh=2, dim=64)
    table, at = rope_table(128, rope_frequencies(64)), torch.tensor([99, 49], dtype=torch.int32, device="cuda")
    k = c.q[:, :2].contiguous()
    want, lse = c.cache.attend(c.q, c.table, c.kv_lens)
    turned = c.cache.append(c.q, k, k, table, at, c.table, c.kv_lens)
    q = c.q.clone().requires_grad_()
    for call, plain in ((lambda: c.cache.append(q, k, k, table, at, c.table, c.kv_lens), turned),
                        (lambda: c.cache.append(c.q, k.clone().requires_grad_(), k, table, at, c.table, c.kv_lens), turned),
                        (lambda: c.cache.attend(q * 1, c.table, c.kv_lens)[0], None), (lambda: c.cache.attend(q, c.table, c.kv_lens)[1], None)):
        y = call()
        assert y.requires_grad and (plain is None or torch.equal(y.detach(), plain))
        y += 1      # (an output may still be changed in place)
        with pytest.raises(RuntimeError, match="no gradient"):
            y.float().sum().backward()
    with torch.no_grad():
        out = torch.empty_like(want)
        got, _ = c.cache.attend(q, c.table, c.kv_lens, out=out)
        assert got is out and not got.requires_grad and rope(q, table, at, out=out) is out
    for call in (lambda: c.cache.attend(q, c.table, c.kv_lens, out=out), lambda: c.cache.append(q, k, k, table, at, c.table, c.kv_lens, q_out=out),
                 lambda: rope(q, table, at, out=out), lambda: rope(c.q, table.clone().requires_grad_(), at)):
        with pytest.raises(ValueError):
            call()
    assert not c.cache.attend(c.q, c.table, c.kv_lens)[0].requires_grad


@pytest.mark.parametrize("dtype", [BF16, torch.float32])
def test_rope_records_positions_outside_the_table(dtype):
    from paper_2608_21163_b200.cache import rope, rope_frequencies, rope_table
    table, x = rope_table(50, rope_frequencies(32)), torch.randn((5, 3, 40), device="cuda").to(dtype)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    good = torch.tensor([0, 49, 7, 49, 0], dtype=torch.int32, device="cuda")
    want = rope(x, table, good, status=status)
    assert status.tolist() == [0]
    bad = torch.tensor([0, 50, 7, (1 << 31) - 1, -1], dtype=torch.int32, device="cuda")
    assert torch.equal(rope(x, table, bad, status=status), want) and status.tolist() == [2]
    assert torch.equal(rope(x, table, bad), want)
    status.zero_()
    rope(x.clone().requires_grad_(), table, bad, status=status)
    assert status.tolist() == [2]
    for wrong in (status.cpu(), status.float(), torch.zeros(2, dtype=torch.int32, device="cuda")):
        with pytest.raises(ValueError):
            rope(x, table, good, status=wrong)


def test_collection_during_a_capture():
    import gc
    from paper_2608_21163_b200.cache import TokenCache, _collected
    c = Case([500, 70], [1, 1], qh=8, kvh=2, dim=64)
    want, lse = c.cache.attend(c.q, c.table, c.kv_lens)
    other = TokenCache(c.k, c.v, q_heads=8)
    other.attend(c.q, c.table, c.kv_lens)
    out, l2, graph = torch.empty_like(want), torch.empty_like(lse), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.cache.attend(c.q, c.table, c.kv_lens, out=out, lse=l2)
        del other
        gc.collect()
        assert len(_collected) >= 1
    graph.replay()
    assert torch.equal(out, want) and torch.equal(l2, lse)
    TokenCache(c.k, c.v, q_heads=8).close()
    assert not _collected


# ---- numerics

@pytest.mark.parametrize("new", [1, 40])     # the streaming kernel, and the one on the tensor cores
def test_many_small_probabilities_count_in_float16(new):
    """64 keys that draw almost all of the weight, and nearly 3,000 that have 2^-25.4 of the weight of one: not one of them is a float16
    number beside 1, and together they are the output."""
    n, seqs, big, value = 3000, 300, 64, 1000.0
    c = Case([n] * seqs, [new] * seqs, qh=4, kvh=1, dim=64, page=60, dtype=F16)
    c.q.zero_(); c.k.zero_(); c.v.fill_(value)
    c.q[..., 0] = 1.0
    c.k[..., 0] = -17.6
    first = c.table[:, :2].long()
    c.k[first[:, 0]], c.v[first[:, 0]] = 0.0, 0.0
    c.k[first[:, 1], : big - 60], c.v[first[:, 1], : big - 60] = 0.0, 0.0
    out, lse = c.cache.attend(c.q, c.table, c.kv_lens, cu_new=c.cu, scale=1.0)
    small = (torch.arange(n - new + 1, n + 1, device="cuda", dtype=torch.float64) - big) * math.exp(float(torch.tensor(-17.6, dtype=F16)))
    want, want_lse = (small / (big + small) * value).repeat(seqs)[:, None, None], (big + small).log().repeat(seqs)[:, None]
    # a probability is rounded to a multiple of 2^-24 where the largest is 2^7 or more, and the sum is at least 64 of those; the
    # sums run in 32 bits
    bound = n * 2.0 ** -32 * value / big + (1.05 * UNIT[F16] + n * 2.0 ** -23) * want
    assert bool((out.double() - want).abs().le(bound).all()), float(((out.double() - want).abs() / bound).max())
    assert bool((lse.double() - want_lse).abs().le(n * 2.0 ** -24 + 2.0 ** -20).all())
    assert c.cache.status() == 0


def test_a_scale_that_overflows_is_refused():
    """Times log2(e) a scale above 2.3e38 is infinite, and infinity times a score of 0 no number."""
    c = Case([100, 50], [1, 1], qh=4, kvh=2, dim=64)
    c.q.zero_()
    want, lse = c.cache.attend(c.q, c.table, c.kv_lens)
    got, _ = c.cache.attend(c.q, c.table, c.kv_lens, scale=1.9e38)
    assert torch.equal(got, want)
    for scale in (2.5e38, -2.5e38, math.inf):
        for call in (lambda: c.cache.attend(c.q, c.table, c.kv_lens, scale=scale), lambda: c.cache.weigh(c.q, lse, c.table, c.kv_lens, scale=scale)):
            with pytest.raises(GrandError, match="2e38"):
                call()

"""What of the token cache needs no GPU: argument checks ahead of any CUDA call, struct layouts, rotary tables."""
import ctypes as C
import math

import pytest
import torch

from paper_2608_21163_b200 import binding, cache

OK = dict(q_heads=8, kv_heads=2, head_dim=64, dtype=cache.BF16, page_size=16, weight_groups=2, num_pages=100)


@pytest.mark.parametrize("change,code", [
    (dict(q_heads=7), -1), (dict(q_heads=0), -1), (dict(kv_heads=0), -1), (dict(page_size=0), -1), (dict(page_size=(1 << 20) + 1), -1),
    (dict(num_pages=0), -1), (dict(num_pages=1 << 31), -1), (dict(weight_groups=3), -1), (dict(max_batch=4097), -1),
    (dict(max_tokens=1 << 29), -1), (dict(dtype=binding.F32), -6), (dict(dtype=binding.U8), -6), (dict(head_dim=60), -6), (dict(head_dim=136), -6),
    (dict(head_dim=0), -6)])
def test_creation_refuses_before_any_cuda_call(change, code):
    lib, h = cache._lib(), C.c_void_p()
    o = cache._Options(**{**OK, **change})
    assert lib.grand_cache_create(C.byref(o), C.byref(h)) == code and not h.value


def test_null_handles_and_arguments():
    lib, h = cache._lib(), C.c_void_p()
    assert lib.grand_cache_create(None, C.byref(h)) == -1 and lib.grand_cache_create(C.byref(cache._Options(**OK)), None) == -1
    assert lib.grand_cache_destroy(None) == 0
    assert lib.grand_cache_status(None, None, None) == -1 and lib.grand_cache_launches(None, None) == -1
    assert lib.grand_cache_append(None, None, None, None, None, None, None, None, None, 0, 0, None, 0, None) == -1
    assert lib.grand_cache_attend(None, None, None, None, 0, 0, 1.0, 1, 0, None, None, None) == -1
    assert lib.grand_cache_weigh(None, None, None, None, 0, 0, None, 1.0, 1, 0, 1.0, None) == -1
    assert lib.grand_cache_evict(None, None, None, 1, 0, 0, None, 0, 0, None, None, None) == -1
    assert lib.grand_cache_last_error(None) == b""


def test_rope_refuses_before_any_cuda_call():
    lib = cache._lib()
    rope = lambda dtype=cache.BF16, tokens=4, heads=2, dim=64, rot=64, table=None: lib.grand_rope(  # noqa: E731
        None, None, dtype, tokens, heads, dim, 128, 64, 128, 64, table, 16, rot, None, 0, 0, None)
    assert rope(dtype=binding.U8) == -6 and rope(dim=257) == -6 and rope(dim=0) == -6
    assert rope(rot=63) == -1 and rope(rot=66) == -1 and rope() == -1        # odd, longer than the head, no table
    assert rope(tokens=1 << 31) == -2
    assert rope(tokens=0) == 0 and rope(heads=0) == 0


def test_struct_layouts_match_the_header():
    assert C.sizeof(cache._Options) == 8 * 4 + 8 + 3 * 8
    assert C.sizeof(cache._Pool) == 3 * 8 + 3 * 8
    assert C.sizeof(cache._Seqs) == 3 * 8 + 8 + 3 * 4 + 4
    # an index keeps no 16-bit vectors
    lib, h = binding.load(), C.c_void_p()
    for dtype in (cache.F16, cache.BF16):
        assert lib.grand_create(C.c_uint32(8), C.c_uint32(dtype), C.c_uint32(0), C.c_uint32(8), C.c_uint32(16), C.c_float(1.2), C.byref(h)) == -1


def test_rope_table_is_exact_far_out():
    f = cache.rope_frequencies(8, base=500.0)
    t = cache.rope_table(100_001, f, magnitude=1.25, device="cpu")
    assert t.shape == (100_001, 8) and t.dtype == torch.float32
    for p in (0, 1, 777, 100_000):
        for i in range(4):
            angle = p * 500.0 ** (-2 * i / 8)
            # a float64 angle of 100,000 is off by 1.5e-11 at most, the table's rounding by 2^-24 of 1.25
            assert abs(float(t[p, i]) - 1.25 * math.cos(angle)) < 1e-7 and abs(float(t[p, 4 + i]) - 1.25 * math.sin(angle)) < 1e-7
    with pytest.raises(ValueError):
        cache.rope_frequencies(7)


def test_a_collected_cache_waits_for_nobody():
    """Its handle is destroyed with the next object that is made or closed, not by the collection."""
    class Lib:
        gone = []

        def grand_cache_destroy(self, h):
            self.gone.append(h)

    def made(h):
        c = cache.TokenCache.__new__(cache.TokenCache)
        c.lib, c.h = Lib(), h
        return c

    before = list(cache._collected)
    cache._collected.clear()
    a, b, c = made(1), made(2), made(3)
    del a, b
    assert Lib.gone == [] and sorted(cache._collected) == [1, 2]
    c.close()
    assert sorted(Lib.gone) == [1, 2, 3] and not cache._collected
    c.close()
    del c
    assert len(Lib.gone) == 3 and not cache._collected
    del made
    cache.TokenCache.__new__(cache.TokenCache).__del__()   # an object that was never made
    cache._collected.extend(before)

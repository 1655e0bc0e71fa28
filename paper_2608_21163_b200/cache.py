"""Token cache: rotary positions, attention over a paged cache of keys and values, and its eviction by attention weight.

Argument marshalling only, like `binding`: every step runs in the CUDA library (include/grand.h, second half), on the
current stream, asynchronously.  The caller owns the pool and the tables, so any allocator of pages fits; a page of one
token makes the page table a list of rows, such as the ids that GrandIndex.search returned.
"""
import ctypes as C
import math

import torch

from .binding import F32, GrandError, load

F16, BF16 = 3, 4
_DTYPE = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}


class _Options(C.Structure):
    _fields_ = [("q_heads", C.c_uint32), ("kv_heads", C.c_uint32), ("head_dim", C.c_uint32), ("dtype", C.c_uint32),
                ("page_size", C.c_uint32), ("weight_groups", C.c_uint32), ("max_batch", C.c_uint32), ("max_tokens", C.c_uint32),
                ("num_pages", C.c_uint64), ("dev_alloc", C.c_void_p), ("dev_free", C.c_void_p), ("user", C.c_void_p)]


class _Pool(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("weights", C.c_void_p),
                ("page_stride", C.c_int64), ("slot_stride", C.c_int64), ("head_stride", C.c_int64)]


class _Seqs(C.Structure):
    _fields_ = [("page_table", C.c_void_p), ("kv_lens", C.c_void_p), ("cu_new", C.c_void_p), ("table_stride", C.c_int64),
                ("pages_per_seq", C.c_uint32), ("batch", C.c_uint32), ("tokens", C.c_uint32)]


_ready = None


def _lib():
    global _ready
    if _ready is None:
        lib = load()
        p, u32, u64, i64, f = C.c_void_p, C.c_uint32, C.c_uint64, C.c_int64, C.c_float
        lib.grand_cache_create.argtypes = [p, p]
        lib.grand_cache_destroy.argtypes = [p]
        lib.grand_cache_status.argtypes = [p, p, p]
        lib.grand_cache_launches.argtypes = [p, p]
        lib.grand_rope.argtypes = [p, p, u32, u64, u32, u32, i64, i64, i64, i64, p, u64, u32, p, u32, u32, p]
        lib.grand_rope_checked.argtypes = lib.grand_rope.argtypes + [p]
        lib.grand_cache_append.argtypes = [p, p, p, p, p, p, p, p, p, u64, u32, p, u32, p]
        lib.grand_cache_attend.argtypes = [p, p, p, p, i64, i64, f, u32, u32, p, p, p]
        lib.grand_cache_weigh.argtypes = [p, p, p, p, i64, i64, p, f, u32, u32, f, p]
        lib.grand_cache_evict.argtypes = [p, p, p, u32, u32, u32, p, i64, u32, p, p, p]
        _ready = lib
    return _ready


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _count(x, name):
    # ctypes would cut a number down to its low 32 bits
    if not 0 <= x < 1 << 32:
        raise ValueError(f"{name} must be a number from 0 below 2^32")
    return x


def _int32(t, length, name, device):
    if t.dtype != torch.int32 or t.get_device() != device or t.shape != (length,):
        raise ValueError(f"{name} must be an int32 tensor of {length} entries on CUDA device {device}")
    return t if t.is_contiguous() else t.contiguous()


def _table(t, name, device):
    if t.dtype == torch.uint32:   # ids as a search returns them; its padding becomes -1, which is no page either
        t = t.view(torch.int32)
    if t.dtype != torch.int32 or t.get_device() != device or t.dim() != 2:
        raise ValueError(f"{name} must be an int32 or uint32 matrix on CUDA device {device}")
    return t if t.stride(1) == 1 else t.contiguous()


def _stream(device):
    # current_stream(device).cuda_stream without the object around it, which takes longer to make than a kernel to launch
    return torch._C._cuda_getCurrentRawStream(device.index)


def _rows16(t):
    """x itself if its last dimension is dense and every row of it starts on 16 bytes, else a packed copy."""
    a, b, c = t.stride()
    return t if c == 1 and not (a % 8 or b % 8 or t.data_ptr() % 16) else t.clone(memory_format=torch.contiguous_format)


def rope_frequencies(rot, base=10000.0, factor=1.0, original_length=None, low=1.0, high=4.0):
    """Angles per position of the rot / 2 pairs (float64).  factor > 1 stretches them for long contexts: all of them where
    original_length is None, else by wavelength - pairs that turn more than `high` times over the original length keep
    their frequency, those that turn less than `low` times are divided by factor, and in between a linear blend."""
    _need(rot > 0 and rot % 2 == 0, "rot must be even")
    f = base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    if factor == 1.0:
        return f
    if original_length is None:
        return f / factor
    turns = original_length * f / (2 * math.pi)
    keep = ((turns - low) / (high - low)).clamp(0, 1)
    return f * keep + f / factor * (1 - keep)


def rope_table(length, frequencies, magnitude=1.0, device="cuda"):
    """The table of `rope` and `append`: cosines, then sines, of every position below `length` (float32, from float64
    angles: a float32 product of position and frequency would be off by 0.01 at position 100,000).  magnitude scales
    both, as some long-context scalings ask for."""
    f = torch.as_tensor(frequencies, dtype=torch.float64, device=device)
    angle = torch.arange(length, dtype=torch.float64, device=device)[:, None] * f
    return torch.cat([angle.cos(), angle.sin()], 1).mul_(magnitude).float()


def _check_table(table, positions, tokens, device):
    if table.dtype != torch.float32 or table.get_device() != device or table.dim() != 2 or not table.is_contiguous():
        raise ValueError(f"table must be a dense float32 matrix on CUDA device {device}")
    return _int32(positions, tokens, "positions", device)


class _Rope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, table, positions, interleaved, inverse, status):
        ctx.save_for_backward(table, positions)
        ctx.interleaved, ctx.inverse = interleaved, inverse
        return rope(x, table, positions, interleaved, inverse, status=status)

    @staticmethod
    def backward(ctx, grad):
        return rope(grad, *ctx.saved_tensors, ctx.interleaved, not ctx.inverse), None, None, None, None, None


class _NoGradient(torch.autograd.Function):
    # Marks the results of a call that has no gradient: a backward pass through them raises instead of losing what was asked.
    @staticmethod
    def forward(ctx, name, results, *tensors):   # the results, then the inputs
        ctx.name = name
        ctx.mark_dirty(*tensors[:results])
        return tensors[:results]

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError(f"TokenCache.{ctx.name} has no gradient")


def _wants_gradient(*tensors):
    for t in tensors:
        if t.requires_grad:
            return torch.is_grad_enabled()
    return False


def rope(x, table, positions, interleaved=False, inverse=False, out=None, status=None):
    """Rotary positions of x [tokens, heads, dim] (float16, bfloat16 or float32, any token and head strides): the first
    table.shape[1] entries of every head are turned by their token's angles, the others copied.  Pairs are (i, i + rot / 2),
    or (2i, 2i + 1) if interleaved.  inverse turns back, which is the gradient of the rotation and what a backward pass does where
    x requires one (out is refused then, and the table is a constant).  out may be x.  A position outside the table takes the
    nearest row of it; status, an int32 CUDA tensor of one entry, then gets bit 2 set (nothing clears it)."""
    if _wants_gradient(x, table):
        _need(out is None and not table.requires_grad, "rope gives a gradient to x alone, and not where out is given")
        return _Rope.apply(x, table, positions, interleaved, inverse, status)
    _need(x.is_cuda and x.dim() == 3 and x.dtype in _DTYPE, "x must be a CUDA tensor [tokens, heads, dim] of a supported type")
    positions = _check_table(table, positions, x.shape[0], x.get_device())
    if x.stride(2) != 1:
        x = x.contiguous()
    if out is None:
        out = torch.empty_like(x) if x.is_contiguous() else x.new_empty(x.shape)
    else:
        _need(out.shape == x.shape and out.dtype == x.dtype and out.device == x.device and out.stride(2) == 1, "out must be like x")
    if status is not None:
        status = _int32(status, 1, "status", x.get_device()).data_ptr()
    lib = _lib()
    rc = lib.grand_rope_checked(x.data_ptr(), out.data_ptr(), _DTYPE[x.dtype], x.shape[0], x.shape[1], x.shape[2], x.stride(0), x.stride(1),
                                out.stride(0), out.stride(1), table.data_ptr(), table.shape[0], table.shape[1], positions.data_ptr(),
                                interleaved, inverse, status, _stream(x.device))
    if rc != 0:
        raise GrandError(rc, lib.grand_strerror(rc).decode())
    return out


# Handles of collected objects.  To destroy one waits for the whole device, which a collection must not do at a time of its own
# choosing: it would stall every stream, and end a graph capture with an error.
_collected = []


def _destroy_collected(lib):
    while _collected:
        lib.grand_cache_destroy(_collected.pop())


class TokenCache:
    """Operators on one pool of pages, with their workspace.

    k_pages, v_pages: [pages, page size, kv heads, head dim], float16 or bfloat16, equal strides (a pool laid out
    [pages, kv heads, page size, head dim] is passed as its transpose(1, 2)).  weights: [pages, groups, page size] float32
    with groups 1 or kv heads, or None.  The methods run on the current stream; one object serves one stream at a time.

    Every method takes page_table [batch, pages per sequence] (int32, or the uint32 ids of a search) and kv_lens [batch] (int32), on
    the GPU: the tokens cached for each sequence, the new ones last among them.  At most max_batch sequences a call (4,096 is
    the limit) and max_tokens new tokens.  The new tokens' rows are packed over the batch; cu_new [batch + 1] (int32)
    says where each sequence's start, None means one new token per sequence.  Rows of no sequence are left as they are.

    The methods have no gradient (`rope` has): a backward pass through what append or attend returned raises, and out, lse and q_out are
    refused where one of the inputs requires a gradient.  What lies in the pool and its weights is never part of one.

    An object's workspace is four partial results an SM (39 MB on 148), whatever its sizes.  close() frees it; that of an object that
    was collected without is freed with the next object that is made or closed.
    """

    def __init__(self, k_pages, v_pages, weights=None, q_heads=None, max_batch=256, max_tokens=8192):
        _need(k_pages.is_cuda and k_pages.dim() == 4 and v_pages.shape == k_pages.shape and v_pages.dtype == k_pages.dtype
              and v_pages.device == k_pages.device, "k_pages and v_pages must be CUDA tensors [pages, page size, kv heads, head dim] of one type")
        _need(k_pages.stride() == v_pages.stride() and k_pages.stride(3) == 1, "k_pages and v_pages must have equal strides, dense along the head")
        pages, size, kv_heads, dim = k_pages.shape
        groups = 0
        if weights is not None:
            groups = weights.shape[1]
            _need(weights.dtype == torch.float32 and weights.device == k_pages.device and weights.is_contiguous()
                  and tuple(weights.shape) == (pages, groups, size) and groups in (1, kv_heads), "weights must be dense float32 [pages, 1 or kv heads, page size]")
        self.lib = _lib()
        _destroy_collected(self.lib)
        self.k_pages, self.v_pages, self.weights = k_pages, v_pages, weights
        self.q_heads, self.kv_heads, self.head_dim, self.page_size, self.groups = q_heads or kv_heads, kv_heads, dim, size, groups
        self.dtype, self.device, self.index = k_pages.dtype, k_pages.device, k_pages.get_device()
        _need(0 < self.q_heads < 1 << 32, "q_heads must be a positive number")
        max_batch, max_tokens = _count(max_batch, "max_batch"), _count(max_tokens, "max_tokens")
        o = _Options(q_heads=self.q_heads, kv_heads=kv_heads, head_dim=dim, dtype=_DTYPE.get(k_pages.dtype, 0), page_size=size,
                     weight_groups=groups, max_batch=max_batch, max_tokens=max_tokens, num_pages=pages)
        h = C.c_void_p()
        rc = self.lib.grand_cache_create(C.byref(o), C.byref(h))
        if rc != 0:
            raise GrandError(rc, self.lib.grand_strerror(rc).decode())
        self.h = h
        st = k_pages.stride()
        self._pool = _Pool(k_pages.data_ptr(), v_pages.data_ptr(), weights.data_ptr() if groups else None, st[0], st[1], st[2])
        self._pool_at = C.byref(self._pool)
        self._seqs = _Seqs()
        self._seqs_at = C.byref(self._seqs)
        self._strides = (C.c_int64 * 6)()

    def close(self):
        """Frees the workspace, and those of collected objects, once the device is idle."""
        if getattr(self, "h", None):
            self.lib.grand_cache_destroy(self.h)
            self.h = None
            _destroy_collected(self.lib)

    def __del__(self):
        if getattr(self, "h", None):
            _collected.append(self.h)
            self.h = None

    def _check(self, rc):
        if rc != 0:
            raise GrandError(rc, self.lib.grand_cache_last_error(self.h).decode() or self.lib.grand_strerror(rc).decode())

    def _sequences(self, page_table, kv_lens, cu_new, tokens):
        """Fills the call's description; returns what has to live until the call is made."""
        page_table = _table(page_table, "page_table", self.index)
        batch, per = page_table.shape
        kv_lens = _int32(kv_lens, batch, "kv_lens", self.index)
        if cu_new is not None:
            cu_new = _int32(cu_new, batch + 1, "cu_new", self.index)
        s = self._seqs
        s.page_table, s.kv_lens, s.cu_new = page_table.data_ptr(), kv_lens.data_ptr(), None if cu_new is None else cu_new.data_ptr()
        s.table_stride, s.pages_per_seq, s.batch, s.tokens = page_table.stride(0), per, batch, tokens
        return page_table, kv_lens, cu_new

    def _heads(self, x, heads, name, tokens=None):
        shape = x.shape
        if (x.dtype != self.dtype or x.device != self.device or len(shape) != 3 or shape[1] != heads or shape[2] != self.head_dim
                or (tokens is not None and shape[0] != tokens)):
            raise ValueError(f"{name} must be [tokens, {heads}, {self.head_dim}] of the cache's type and on its device")
        return x

    def append(self, q, k, v, table, positions, page_table, kv_lens, cu_new=None, interleaved=False, q_out=None):
        """New tokens enter the cache: k [tokens, kv heads, dim] is turned (see `rope`) and written with v into the last slots
        of its sequences, whose weights become 0; returns q [tokens, q heads, dim] turned, or None if q is None.  table None:
        no rotation."""
        tokens = k.shape[0]
        k, v = self._heads(k, self.kv_heads, "k"), self._heads(v, self.kv_heads, "v", tokens)
        k, v = (x if x.stride(2) == 1 else x.contiguous() for x in (k, v))
        if q is not None:
            q = self._heads(q, self.q_heads, "q", tokens)
            q = q if q.stride(2) == 1 else q.contiguous()
            wants = _wants_gradient(q, k, v)
            if q_out is None:
                q_out = torch.empty_like(q) if q.is_contiguous() else q.new_empty(q.shape)
            else:
                _need(q_out.shape == q.shape and q_out.dtype == q.dtype and q_out.device == q.device and q_out.is_contiguous(), "q_out must be dense and like q")
                _need(not wants, "append has no gradient")
        if table is not None:
            positions = _check_table(table, positions, tokens, self.index)
        hold = self._sequences(page_table, kv_lens, cu_new, tokens)
        strides = self._strides
        if q is not None:
            strides[0], strides[1], _ = q.stride()
        strides[2], strides[3], _ = k.stride()
        strides[4], strides[5], _ = v.stride()
        self._check(self.lib.grand_cache_append(
            self.h, self._pool_at, self._seqs_at, None if q is None else q.data_ptr(), None if q is None else q_out.data_ptr(), k.data_ptr(),
            v.data_ptr(), strides, None if table is None else table.data_ptr(), 0 if table is None else table.shape[0],
            0 if table is None else table.shape[1], None if table is None else positions.data_ptr(), interleaved,
            _stream(self.device)))
        del hold
        if q is not None and wants:
            (q_out,) = _NoGradient.apply("append", 1, q_out, q, k, v)
        return None if q is None else q_out

    def attend(self, q, page_table, kv_lens, cu_new=None, scale=None, causal=True, window=0, out=None, lse=None):
        """softmax(scale q k) v of the new tokens' queries q [tokens, q heads, dim] over their sequences: new token i of m, with
        n tokens cached, sees token j if j <= n - m + i (causal) and, with a window, j > n - m + i - window.  scale defaults to
        1 / sqrt(dim).  Returns the output, like q, and the log of every row's sum [tokens, q heads]; a row that sees nothing
        gives 0 and -inf."""
        wants = _wants_gradient(q)
        _need(not wants or (out is None and lse is None), "attend has no gradient")
        q = _rows16(self._heads(q, self.q_heads, "q"))
        shape = q.shape
        if out is None:
            out = torch.empty_like(q) if q.is_contiguous() else q.new_empty(shape)
        else:
            _need(out.shape == shape and out.dtype == q.dtype and out.device == q.device and out.is_contiguous(), "out must be dense and like q")
        if lse is None:
            lse = q.new_empty(shape[:2], dtype=torch.float32)
        else:
            _need(lse.shape == shape[:2] and lse.dtype == torch.float32 and lse.device == q.device and lse.is_contiguous(),
                  "lse must be dense float32 [tokens, q heads]")
        hold = self._sequences(page_table, kv_lens, cu_new, shape[0])
        self._check(self.lib.grand_cache_attend(
            self.h, self._pool_at, self._seqs_at, q.data_ptr(), q.stride(0), q.stride(1), self.head_dim ** -0.5 if scale is None else scale,
            causal, _count(window, "window"), out.data_ptr(), lse.data_ptr(), _stream(self.device)))
        del hold
        return _NoGradient.apply("attend", 2, out, lse, q) if wants else (out, lse)

    def weigh(self, q, lse, page_table, kv_lens, cu_new=None, scale=None, causal=True, window=0, decay=1.0):
        """Adds to every cached token's weight (times decay) the attention that the queries q pay it; lse is what `attend`
        returned for them with the same arguments.  The sequences of a call must not share pages.  Returns the weights."""
        q = _rows16(self._heads(q, self.q_heads, "q"))
        _need(lse.shape == q.shape[:2] and lse.dtype == torch.float32 and lse.device == q.device, "lse must be float32 [tokens, q heads]")
        lse = lse if lse.is_contiguous() else lse.contiguous()
        hold = self._sequences(page_table, kv_lens, cu_new, q.shape[0])
        self._check(self.lib.grand_cache_weigh(
            self.h, self._pool_at, self._seqs_at, q.data_ptr(), q.stride(0), q.stride(1), lse.data_ptr(),
            self.head_dim ** -0.5 if scale is None else scale, causal, _count(window, "window"), decay, _stream(self.device)))
        del hold
        return self.weights

    def evict(self, page_table, kv_lens, keep, sinks=0, recent=0, into=None):
        """Brings every sequence down to `keep` tokens: its first `sinks`, its last `recent` and the heaviest of the others (ties:
        the lowest index), moved together in their order, in place or into the pages of the table `into` (other pages than
        the sequences').  Tokens without a page are not kept.  Returns the kept tokens' indices [batch, groups, keep], -1 behind
        the last, and the new lengths."""
        keep, sinks, recent = _count(keep, "keep"), _count(sinks, "sinks"), _count(recent, "recent")
        hold = self._sequences(page_table, kv_lens, None, page_table.shape[0])
        batch = page_table.shape[0]
        if into is not None:
            into = _table(into, "into", self.index)
            _need(into.shape[0] == batch, "into must have a row per sequence")
        kept = page_table.new_empty((batch, max(1, self.groups), keep), dtype=torch.int32)
        lens = page_table.new_empty(batch, dtype=torch.int32)
        self._check(self.lib.grand_cache_evict(
            self.h, self._pool_at, self._seqs_at, keep, sinks, recent, None if into is None else into.data_ptr(),
            0 if into is None else into.stride(0), 0 if into is None else into.shape[1], kept.data_ptr(), lens.data_ptr(),
            _stream(self.device)))
        del hold
        return kept, lens

    def status(self):
        """What the calls since the last one found wrong in device data (bits of grand_cache_status); waits for the stream."""
        bits = C.c_uint32()
        self._check(self.lib.grand_cache_status(self.h, C.byref(bits), _stream(self.device)))
        return bits.value

    @property
    def launches(self):
        n = C.c_uint64()
        self._check(self.lib.grand_cache_launches(self.h, C.byref(n)))
        return n.value

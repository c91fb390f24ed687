"""The paged key-value caches over PyTorch tensors.

A `PagedCache` holds the pages and the page table of one layer; its calls
append rows to the pages and attend over them (include/gvc.h, "paged cache",
says what each computes).  A `QuantPagedCache` has the same calls over pages of
8 bits ("quantised paged cache"), and reads rows back in 16.  PyTorch provides
memory and streams; every computation is a call into libgvc on the current
stream of the cache's GPU, asynchronous and fit for capture into a graph.  There
are no derivatives:
tensors that require a gradient are refused unless autograd is off
(`torch.no_grad()`; pages and outputs always), and so are duals of forward mode.

    cache = PagedCache.empty(n_pages, page_size, n_kv_heads, head_dim, n_seqs, max_pages)
    q = cache.append(q, k, v, row_seq, row_slot, rope_pairs=(16, 24, 24), positions=thw)
    o = cache.prefill(q, row_slot, row_begin)            # the rows of a prompt
    o = cache.decode(q, lengths, window=4096, sinks=4)   # one new token per sequence

    cache = QuantPagedCache.empty(n_pages, page_size, n_kv_heads, head_dim, n_seqs, max_pages)
    q = cache.append(q, k, v, row_seq, row_slot)         # and prefill and decode, as above
    k, v = cache.read(row_seq, row_slot)                 # rows back in 16 bits
"""
import torch
from torch.autograd import forward_ad

from . import gvc

_DTYPES = {torch.bfloat16: gvc.BF16, torch.float16: gvc.FP16}

# Descriptors (by query heads) and workspace sizes (by a call's numbers) of each
# shape of cache: making one costs more than a short call's other checks together.
_shapes = {}
_KEPT = 4096

_INT = 2 ** 31   # numbers from here on would reach the C call cut to 32 bits


def _kept(store, key, make):
    value = store.get(key)
    if value is None:
        if len(store) >= _KEPT:
            store.clear()
        value = store[key] = make()
    return value


def _no_tangents(*tensors):
    """Refuses duals, whose tangents would be lost (called within a level of forward mode only)."""
    if any(t is not None and forward_ad.unpack_dual(t).tangent is not None for t in tensors):
        raise ValueError("tensors with a tangent of forward mode: the paged cache has no derivatives")


def _address(t):
    return (None, 0) if t is None else (t.data_ptr(), t.numel())


class PagedCache:
    """Pages k_pages [n_pages][n_kv_heads][page_size][head_dim] and v_pages
    [n_pages][n_kv_heads][head_dim][page_size] (bfloat16 or float16) and
    page_table int32 [n_seqs][max_pages], all contiguous on one GPU.  The
    tensors stay the caller's: the table may be changed between calls."""

    _append, _decode = staticmethod(gvc.paged_append), staticmethod(gvc.paged_decode)
    _prefill, _workspace_size = staticmethod(gvc.paged_prefill), staticmethod(gvc.paged_workspace)

    def __init__(self, k_pages, v_pages, page_table):
        dtype = k_pages.dtype
        if dtype not in _DTYPES or v_pages.dtype != dtype:
            raise ValueError("pages must be bfloat16 or float16, both alike")
        if k_pages.dim() != 4:
            raise ValueError("k_pages must be [n_pages][n_kv_heads][page_size][head_dim]")
        n_pages, kv, page, dh = k_pages.shape
        if v_pages.shape != (n_pages, kv, dh, page):
            raise ValueError("v_pages must be [n_pages][n_kv_heads][head_dim][page_size]")
        if page_table.dtype != torch.int32 or page_table.dim() != 2:
            raise ValueError("page_table must be int32 [n_seqs][max_pages]")
        if k_pages.requires_grad or v_pages.requires_grad:
            raise ValueError("pages must not require a gradient")
        if forward_ad._current_level >= 0:
            _no_tangents(k_pages, v_pages)
        if not (k_pages.is_contiguous() and v_pages.is_contiguous() and page_table.is_contiguous()):
            raise ValueError("pages and page table must be contiguous")
        index = k_pages.get_device()
        if index < 0 or v_pages.get_device() != index or page_table.get_device() != index:
            raise ValueError("pages and page table must be on one GPU")
        self._hold(k_pages, v_pages, page_table, dtype, index, False)

    def _hold(self, k_pages, v_pages, page_table, dtype, index, quant):
        self.k_pages, self.v_pages, self.page_table = k_pages, v_pages, page_table
        self.n_seqs, columns = page_table.shape
        shape = k_pages.shape
        self.n_kv_heads, self.head_dim = shape[1], shape[3]
        self._dtype, self._index = dtype, index
        self._shape = (dtype, *shape, self.n_seqs, columns)
        self._descs, self._sizes = _kept(_shapes, (quant, self._shape), lambda: ({}, {}))

    @property
    def device(self):
        return self.k_pages.device

    @classmethod
    def empty(cls, n_pages, page_size, n_kv_heads, head_dim, n_seqs, max_pages, dtype=torch.bfloat16, device="cuda"):
        """A cache of its own memory, no page of it in the table yet (every entry -1)."""
        k = torch.zeros(n_pages, n_kv_heads, page_size, head_dim, dtype=dtype, device=device)
        v = torch.zeros(n_pages, n_kv_heads, head_dim, page_size, dtype=dtype, device=device)
        return cls(k, v, torch.full((n_seqs, max_pages), -1, dtype=torch.int32, device=device))

    def append(self, q, k, v, row_seq, row_slot, *, positions=None, rope_pairs=None, rope_theta=10000.0, q_norm=None,
               k_norm=None, rms_eps=1e-5, q_out=None):
        """Writes k (normalised and rotated) and v [rows][n_kv_heads][head_dim]
        into slot row_slot[r] of sequence row_seq[r] (int32) and returns q
        [rows][n_heads][head_dim] normalised and rotated (None for q None).
        rope_pairs: rotated pairs of each axis, at most three (default: the
        whole head on one axis; () rotates nothing); positions: int32
        [axes][rows], default the slots.  q_out may be q itself."""
        if forward_ad._current_level >= 0:
            _no_tangents(q, k, v, q_norm, k_norm, q_out)
        kv = self.n_kv_heads
        n, ks = self._rows(k, "k", kv)
        m, vs = self._rows(v, "v", kv)
        if m != n:
            raise ValueError("k and v must have the same rows")
        self._ints(row_seq, "row_seq", n)
        self._ints(row_slot, "row_slot", n)
        pairs = (self.head_dim // 2,) if rope_pairs is None else tuple(rope_pairs)
        if len(pairs) > 3 or pairs and not -_INT <= min(pairs) <= max(pairs) < _INT:
            raise ValueError("rope_pairs has at most three axes, each a number of 32 bits")
        where = None
        if positions is not None:
            if (positions.dtype != torch.int32 or positions.get_device() != self._index or
                    positions.shape != (len(pairs), n) or not positions.is_contiguous()):
                raise ValueError("positions must be contiguous int32 [axes][rows]")
            where = positions.data_ptr()
        rope = gvc.PagedRope(pairs, rope_theta, rms_eps, self._gain(q_norm, "q_norm"), self._gain(k_norm, "k_norm"),
                             where, n)
        if q is None:
            if q_out is not None:
                raise ValueError("q_out without q")
            heads, qp, qs, op, os = kv, None, 0, None, 0
        else:
            heads, m, qs, q_out, os = self._q_out(q, q_out)
            if m != n:
                raise ValueError("q and k must have the same rows")
            qp, op = q.data_ptr(), q_out.data_ptr()
        self._call(self._append, self._desc(heads), rope, qp, qs, k.data_ptr(), ks, v.data_ptr(), vs,
                   row_seq.data_ptr(), row_slot.data_ptr(), n, *self._pages(), op, os)
        return q_out

    def decode(self, q, lengths, *, scale=None, window=0, sinks=0, out=None):
        """Attention of one token per sequence: q [n_seqs][n_heads][head_dim],
        row s over the first lengths[s] slots (int32; 0: an idle slot of the
        batch, zeros).  scale: default head_dim^-1/2.  out may be q itself."""
        if forward_ad._current_level >= 0:
            _no_tangents(q, out)
        heads, n, qs, out, os = self._q_out(q, out)
        if n != self.n_seqs:
            raise ValueError("q must have one row per sequence")
        self._ints(lengths, "lengths", n)
        desc = self._desc(heads)
        work = self._workspace(desc, heads, False, n, window, sinks)
        self._call(self._decode, desc, self.head_dim ** -0.5 if scale is None else scale, window, sinks, q.data_ptr(),
                   qs, lengths.data_ptr(), *self._pages(), out.data_ptr(), os, *_address(work))
        return out

    def prefill(self, q, row_last, row_begin, *, scale=None, window=0, sinks=0, out=None):
        """Attention of rows q [rows][n_heads][head_dim]: rows row_begin[s] to
        row_begin[s + 1] - 1 (int32 [n_seqs + 1]) are sequence s's, and row r
        sees slots up to row_last[r] (int32; -1: none).  Rows of no sequence
        are left as they are in `out` (undefined in a new one), which may be q
        itself."""
        if forward_ad._current_level >= 0:
            _no_tangents(q, out)
        heads, n, qs, out, os = self._q_out(q, out)
        self._ints(row_last, "row_last", n)
        self._ints(row_begin, "row_begin", self.n_seqs + 1)
        desc = self._desc(heads)
        work = self._workspace(desc, heads, True, n, window, sinks)
        self._call(self._prefill, desc, self.head_dim ** -0.5 if scale is None else scale, window, sinks,
                   q.data_ptr(), qs, row_last.data_ptr(), row_begin.data_ptr(), n, *self._pages(), out.data_ptr(), os,
                   *_address(work))
        return out

    def check(self, lengths=None, row_seq=None, row_slot=None):
        """Raises GvcError where the page table, lengths or rows to be appended
        name a place that does not exist, or two rows the same one.  Copies
        them to the host: a debugging aid, not for the serving loop."""
        host = [t if t is None else t.to("cpu") for t in (self.page_table, lengths, row_seq, row_slot)]
        # wider numbers than the calls take: to places as far outside
        host = [t if t is None else t.to(torch.int64).clamp(-_INT, _INT - 1).to(torch.int32).contiguous() for t in host]
        if (row_seq is None) != (row_slot is None):
            raise ValueError("row_seq and row_slot come together")
        if lengths is not None and lengths.numel() != self.n_seqs:
            raise ValueError("lengths must have one entry per sequence")
        if row_seq is not None and row_seq.numel() != row_slot.numel():
            raise ValueError("row_seq and row_slot must have the same rows")
        gvc.paged_check(self._desc(self.n_kv_heads), *(None if t is None else t.data_ptr() for t in host),
                        0 if row_seq is None else row_seq.numel())

    # ---- argument checks and marshalling
    def _pages(self):
        """Addresses of the pages and the page table."""
        return self.k_pages.data_ptr(), self.v_pages.data_ptr(), self.page_table.data_ptr()

    def _desc(self, heads):
        """The descriptor for this many query heads."""
        desc = self._descs.get(heads)
        if desc is None:
            dtype, n_pages, kv, page, dh, n_seqs, columns = self._shape
            if max(n_pages, kv, page, dh, n_seqs, columns, heads) >= _INT:
                raise ValueError("dimensions of pages and page table must fit 32 bits")
            desc = gvc.PagedDesc(_DTYPES[dtype], heads, kv, dh, page, n_pages, n_seqs, columns)
            self._descs[heads] = desc
        return desc

    def _workspace(self, desc, heads, prefill, n, window, sinks):
        """Workspace for one call (None: none needed), from the caching
        allocator: it is this call's alone on any stream and in any graph."""
        key = (heads, prefill, n, window, sinks)
        size = self._sizes.get(key)
        if size is None:
            if not (-_INT <= window < _INT and -_INT <= sinks < _INT):
                raise ValueError("window and sinks must fit 32 bits")
            size = _kept(self._sizes, key, lambda: self._workspace_size(desc, prefill, n, window, sinks))
        return torch.empty(size, dtype=torch.uint8, device=self.k_pages.device) if size else None

    def _rows(self, t, name, heads):
        """(rows, row stride) of t [rows][heads][head_dim]."""
        shape = t.shape
        if t.dtype != self._dtype or t.get_device() != self._index or len(shape) != 3 or (
                t.requires_grad and torch.is_grad_enabled()):
            raise ValueError(name + " must be [rows][heads][head_dim] of the pages' type and device, without gradient")
        n, h, dh = shape
        rs, hs, es = t.stride()
        if h != heads or dh != self.head_dim or h < 1 or n >= _INT or (n and (es != 1 or (h > 1 and hs != dh))):
            raise ValueError(name + " must be [rows][heads][head_dim] with dense heads")
        return n, rs if n > 1 else h * dh

    def _ints(self, t, name, n):
        if t.dtype != torch.int32 or t.get_device() != self._index or t.shape != (n,) or (n > 1 and t.stride(0) != 1):
            raise ValueError("%s must be a contiguous int32 vector of %d on the cache's GPU" % (name, n))

    def _gain(self, t, name):
        if t is None:
            return None
        if (t.dtype != self._dtype or t.get_device() != self._index or t.shape != (self.head_dim,) or t.stride(0) != 1 or
                t.requires_grad and torch.is_grad_enabled()):
            raise ValueError(name + " must be a contiguous vector of head_dim of the pages' type and device, without "
                             "gradient")
        return t.data_ptr()

    def _q_out(self, q, out):
        """(heads, rows, row stride, output, its row stride) of q and the given or a new output."""
        heads = q.shape[1] if q.dim() == 3 else 0
        n, qs = self._rows(q, "q", heads)
        if out is None:
            # contiguous, whatever q's strides
            return heads, n, qs, torch.empty_like(q, memory_format=torch.contiguous_format), heads * self.head_dim
        m, os = self._rows(out, "the output", heads)
        if m != n or out.requires_grad:
            raise ValueError("the output must have q's rows and not require a gradient")
        return heads, n, qs, out, os

    def _call(self, f, *args):
        """f on the current stream of the cache's GPU."""
        if torch._C._cuda_getDevice() != self._index:
            with torch.cuda.device(self._index):
                return f(*args, torch._C._cuda_getCurrentRawStream(self._index))
        return f(*args, torch._C._cuda_getCurrentRawStream(self._index))


class QuantPagedCache(PagedCache):
    """A paged cache of 8 bits: codes k_pages [n_pages][n_kv_heads][page_size][head_dim]
    and v_pages [n_pages][n_kv_heads][head_dim][page_size] (float8_e4m3fn), a scale
    for each head of a slot in k_scales and v_scales [n_pages][n_kv_heads][page_size]
    (float8_e8m0fnu: powers of two), and page_table as in PagedCache.  A head of a slot
    is its codes times its scale in `dtype` (bfloat16 or float16), which is also the
    type of q, k, v and outputs; `append` quantises k and v as it writes them."""

    _append, _decode = staticmethod(gvc.quant_append), staticmethod(gvc.quant_decode)
    _prefill, _workspace_size = staticmethod(gvc.quant_prefill), staticmethod(gvc.quant_workspace)

    def __init__(self, k_pages, k_scales, v_pages, v_scales, page_table, dtype=torch.bfloat16):
        if dtype not in _DTYPES:
            raise ValueError("dtype must be bfloat16 or float16")
        if k_pages.dtype != torch.float8_e4m3fn or v_pages.dtype != torch.float8_e4m3fn:
            raise ValueError("pages must be float8_e4m3fn")
        if k_scales.dtype != torch.float8_e8m0fnu or v_scales.dtype != torch.float8_e8m0fnu:
            raise ValueError("scales must be float8_e8m0fnu")
        shape = k_pages.shape
        if len(shape) != 4:
            raise ValueError("k_pages must be [n_pages][n_kv_heads][page_size][head_dim]")
        n_pages, kv, page, dh = shape
        if v_pages.shape != (n_pages, kv, dh, page):
            raise ValueError("v_pages must be [n_pages][n_kv_heads][head_dim][page_size]")
        if k_scales.shape != shape[:3] or v_scales.shape != shape[:3]:
            raise ValueError("scales must be [n_pages][n_kv_heads][page_size]")
        if page_table.dtype != torch.int32 or page_table.dim() != 2:
            raise ValueError("page_table must be int32 [n_seqs][max_pages]")
        if k_pages.requires_grad or k_scales.requires_grad or v_pages.requires_grad or v_scales.requires_grad:
            raise ValueError("pages and scales must not require a gradient")
        if forward_ad._current_level >= 0:
            _no_tangents(k_pages, k_scales, v_pages, v_scales)
        if not (k_pages.is_contiguous() and k_scales.is_contiguous() and v_pages.is_contiguous() and
                v_scales.is_contiguous() and page_table.is_contiguous()):
            raise ValueError("pages, scales and page table must be contiguous")
        index = k_pages.get_device()
        if index < 0 or not (k_scales.get_device() == v_pages.get_device() == v_scales.get_device() ==
                             page_table.get_device() == index):
            raise ValueError("pages, scales and page table must be on one GPU")
        self.k_scales, self.v_scales = k_scales, v_scales
        self._hold(k_pages, v_pages, page_table, dtype, index, True)

    @classmethod
    def empty(cls, n_pages, page_size, n_kv_heads, head_dim, n_seqs, max_pages, dtype=torch.bfloat16, device="cuda"):
        """A cache of its own memory, no page of it in the table yet (every entry -1)."""
        def zeros(t, *shape):
            return torch.zeros(n_pages, n_kv_heads, *shape, dtype=torch.uint8, device=device).view(t)
        return cls(zeros(torch.float8_e4m3fn, page_size, head_dim), zeros(torch.float8_e8m0fnu, page_size),
                   zeros(torch.float8_e4m3fn, head_dim, page_size), zeros(torch.float8_e8m0fnu, page_size),
                   torch.full((n_seqs, max_pages), -1, dtype=torch.int32, device=device), dtype)

    def read(self, row_seq, row_slot, *, k_out=None, v_out=None):
        """(k, v) [rows][n_kv_heads][head_dim] of slots row_slot[r] of sequences
        row_seq[r] (int32) in 16 bits, zeros for a row whose place does not exist."""
        if forward_ad._current_level >= 0:
            _no_tangents(k_out, v_out)
        n, kv = row_seq.numel(), self.n_kv_heads
        self._ints(row_seq, "row_seq", n)
        self._ints(row_slot, "row_slot", n)
        if n >= _INT:
            raise ValueError("rows must fit 32 bits")
        (k_out, ks), (v_out, vs) = self._read_out(k_out, "k_out", n), self._read_out(v_out, "v_out", n)
        self._call(gvc.quant_read, self._desc(kv), row_seq.data_ptr(), row_slot.data_ptr(), n, *self._pages(),
                   k_out.data_ptr(), ks, v_out.data_ptr(), vs)
        return k_out, v_out

    def _read_out(self, out, name, n):
        """The given or a new output of n rows, and its row stride."""
        kv = self.n_kv_heads
        if out is None:
            return torch.empty(n, kv, self.head_dim, dtype=self._dtype, device=self.k_pages.device), kv * self.head_dim
        m, stride = self._rows(out, name, kv)
        if m != n or out.requires_grad:
            raise ValueError("%s must have a row for each of row_seq and not require a gradient" % name)
        return out, stride

    def _pages(self):
        return (self.k_pages.data_ptr(), self.k_scales.data_ptr(), self.v_pages.data_ptr(), self.v_scales.data_ptr(),
                self.page_table.data_ptr())

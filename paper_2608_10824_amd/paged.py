"""The paged key-value cache over PyTorch tensors.

A `PagedCache` holds the pages and the page table of one layer; its calls
append rows to the pages and attend over them (include/gvc.h, "paged cache",
says what each computes).  PyTorch provides memory and streams; every
computation is a call into libgvc on the current stream of the cache's GPU,
asynchronous and fit for capture into a graph.  There is no backward pass:
tensors that require a gradient are refused.

    cache = PagedCache.empty(n_pages, page_size, n_kv_heads, head_dim, n_seqs, max_pages)
    q = cache.append(q, k, v, row_seq, row_slot, rope_pairs=(16, 24, 24), positions=thw)
    o = cache.prefill(q, row_slot, row_begin)            # the rows of a prompt
    o = cache.decode(q, lengths, window=4096, sinks=4)   # one new token per sequence
"""
import ctypes

import torch

from . import gvc

_DTYPES = {torch.bfloat16: gvc.BF16, torch.float16: gvc.FP16}


def _need(ok, text):
    if not ok:
        raise ValueError(text)


def _address(t):
    return (None, 0) if t is None else (t.data_ptr(), t.numel())


class PagedCache:
    """Pages k_pages [n_pages][n_kv_heads][page_size][head_dim] and v_pages
    [n_pages][n_kv_heads][head_dim][page_size] (bfloat16 or float16) and
    page_table int32 [n_seqs][max_pages], all contiguous on one GPU.  The
    tensors stay the caller's: the table may be changed between calls."""

    def __init__(self, k_pages, v_pages, page_table):
        _need(k_pages.dtype in _DTYPES and v_pages.dtype == k_pages.dtype, "pages must be bfloat16 or float16, both alike")
        _need(k_pages.dim() == 4, "k_pages must be [n_pages][n_kv_heads][page_size][head_dim]")
        n_pages, kv, page, dh = k_pages.shape
        _need(v_pages.shape == (n_pages, kv, dh, page), "v_pages must be [n_pages][n_kv_heads][head_dim][page_size]")
        _need(page_table.dtype == torch.int32 and page_table.dim() == 2, "page_table must be int32 [n_seqs][max_pages]")
        _need(k_pages.is_contiguous() and v_pages.is_contiguous() and page_table.is_contiguous(),
              "pages and page table must be contiguous")
        self.device = k_pages.device
        _need(self.device.type == "cuda" and v_pages.device == self.device and page_table.device == self.device,
              "pages and page table must be on one GPU")
        self.k_pages, self.v_pages, self.page_table = k_pages, v_pages, page_table
        self.n_seqs = page_table.shape[0]
        self.n_kv_heads, self.head_dim = kv, dh
        self._desc = gvc.PagedDesc(_DTYPES[k_pages.dtype], kv, kv, dh, page, n_pages, self.n_seqs, page_table.shape[1])
        self._pages = (k_pages.data_ptr(), v_pages.data_ptr(), page_table.data_ptr())

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
        [axes][rows], default the slots."""
        n, ks = self._rows(k, "k", self.n_kv_heads)
        _need(self._rows(v, "v", self.n_kv_heads)[0] == n, "k and v must have the same rows")
        self._ints(row_seq, "row_seq", n)
        self._ints(row_slot, "row_slot", n)
        pairs = (self.head_dim // 2,) if rope_pairs is None else tuple(rope_pairs)
        _need(len(pairs) <= 3, "rope_pairs has at most three axes")
        rope = gvc.PagedRope((ctypes.c_int32 * 3)(*pairs), rope_theta, rms_eps, self._gain(q_norm, "q_norm"),
                             self._gain(k_norm, "k_norm"))
        if positions is not None:
            _need(positions.dtype == torch.int32 and positions.device == self.device and
                  positions.shape == (len(pairs), n) and positions.is_contiguous(),
                  "positions must be contiguous int32 [axes][rows]")
            rope.positions, rope.position_stride = positions.data_ptr(), n
        heads, qs, os, qp, op = self.n_kv_heads, 0, 0, None, None
        if q is None:
            _need(q_out is None, "q_out without q")
        else:
            heads = q.shape[1] if q.dim() == 3 else 0
            m, qs = self._rows(q, "q", heads)
            _need(m == n, "q and k must have the same rows")
            if q_out is None:
                q_out = torch.empty((n, heads, self.head_dim), dtype=q.dtype, device=self.device)
            m, os = self._rows(q_out, "q_out", heads)
            _need(m == n, "q_out must have q's rows")
            qp, op = q.data_ptr(), q_out.data_ptr()
        kp, vp, table = self._pages
        self._call(gvc.paged_append, self._with(heads), rope, qp, qs, k.data_ptr(), ks, v.data_ptr(), v.stride(0),
                   row_seq.data_ptr(), row_slot.data_ptr(), n, kp, vp, table, op, os)
        return q_out

    def decode(self, q, lengths, *, scale=None, window=0, sinks=0, out=None):
        """Attention of one token per sequence: q [n_seqs][n_heads][head_dim],
        row s over the first lengths[s] slots (int32; 0: an idle slot of the
        batch, zeros).  scale: default head_dim^-1/2."""
        heads, n, qs, out, os = self._q_out(q, out)
        _need(n == self.n_seqs, "q must have one row per sequence")
        self._ints(lengths, "lengths", n)
        desc = self._with(heads)
        work = self._workspace(desc, False, n, window, sinks)
        self._call(gvc.paged_decode, desc, self._scale(scale), window, sinks, q.data_ptr(), qs, lengths.data_ptr(),
                   *self._pages, out.data_ptr(), os,
                   *_address(work))
        return out

    def prefill(self, q, row_last, row_begin, *, scale=None, window=0, sinks=0, out=None):
        """Attention of rows q [rows][n_heads][head_dim]: rows row_begin[s] to
        row_begin[s + 1] - 1 (int32 [n_seqs + 1]) are sequence s's, and row r
        sees slots up to row_last[r] (int32; -1: none).  Rows of no sequence
        are left as they are in `out` (undefined in a new one)."""
        heads, n, qs, out, os = self._q_out(q, out)
        self._ints(row_last, "row_last", n)
        self._ints(row_begin, "row_begin", self.n_seqs + 1)
        desc = self._with(heads)
        work = self._workspace(desc, True, n, window, sinks)
        self._call(gvc.paged_prefill, desc, self._scale(scale), window, sinks, q.data_ptr(), qs, row_last.data_ptr(),
                   row_begin.data_ptr(), n, *self._pages, out.data_ptr(), os,
                   *_address(work))
        return out

    def check(self, lengths=None, row_seq=None, row_slot=None):
        """Raises GvcError where the page table, lengths or rows to be appended
        name a place that does not exist, or two rows the same one.  Copies
        them to the host: a debugging aid, not for the serving loop."""
        host = [None if t is None else t.to("cpu", torch.int32).contiguous()
                for t in (self.page_table, lengths, row_seq, row_slot)]
        _need((row_seq is None) == (row_slot is None), "row_seq and row_slot come together")
        _need(lengths is None or lengths.numel() == self.n_seqs, "lengths must have one entry per sequence")
        _need(row_seq is None or row_seq.numel() == row_slot.numel(), "row_seq and row_slot must have the same rows")
        gvc.paged_check(self._desc, *(None if t is None else t.data_ptr() for t in host),
                        0 if row_seq is None else row_seq.numel())

    # ---- argument checks and marshalling
    def _with(self, heads):
        """The descriptor for this many query heads."""
        d = self._desc
        if d.n_heads != heads:
            d = gvc.PagedDesc(d.dtype, heads, d.n_kv_heads, d.head_dim, d.page_size, d.n_pages, d.n_seqs, d.max_pages)
        return d

    def _rows(self, t, name, heads):
        """(rows, row stride) of t [rows][heads][head_dim]."""
        if t.dtype != self.k_pages.dtype or t.device != self.device or t.dim() != 3 or t.requires_grad:
            raise ValueError(name + " must be [rows][heads][head_dim] of the pages' type and device, without gradient")
        n, h, dh = t.shape
        rs, hs, es = t.stride()
        if h != heads or dh != self.head_dim or h < 1 or (n and (es != 1 or (h > 1 and hs != dh))):
            raise ValueError(name + " must be [rows][heads][head_dim] with dense heads")
        return n, rs if n > 1 else h * dh

    def _ints(self, t, name, n):
        if t.dtype != torch.int32 or t.device != self.device or t.shape != (n,) or (n > 1 and t.stride(0) != 1):
            raise ValueError("%s must be a contiguous int32 vector of %d on the cache's GPU" % (name, n))

    def _gain(self, t, name):
        if t is None:
            return None
        if t.dtype != self.k_pages.dtype or t.device != self.device or t.shape != (self.head_dim,) or t.stride(0) != 1:
            raise ValueError(name + " must be a contiguous vector of head_dim of the pages' type and device")
        return t.data_ptr()

    def _q_out(self, q, out):
        heads = q.shape[1] if q.dim() == 3 else 0
        n, qs = self._rows(q, "q", heads)
        if out is None:
            out = torch.empty((n, heads, self.head_dim), dtype=q.dtype, device=self.device)
            return heads, n, qs, out, heads * self.head_dim
        m, os = self._rows(out, "out", heads)
        _need(m == n, "out must have q's rows")
        return heads, n, qs, out, os

    def _scale(self, scale):
        return self.head_dim ** -0.5 if scale is None else scale

    def _workspace(self, desc, prefill, n, window, sinks):
        """Workspace for one call (None: none needed), from the caching
        allocator: it is this call's alone on any stream and in any graph."""
        size = gvc.paged_workspace(desc, prefill, n, window, sinks)
        return torch.empty(size, dtype=torch.uint8, device=self.device) if size else None

    def _call(self, f, *args):
        if torch.cuda.current_device() != self.device.index:
            with torch.cuda.device(self.device):
                return f(*args, torch.cuda.current_stream().cuda_stream)
        return f(*args, torch.cuda.current_stream().cuda_stream)

"""Paged K/V caches of include/sd2.h on torch tensors: argument checks and marshalling only.

    cache = PagedCache.empty(n_pages=512, page_size=64, n_layers=32, n_kv_heads=8, head_dim=128,
                             max_seqs=16, max_pages=64)
    cache.reserve(first, last)                       # pages for the positions about to be written
    cache.append(k, v, lens, layer=l)                # this step's rows
    out = cache.attend(q, lens, layer=l)             # causal attention over them and all before
    cache.fork([0], [1])                             # sequence 1 goes on from sequence 0's pages
    cache.trim(lens)                                 # pages behind these lengths become free

Sequences are rows of the table; lens, first, last, keep, row_off are int32 tensors on the cache's
device (their values are not read here: the calls do not wait for the GPU).  Every call runs on the
current stream of that device.
"""
import ctypes
import math

import torch
from torch.autograd import forward_ad

from . import binding as B

DTYPES = {torch.float32: 0, torch.bfloat16: 1}
# the current stream of a device, as HIP's handle (torch's own shortcut to it where there is one: a
# microsecond less per call)
_stream_of = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)


def _need(ok, msg):
    if not ok:
        raise B.Sd2Error(msg)


def _tangent(t):
    """Whether t carries a forward-mode tangent (outside a dual level, which is quick to see, none does)."""
    return getattr(forward_ad, "_current_level", 0) >= 0 and forward_ad.unpack_dual(t).tangent is not None


class PagedCache:
    """k and v: contiguous [n_pages][n_layers][n_kv_heads][page_size][head_dim], float32 or bfloat16;
    table: contiguous int32 [max_seqs][max_pages], -1 where there is no page; refs: int32 [n_pages],
    the table entries that name each page.  The cache works on these tensors and keeps them."""

    def __init__(self, k, v, table, refs):
        _need(k.is_cuda and k.dim() == 5 and k.dtype in DTYPES, "k: a float32 or bfloat16 GPU tensor "
              "[n_pages][n_layers][n_kv_heads][page_size][head_dim]")
        _need(v.shape == k.shape and v.dtype == k.dtype and v.device == k.device, "v has to be like k")
        _need(k.is_contiguous() and v.is_contiguous(), "k and v have to be contiguous")
        _need(not any(t.requires_grad or _tangent(t) for t in (k, v)), "k and v: no gradients here (detach them)")
        self._int32(table, 2, "table", k.device)
        self._int32(refs, 1, "refs", k.device)
        n_pages, n_layers, n_kv, page, hd = k.shape
        _need(refs.numel() == n_pages, "refs: one for every page")
        self.k, self.v, self.table, self.refs = k, v, table, refs
        self.device, self.dtype = k.device, k.dtype
        self._index, self._sizes = k.device.index, {}
        self._unused = torch.empty(256, dtype=torch.uint8, device=k.device)  # workspace of calls that need none
        self.n_pages, self.n_layers, self.n_kv_heads, self.page_size, self.head_dim = n_pages, n_layers, n_kv, page, hd
        self.max_seqs, self.max_pages = table.shape
        self.lib = B.load()
        size = k.element_size()
        pages = B.Pages(page, n_pages, self.max_seqs, self.max_pages, table.data_ptr(), refs.data_ptr(), 2)
        for i, pool in enumerate((k, v)):
            pages.arrays[i] = B.PageArray(pool.data_ptr(), n_layers * n_kv, hd * size)
        self._pages = pages
        self._pages_ws = self.lib.sd2_pages_workspace_bytes(ctypes.byref(pages))
        _need(self._pages_ws > 0, "the cache's sizes are outside what sd2_pages takes")
        self._scale = 1.0 / math.sqrt(hd)
        layer = n_kv * page * hd
        self._kv = [B.PagedKv(k.data_ptr() + l * layer * size, v.data_ptr() + l * layer * size, n_layers * layer,
                              DTYPES[k.dtype], page, n_pages, n_kv, hd, self.max_pages, table.data_ptr())
                    for l in range(n_layers)]

    @classmethod
    def empty(cls, n_pages, page_size, n_layers, n_kv_heads, head_dim, max_seqs, max_pages, dtype=torch.bfloat16,
              device="cuda"):
        """A cache of free pages and no sequences."""
        shape = (n_pages, n_layers, n_kv_heads, page_size, head_dim)
        return cls(torch.empty(shape, dtype=dtype, device=device), torch.empty(shape, dtype=dtype, device=device),
                   torch.full((max_seqs, max_pages), -1, dtype=torch.int32, device=device),
                   torch.zeros(n_pages, dtype=torch.int32, device=device))

    # ---- checks ------------------------------------------------------------------------------------
    @staticmethod
    def _int32(t, dim, what, device):
        _need(isinstance(t, torch.Tensor) and t.dtype == torch.int32 and t.dim() == dim and t.device == device and
              t.is_contiguous(), f"{what}: a contiguous int32 tensor of {dim} dimension(s) on the cache's device")

    def _layer(self, layer):
        _need(isinstance(layer, int) and 0 <= layer < self.n_layers, f"layer {layer} of {self.n_layers}")
        return ctypes.byref(self._kv[layer])

    def _packed(self, t, what):
        """A tensor [rows][heads][head_dim] whose rows may be apart: its row stride."""
        _need(isinstance(t, torch.Tensor) and t.device == self.device and t.dtype == self.dtype and t.dim() == 3 and
              t.shape[2] == self.head_dim, f"{what}: [rows][heads][head_dim] of the cache's type, on its device")
        _need(not t.requires_grad or not torch.is_grad_enabled(), f"{what}: no gradients here (torch.no_grad(), or detach it)")
        _need(not _tangent(t), f"{what}: no forward-mode tangents here (take its primal)")
        if t.numel():
            _need(t.stride(2) == 1 and (t.shape[1] == 1 or t.stride(1) == self.head_dim),
                  f"{what}: heads and head dimension have to be contiguous")
        return t.stride(0) if t.shape[0] > 1 else t.shape[1] * self.head_dim

    def _rows(self, total, lens, row_off, max_rows):
        self._int32(lens, 1, "lens", self.device)
        n = lens.numel()
        _need(n <= self.max_seqs, f"{n} sequences, the table has {self.max_seqs}")
        if row_off is None:
            _need(n > 0 and total % n == 0 or total == 0, f"{total} rows do not divide into {n} sequences: row_off says which are whose")
            each = total // n if n else 0
            _need(max_rows is None or max_rows == each, f"max_rows {max_rows}, but {each} rows each")
            if each == 0:
                n = 0
            return B.PagedRows(n, max(each, 1), total if n else 0, None, lens.data_ptr())
        self._int32(row_off, 1, "row_off", self.device)
        _need(row_off.numel() == n + 1, "row_off: one more than lens")
        _need(max_rows is None or max_rows >= 1, "max_rows: at least 1")
        return B.PagedRows(n, max(total, 1) if max_rows is None else max_rows, total, row_off.data_ptr(), lens.data_ptr())

    def _seqs(self, what, *tensors):
        n = tensors[0].numel() if isinstance(tensors[0], torch.Tensor) else 0
        for t in tensors:
            self._int32(t, 1, what, self.device)
            _need(t.numel() == n, f"{what}: tensors of one length")
        _need(n <= self.max_seqs, f"{what}: {n} sequences, the table has {self.max_seqs}")
        return n

    def _workspace(self, nbytes):
        return torch.empty(nbytes, dtype=torch.uint8, device=self.device)

    def _call(self, fn, *args):
        """A C call on the current stream of the cache's device, which is the current one meanwhile."""
        if torch.cuda.current_device() == self._index:
            rc = fn(*args, _stream_of(self._index))
        else:
            with torch.cuda.device(self._index):
                rc = fn(*args, _stream_of(self._index))
        if rc:
            B.check(rc, None, fn.__name__)

    # ---- rows --------------------------------------------------------------------------------------
    def append(self, k, v, lens, layer=0, row_off=None, max_rows=None):
        """Write rows k, v [rows][n_kv_heads][head_dim] to their positions (sd2_paged_append): those of
        sequence b are the last ones of its lens[b] positions, rows row_off[b] .. row_off[b + 1] - 1, or
        without row_off an equal number for every sequence."""
        kv = self._layer(layer)
        ks, vs = self._packed(k, "k"), self._packed(v, "v")
        _need(k.shape == v.shape and k.shape[1] == self.n_kv_heads, "k and v: [rows][n_kv_heads][head_dim]")
        rows = self._rows(k.shape[0], lens, row_off, max_rows)
        self._call(self.lib.sd2_paged_append, kv, ctypes.byref(rows), k.data_ptr(), ks, v.data_ptr(), vs)

    def attend(self, q, lens, layer=0, row_off=None, max_rows=None, max_len=None, scale=None, out=None):
        """Causal attention of rows q [rows][heads][head_dim] over their sequences' pages
        (sd2_paged_attn), rows and positions as in append; returns out, like q.  scale: 1 / sqrt(head_dim)
        unless given; max_rows, max_len: the most rows and the largest length, where they are known (they
        decide how the work is split)."""
        kv = self._layer(layer)
        qs = self._packed(q, "q")
        heads = q.shape[1]
        _need(heads > 0 and heads % self.n_kv_heads == 0, f"{heads} heads on {self.n_kv_heads} KV heads")
        if out is None:
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
            os = heads * self.head_dim
        else:
            _need(isinstance(out, torch.Tensor) and out.shape == q.shape, "out has to be like q")
            _need(not q.numel() or out.data_ptr() != q.data_ptr(), "out must not be q")
            os = self._packed(out, "out")
        rows = self._rows(q.shape[0], lens, row_off, max_rows)
        if max_len is None:
            max_len = self.max_pages * self.page_size
        key = (heads, rows.nseq, rows.max_rows, rows.total_rows, row_off is None, max_len)
        nbytes = self._sizes.get(key)
        if nbytes is None:
            _need(1 <= max_len <= self.max_pages * self.page_size, f"max_len {max_len} of {self.max_pages} pages")
            nbytes = self.lib.sd2_paged_attn_workspace_bytes(kv, ctypes.byref(rows), heads, max_len)
            _need(nbytes > 0, "attend: sizes outside what sd2_paged_attn takes")
            if len(self._sizes) > 1000:
                self._sizes.clear()
            self._sizes[key] = nbytes
        # (the smallest size is that of calls without partial sums)
        ws = self._unused if nbytes == 256 else self._workspace(nbytes)
        self._call(self.lib.sd2_paged_attn, kv, ctypes.byref(rows), q.data_ptr(), qs, out.data_ptr(), os, heads,
                   self._scale if scale is None else scale, max_len, ws.data_ptr(), nbytes)
        return out

    # ---- pages -------------------------------------------------------------------------------------
    def reserve(self, first, last, keep=None):
        """Make positions first[b] .. last[b] - 1 writable (sd2_pages_reserve); returns granted, int32
        per sequence: last[b], or where the first page begins that could not be had."""
        n = self._seqs("first, last, keep", first, last, *(() if keep is None else (keep,)))
        granted = torch.empty_like(last)
        ws = self._workspace(self._pages_ws)
        self._call(self.lib.sd2_pages_reserve, ctypes.byref(self._pages), n, first.data_ptr(), last.data_ptr(),
                   None if keep is None else keep.data_ptr(), granted.data_ptr(), ws.data_ptr(), self._pages_ws)
        return granted

    def fork(self, src, dst):
        """Sequence dst[i] gives up its pages and takes those of src[i], shared (sd2_pages_fork; lists of
        ints)."""
        src, dst = list(src), list(dst)
        _need(len(src) == len(dst), "fork: as many src as dst")
        _need(all(0 <= b < self.max_seqs for b in src + dst), f"fork: the table has {self.max_seqs} sequences")
        n = len(src)
        arr = ctypes.c_int32 * max(n, 1)
        self._call(self.lib.sd2_pages_fork, ctypes.byref(self._pages), n, arr(*src), arr(*dst))

    def trim(self, lens):
        """Sequences 0 .. len(lens) - 1 keep the pages of their first lens[b] positions (sd2_pages_trim;
        a negative length: all)."""
        n = self._seqs("lens", lens)
        self._call(self.lib.sd2_pages_trim, ctypes.byref(self._pages), n, lens.data_ptr())

    def compact(self):
        """Move the pages in use to the front (sd2_pages_compact); returns their number, int32 [1]."""
        live = torch.empty(1, dtype=torch.int32, device=self.device)
        ws = self._workspace(self._pages_ws)
        self._call(self.lib.sd2_pages_compact, ctypes.byref(self._pages), live.data_ptr(), ws.data_ptr(), self._pages_ws)
        return live

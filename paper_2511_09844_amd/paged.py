"""Paged K/V caches of include/sd2.h on torch tensors: argument checks and marshalling only.  A call whose arguments are
plain cases of what it takes goes through csrc/torch_paged.cpp in one step; any other comes back from there, untouched, to
the checks here.

    cache = PagedCache.empty(n_pages=512, page_size=64, n_layers=32, n_kv_heads=8, head_dim=128,
                             max_seqs=16, max_pages=64)
    cache.reserve(first, last)                       # pages for the positions about to be written
    cache.append(k, v, lens, layer=l)                # this step's rows
    out = cache.attend(q, lens, layer=l)             # causal attention over them and all before
    cache.fork([0], [1])                             # sequence 1 goes on from sequence 0's pages
    cache.trim(lens)                                 # pages behind these lengths become free

A cache of dtype=torch.float8_e4m3fn holds 8 bits a value, with a power of two for every 16 positions of a layer and KV
head; rows, q and out are then float32 or bfloat16, whichever a call brings.  Under a window a row reads the last
positions and a few first ones only, and the pages between can be given up:

    out = cache.attend(q, lens, layer=l, window=4096, sinks=4)
    cache.slide(lens, window=4096, sinks=4)          # pages that no later row reads become free

Sequences are rows of the table; lens, first, last, keep, row_off are int32 tensors on the cache's
device (their values are not read here: the calls do not wait for the GPU).  Every call runs on the
current stream of that device.
"""
import ctypes
import math
import warnings

import torch
from torch.autograd import forward_ad

from . import binding as B

DTYPES = {torch.float32: 0, torch.bfloat16: 1}
HELD8, SCALES = torch.float8_e4m3fn, torch.float8_e8m0fnu
BLOCK = 16  # positions that share a power of two
MOST_POSITIONS = 1 << 30
# the current stream of a device, as HIP's handle (torch's own shortcut to it where there is one: a
# microsecond less per call)
_stream_of = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)
_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _need(ok, msg):
    if not ok:
        raise B.Sd2Error(msg)


def _tangent(t):
    """Whether t carries a forward-mode tangent (outside a dual level, which is quick to see, none does)."""
    return getattr(forward_ad, "_current_level", 0) >= 0 and forward_ad.unpack_dual(t).tangent is not None


class PagedCache:
    """k and v: contiguous [n_pages][n_layers][n_kv_heads][page_size][head_dim], float32, bfloat16 or float8_e4m3fn;
    table: contiguous int32 [max_seqs][max_pages], -1 where there is no page; refs: int32 [n_pages],
    the table entries that name each page; scales (float8_e4m3fn only): contiguous float8_e8m0fnu
    [n_pages][n_layers][n_kv_heads][page_size / 16][2], the powers of two of k and of v.  The cache works on these
    tensors and keeps them."""

    def __init__(self, k, v, table, refs, scales=None):
        _need(k.is_cuda and k.dim() == 5 and (k.dtype in DTYPES or k.dtype == HELD8), "k: a float32, bfloat16 or "
              "float8_e4m3fn GPU tensor [n_pages][n_layers][n_kv_heads][page_size][head_dim]")
        _need(v.shape == k.shape and v.dtype == k.dtype and v.device == k.device, "v has to be like k")
        _need(k.is_contiguous() and v.is_contiguous(), "k and v have to be contiguous")
        _need(not any(t.requires_grad or _tangent(t) for t in (k, v)), "k and v: no gradients here (detach them)")
        self._int32(table, 2, "table", k.device)
        self._int32(refs, 1, "refs", k.device)
        n_pages, n_layers, n_kv, page, hd = k.shape
        _need(refs.numel() == n_pages, "refs: one for every page")
        self.held8 = k.dtype == HELD8
        if self.held8:
            _need(isinstance(scales, torch.Tensor) and scales.dtype == SCALES and scales.device == k.device and
                  page % BLOCK == 0 and scales.shape == (n_pages, n_layers, n_kv, page // BLOCK, 2) and scales.is_contiguous(),
                  "scales: a contiguous float8_e8m0fnu tensor [n_pages][n_layers][n_kv_heads][page_size / 16][2] on k's device")
        else:
            _need(scales is None, "scales: only float8_e4m3fn caches have them")
        self.k, self.v, self.table, self.refs, self.scales = k, v, table, refs, scales
        self.device, self.dtype = k.device, k.dtype
        self._index, self._sizes = k.device.index, {}
        self._unused = torch.empty(256, dtype=torch.uint8, device=k.device)  # workspace of calls that need none
        self.n_pages, self.n_layers, self.n_kv_heads, self.page_size, self.head_dim = n_pages, n_layers, n_kv, page, hd
        self.max_seqs, self.max_pages = table.shape
        self.lib = B.load()
        size = k.element_size()
        pages = B.Pages(page, n_pages, self.max_seqs, self.max_pages, table.data_ptr(), refs.data_ptr(), 3 if self.held8 else 2)
        for i, pool in enumerate((k, v)):
            pages.arrays[i] = B.PageArray(pool.data_ptr(), n_layers * n_kv, hd * size)
        record = n_kv * (page // BLOCK) * 2  # bytes of the scales of a page and layer
        if self.held8:
            pages.arrays[2] = B.PageArray(scales.data_ptr(), n_layers, -record)
        self._pages = pages
        self._pages_ws = self.lib.sd2_pages_workspace_bytes(ctypes.byref(pages))
        _need(self._pages_ws > 0, "the cache's sizes are outside what sd2_pages takes")
        self._scale = 1.0 / math.sqrt(hd)
        layer = n_kv * page * hd
        # for a dtype of a call's rows: a layer's view of the cache
        self._kv = {t: [B.PagedKv(k.data_ptr() + l * layer * size, v.data_ptr() + l * layer * size, n_layers * layer,
                                  DTYPES[t], page, n_pages, n_kv, hd, self.max_pages, table.data_ptr())
                        for l in range(n_layers)] for t in (DTYPES if self.held8 else (k.dtype,))}
        if self.held8:
            self._kv = {t: [B.PagedScaled(kv, scales.data_ptr() + l * record, n_layers * record) for l, kv in enumerate(kvs)]
                        for t, kvs in self._kv.items()}
        try:
            self._quick = B.load_torch_paged()
        except (RuntimeError, ImportError) as e:  # (libsd2.so is there: the same calls, in more steps)
            warnings.warn(f"{e}; until then each call takes 5 to 9 us more of the host", RuntimeWarning, stacklevel=2)
            self._quick = None
            return
        views = [(type(self._kv[t][0]) * n_layers)(*self._kv[t]) if t in self._kv else None for t in (torch.float32, torch.bfloat16)]
        self._cache = self._quick.cache(
            self._index, n_layers, hd, n_kv, self.max_seqs, self.max_pages, page, int(self.held8),
            *(0 if v is None else ctypes.addressof(v) for v in views), ctypes.addressof(pages), self._unused.data_ptr(),
            self._pages_ws, self._scale)

    @classmethod
    def empty(cls, n_pages, page_size, n_layers, n_kv_heads, head_dim, max_seqs, max_pages, dtype=torch.bfloat16,
              device="cuda"):
        """A cache of free pages and no sequences."""
        shape = (n_pages, n_layers, n_kv_heads, page_size, head_dim)
        scales = None
        if dtype == HELD8:
            scales = torch.empty((n_pages, n_layers, n_kv_heads, page_size // BLOCK, 2), dtype=SCALES, device=device)
        return cls(torch.empty(shape, dtype=dtype, device=device), torch.empty(shape, dtype=dtype, device=device),
                   torch.full((max_seqs, max_pages), -1, dtype=torch.int32, device=device),
                   torch.zeros(n_pages, dtype=torch.int32, device=device), scales)

    # ---- checks ------------------------------------------------------------------------------------
    @staticmethod
    def _int32(t, dim, what, device):
        _need(isinstance(t, torch.Tensor) and t.dtype == torch.int32 and t.dim() == dim and t.device == device and
              t.is_contiguous(), f"{what}: a contiguous int32 tensor of {dim} dimension(s) on the cache's device")

    def _layer(self, layer, like):
        _need(isinstance(layer, int) and 0 <= layer < self.n_layers, f"layer {layer} of {self.n_layers}")
        return ctypes.byref(self._kv[like.dtype][layer])

    def _packed(self, t, what):
        """A tensor [rows][heads][head_dim] whose rows may be apart: its row stride."""
        _need(isinstance(t, torch.Tensor) and t.device == self.device and t.dtype in self._kv and t.dim() == 3 and
              t.shape[2] == self.head_dim, f"{what}: [rows][heads][head_dim] of the cache's type (float32 or bfloat16 for 8 bits), on its device")
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

    @staticmethod
    def _window(window, sinks):
        _need(isinstance(window, int) and 1 <= window <= MOST_POSITIONS, f"window {window}: 1 to 2^30 positions")
        _need(isinstance(sinks, int) and 0 <= sinks <= MOST_POSITIONS, f"sinks {sinks}: 0 to 2^30 positions")

    def _workspace(self, nbytes):
        return torch.empty(nbytes, dtype=torch.uint8, device=self.device)

    def _plain(self):
        """Whether a call may go the short way: if there is one, on the current device, and where no tensor carries a tangent."""
        return self._quick is not None and _device() == self._index and getattr(forward_ad, "_current_level", 0) < 0

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
        if self._plain() and self._quick.append(self._cache, _stream_of(self._index), k, v, lens, layer, row_off, max_rows):
            return
        ks, vs = self._packed(k, "k"), self._packed(v, "v")
        kv = self._layer(layer, k)
        _need(k.dtype == v.dtype, "k and v: one type")
        _need(k.shape == v.shape and k.shape[1] == self.n_kv_heads, "k and v: [rows][n_kv_heads][head_dim]")
        rows = self._rows(k.shape[0], lens, row_off, max_rows)
        self._call(self.lib.sd2_paged_append_scaled if self.held8 else self.lib.sd2_paged_append, kv, ctypes.byref(rows), k.data_ptr(),
                   ks, v.data_ptr(), vs)

    def attend(self, q, lens, layer=0, row_off=None, max_rows=None, max_len=None, scale=None, out=None, window=None, sinks=0):
        """Causal attention of rows q [rows][heads][head_dim] over their sequences' pages
        (sd2_paged_attn), rows and positions as in append; returns out, like q.  scale: 1 / sqrt(head_dim)
        unless given; max_rows, max_len: the most rows and the largest length, where they are known (they
        decide how the work is split, and max_rows how bf16 rows' weights are rounded; with row_off it is all rows
        unless given).  With a window a row reads the last `window` positions up to its own and the
        first `sinks` ones (sd2_paged_attn_window); caches of 8 bits: sd2_paged_attn_scaled."""
        if self._plain():
            res = self._quick.attend(self._cache, _stream_of(self._index), q, lens, layer, row_off, max_rows, max_len, scale, out,
                                     window, sinks)
            if res is not None:
                return res
        qs = self._packed(q, "q")
        kv = self._layer(layer, q)
        heads = q.shape[1]
        _need(heads > 0 and heads % self.n_kv_heads == 0, f"{heads} heads on {self.n_kv_heads} KV heads")
        if out is None:
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
            os = heads * self.head_dim
        else:
            _need(isinstance(out, torch.Tensor) and out.shape == q.shape, "out has to be like q")
            _need(not q.numel() or out.data_ptr() != q.data_ptr(), "out must not be q")
            os = self._packed(out, "out")
            _need(out.dtype == q.dtype, "out has to be like q")
        if window is None:
            _need(sinks == 0, "sinks: only with a window")
            window = 0
        else:
            self._window(window, sinks)
        rows = self._rows(q.shape[0], lens, row_off, max_rows)
        if max_len is None:
            max_len = self.max_pages * self.page_size
        size, call, more = self.lib.sd2_paged_attn_workspace_bytes, self.lib.sd2_paged_attn, ()
        if self.held8:
            size, call, more = self.lib.sd2_paged_attn_scaled_workspace_bytes, self.lib.sd2_paged_attn_scaled, (window, sinks)
        elif window:
            size, call, more = self.lib.sd2_paged_attn_window_workspace_bytes, self.lib.sd2_paged_attn_window, (window, sinks)
        key = (heads, rows.nseq, rows.max_rows, rows.total_rows, row_off is None, max_len, q.dtype, *more)
        nbytes = self._sizes.get(key)
        if nbytes is None:
            _need(1 <= max_len <= self.max_pages * self.page_size, f"max_len {max_len} of {self.max_pages} pages")
            nbytes = size(kv, ctypes.byref(rows), heads, max_len, *more)
            _need(nbytes > 0, "attend: sizes outside what sd2_paged_attn takes")
            if len(self._sizes) > 1000:
                self._sizes.clear()
            self._sizes[key] = nbytes
        # (the smallest size is that of calls without partial sums)
        ws = self._unused if nbytes == 256 else self._workspace(nbytes)
        self._call(call, kv, ctypes.byref(rows), q.data_ptr(), qs, out.data_ptr(), os, heads,
                   self._scale if scale is None else scale, max_len, *more, ws.data_ptr(), nbytes)
        return out

    # ---- pages -------------------------------------------------------------------------------------
    def reserve(self, first, last, keep=None):
        """Make positions first[b] .. last[b] - 1 writable (sd2_pages_reserve); returns granted, int32
        per sequence: last[b], or where the first page begins that could not be had."""
        if self._plain():
            granted = self._quick.reserve(self._cache, _stream_of(self._index), first, last, keep)
            if granted is not None:
                return granted
        n = self._seqs("first, last, keep", first, last, *(() if keep is None else (keep,)))
        granted = torch.empty_like(last)
        ws = self._workspace(self._pages_ws)
        self._call(self.lib.sd2_pages_reserve, ctypes.byref(self._pages), n, first.data_ptr(), last.data_ptr(),
                   None if keep is None else keep.data_ptr(), granted.data_ptr(), ws.data_ptr(), self._pages_ws)
        return granted

    def fork(self, src, dst):
        """Sequence dst[i] gives up its pages and takes those of src[i], shared (sd2_pages_fork; lists of
        ints)."""
        if self._plain() and self._quick.fork(self._cache, _stream_of(self._index), src, dst):
            return
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

    def slide(self, lens, window, sinks=0):
        """Sequences 0 .. len(lens) - 1 give up the pages that, under this window, no row from position lens[b] on
        reads (sd2_pages_slide; a negative length: none)."""
        if self._plain() and self._quick.slide(self._cache, _stream_of(self._index), lens, window, sinks):
            return
        self._window(window, sinks)
        n = self._seqs("lens", lens)
        self._call(self.lib.sd2_pages_slide, ctypes.byref(self._pages), n, lens.data_ptr(), window, sinks)

    def compact(self):
        """Move the pages in use to the front (sd2_pages_compact); returns their number, int32 [1]."""
        live = torch.empty(1, dtype=torch.int32, device=self.device)
        ws = self._workspace(self._pages_ws)
        self._call(self.lib.sd2_pages_compact, ctypes.byref(self._pages), live.data_ptr(), ws.data_ptr(), self._pages_ws)
        return live

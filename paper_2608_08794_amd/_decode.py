"""ctypes binding of the rotary, paged-cache and decode calls of include/apack.h
(argument marshalling only)."""

import array
import ctypes

from . import _lib
from ._lib import ApackError, _alloc_on, _check, _torch, library

ROPE_LAYOUTS = {"half": 0, "interleaved": 1}
ROPE_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "by_parts": 3}

# Address of a table without entries, which torch gives none: never read, and not NULL, which stands for planes.
_NO_ENTRIES = 256

_P = ctypes.c_void_p
_I32, _I64, _SZ, _F64 = ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_double


class Rope(ctypes.Structure):
    _fields_ = [("rot_dim", _I32), ("layout", _I32), ("pos_rows", _I32), ("transpose", _I32),
                ("sections", _I32 * 4), ("factor", _F64), ("freq", _F64 * 128)]


class Heads(ctypes.Structure):
    _fields_ = [("data", _P), ("heads", _I32), ("reserved", _I32), ("head_stride", _I64), ("row_stride", _I64)]


class Pages(ctypes.Structure):
    _fields_ = [("n_layers", _I32), ("n_pages", _I32), ("page_rows", _I32), ("hkv", _I32), ("d", _I32),
                ("table_width", _I32), ("dtype", ctypes.c_int), ("reserved", _I32), ("page_stride", _I64),
                ("head_stride", _I64), ("row_stride", _I64), ("k", _P), ("v", _P), ("table", _P),
                ("table_stride", _I64)]


class Move(ctypes.Structure):
    _fields_ = [("src_off", _I64), ("n_in", _I64), ("dst_off", _I64), ("n_out", _I64)]


_R, _H, _PG, _I32P = (ctypes.POINTER(x) for x in (Rope, Heads, Pages, _I32))
_lib._SIGS.update({
    "apack_rope_init": (ctypes.c_int, [_R, _I32, _I32, _F64, _I32, _F64, _I64]),
    "apack_rotary": (ctypes.c_int, [_R, _I64, _P, _I64, ctypes.c_int, _I32, _H, _H, _H, _H, _P]),
    "apack_pages_alloc": (ctypes.c_int, [_I32, _P, _I64, _P]),
    "apack_pages_free": (ctypes.c_int, [_I32, _P, _I64, _P]),
    "apack_pages_fork": (ctypes.c_int, [_I32, _P, _I32, _I64, _P, _I32, _P, _P, ctypes.POINTER(_I64)]),
    "apack_pages_copy": (ctypes.c_int, [_PG, _I64, _P, _P]),
    "apack_compact_kv_pages": (ctypes.c_int, [_I32, ctypes.POINTER(Move), _P, _PG, _PG, _P]),
    "apack_rotary_append": (ctypes.c_int, [_R, _I64, _P, _I64, _P, _H, _H, _H, _H, _PG, _P]),
    "apack_paged_attention_workspace": (_SZ, [_I64, _I32, _I32, _I32, _I64]),
    "apack_paged_attention": (ctypes.c_int, [_I64, _I32, _H, _H, _P, _PG, _P, _I64, _P, _I64, _I64, _F64, _P, _SZ,
                                             _P]),
})


# ---------------------------------------------------------------------------
# Tensors as the C structures
# ---------------------------------------------------------------------------

def _fail(status, message):
    raise ApackError(status, message)


def _on_device(tensors, names):
    """The device that every tensor lies on; it must be the current one.  names: theirs, in one text."""
    index = tensors[0].get_device()
    for i, t in enumerate(tensors):
        if t.get_device() != index or index < 0:
            _fail(1, f"{names.split()[i]} must be a CUDA tensor on the call's device")
    if index != _torch().cuda.current_device():
        _fail(1, f"the tensors lie on device {index}, which is not the current one")
    return index


def _stream_on(stream, index):
    """The stream's handle: the given one, or the device's current one."""
    if stream is None:
        return _torch()._C._cuda_getCurrentRawStream(index)
    return stream if isinstance(stream, int) else stream.cuda_stream


def _heads(t, name, dtype):
    """[heads, rows, d] with contiguous elements and any order of heads and rows."""
    if t.dtype is not dtype:
        _fail(3, f"{name} must be {dtype}, not {t.dtype}")
    if t.dim() != 3:
        _fail(2, f"{name} must be [heads, rows, d]")
    sh, sr, se = t.stride()
    heads, _, d = t.shape
    if se != 1 and d > 1:
        _fail(2, f"{name} must have contiguous elements")
    return Heads(t.data_ptr(), heads, 0, sh, sr)


def _int32(t, name, dims):
    """A contiguous int32 tensor."""
    if t.dtype is not _torch().int32:
        _fail(3, f"{name} must be int32, not {t.dtype}")
    if t.dim() != dims or not t.is_contiguous():
        _fail(2, f"{name} must be contiguous, of {dims} dimension{'s' if dims > 1 else ''}")
    return t.data_ptr()


def _first(x, name):
    """One of the tensors of a list of layers, or of one tensor of them all."""
    if isinstance(x, (list, tuple)):
        if not x:
            _fail(1, f"{name} needs one tensor per layer")
        return x[0]
    return x


def _pointers(x, dims, name):
    """(pointers, shape, strides, dtype) of a tensor per layer: a list of them, or one tensor whose first dimension is
    the layer."""
    if isinstance(x, (list, tuple)):
        first = _first(x, name)
        shape, stride, dtype, index = first.shape, first.stride(), first.dtype, first.get_device()
        ptrs = []
        for t in x:
            if t.shape != shape or t.stride() != stride:
                _fail(2, f"the layers of {name} differ in shape or strides")
            if t.dtype is not dtype or t.get_device() != index:
                _fail(3, f"the layers of {name} differ in dtype or device")
            ptrs.append(t.data_ptr())
    else:
        if x.dim() != dims + 1:
            _fail(2, f"{name} must be a list of layers or one tensor [layers, ...] of {dims + 1} dimensions")
        n, stride, dtype = x.shape[0], x.stride(), x.dtype
        shape, step, stride = x.shape[1:], stride[0], stride[1:]
        base, step = x.data_ptr(), step * x.element_size()
        ptrs = range(base, base + n * step, step) if step > 0 else [base] * n
    if len(shape) != dims:
        _fail(2, f"the layers of {name} must have {dims} dimensions")
    if stride[-1] != 1 and shape[-1] > 1:
        _fail(2, f"{name} must have contiguous elements")
    return array.array("Q", ptrs), shape, stride, dtype


def _given(v):
    """Whether there is a V beside the K: a tensor, or a list that is not empty."""
    return v is not None and (not isinstance(v, (list, tuple)) or len(v) > 0)


def _pages(k, v, table=None, n_seq=0, name="pages", planes=False):
    """An apack_pages of [pages, heads, rows, d] tensors, or of planes [heads, rows, d]."""
    dims = 3 if planes else 4
    kp, shape, stride, dtype = _pointers(k, dims, f"k_{name}")
    vp = None
    if _given(v):
        vp, vshape, vstride, vdtype = _pointers(v, dims, f"v_{name}")
        if len(vp) != len(kp) or vshape != shape or vstride != stride:
            _fail(2, f"v_{name} must match k_{name} in layers, shape and strides")
        if vdtype is not dtype:
            _fail(3, f"v_{name} must match k_{name} in dtype")
    if planes:
        pages, (hkv, rows, d), (sh, sr, _), sp = 1, shape, stride, 0
    else:
        (pages, hkv, rows, d), (sp, sh, sr, _) = shape, stride
    tp, width, ts = (None, 0, 0) if table is None else _table(table, n_seq)
    p = Pages(len(kp), pages, rows, hkv, d, width, _code(dtype), 0, sp, sh, sr, kp.buffer_info()[0],
              None if vp is None else vp.buffer_info()[0], tp, ts)
    p.pointers = kp, vp   # kept while p is
    return p


def _table(table, n_seq):
    """(pointer, width, row stride) of a page table."""
    if table.dtype is not _torch().int32:
        _fail(3, f"the table must be int32, not {table.dtype}")
    if table.dim() != 2 or table.shape[0] != n_seq:
        _fail(2, f"the table must be [{n_seq}, pages]")
    width = table.shape[1]
    ts, se = table.stride()
    if se != 1 and width > 1:
        _fail(2, "the table must have contiguous rows")
    return table.data_ptr() or _NO_ENTRIES, width, ts if n_seq > 1 else width


def _one_layer(k, v, dtype, table, n_seq, d):
    """An apack_pages of one layer's [pages, heads, rows, d] K and V, as a decode step uses them."""
    if k.dim() != 4:
        _fail(2, "k_pages must be [pages, heads, rows, d]")
    shape, stride = k.shape, k.stride()
    if v.shape != shape or v.stride() != stride:
        _fail(2, "v_pages must match k_pages in shape and strides")
    if k.dtype is not dtype or v.dtype is not dtype:
        _fail(3, "q and the pages must share a dtype")
    pages, hkv, rows, width = shape
    sp, sh, sr, se = stride
    if width != d:
        _fail(2, "q and the pages differ in d")
    if se != 1 and d > 1:
        _fail(2, "the pages must have contiguous elements")
    tp, width, ts = _table(table, n_seq)
    kv = array.array("Q", (k.data_ptr(), v.data_ptr()))
    at = kv.buffer_info()[0]
    p = Pages(1, pages, rows, hkv, d, width, _code(dtype), 0, sp, sh, sr, at, at + 8, tp, ts)
    p.pointers = kv   # kept while p is
    return p


def _code(dtype):
    torch = _torch()
    if dtype is torch.bfloat16:
        return _lib.APACK_BF16
    if dtype is torch.float32:
        return _lib.APACK_F32
    _fail(3, f"unsupported dtype {dtype}")


def _like(stream, x):
    """A contiguous output of x's shape, allocated on the stream that the call runs on."""
    torch = _torch()
    if stream is None:
        return torch.empty_like(x, memory_format=torch.contiguous_format)
    with _alloc_on(stream):
        return torch.empty_like(x, memory_format=torch.contiguous_format)


def _new(stream, shape, dtype, device):
    torch = _torch()
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with _alloc_on(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _positions(pos, rope, rows):
    """(pointer, row stride) of position ids [rows] or [pos_rows, rows]."""
    if pos.dtype is not _torch().int32:
        _fail(3, f"pos must be int32, not {pos.dtype}")
    n, shape = rope.pos_rows, pos.shape
    if shape != (n, rows) and not (n == 1 and shape == (rows,)):
        _fail(2, f"pos must be [{n}, {rows}]")
    stride = pos.stride()
    if rows > 1 and stride[-1] != 1:
        _fail(2, "pos must have contiguous rows")
    return pos.data_ptr(), stride[0] if n > 1 else rows


def _int32_cpu(t, name):
    """A contiguous int32 tensor in host memory (bookkeeping)."""
    torch = _torch()
    if not isinstance(t, torch.Tensor) or t.is_cuda or t.dtype != torch.int32 or not t.is_contiguous():
        _fail(1, f"{name} must be a contiguous int32 CPU tensor")
    return t.data_ptr()


# ---------------------------------------------------------------------------
# Entry points
# ---------------------------------------------------------------------------

def apack_rope(rot_dim, base=10000.0, layout="half", scaling="none", factor=1.0, trained_len=1, sections=None,
               transpose=False):
    """How positions turn queries and keys: the first rot_dim elements of a
    head, in pairs of the given layout ("half" or "interleaved"), at
    frequencies base^(-2i/rot_dim), scaled for long contexts by `scaling`
    ("linear", "ntk" or "by_parts", by `factor`, from trained_len rows).
    sections: the pairs that each row of position ids turns, for more than one
    row.  The result's freq and factor may be overwritten."""
    r = Rope()
    if layout not in ROPE_LAYOUTS or scaling not in ROPE_SCALINGS:
        _fail(1, f"layout must be one of {list(ROPE_LAYOUTS)}, scaling one of {list(ROPE_SCALINGS)}")
    _check(library().apack_rope_init(ctypes.byref(r), int(rot_dim), ROPE_LAYOUTS[layout], float(base),
                                     ROPE_SCALINGS[scaling], float(factor), int(trained_len)))
    if sections is not None:
        if not 1 <= len(sections) <= 4:
            _fail(1, "sections must name 1 to 4 rows of position ids")
        r.pos_rows = len(sections)
        r.sections = (_I32 * 4)(*[int(x) for x in sections])
    r.transpose = 1 if transpose else 0
    return r


def apack_rotary(pos, rope, q=None, k=None, q_out=None, k_out=None, transpose=None, stream=None):
    """Turns q and k [heads, rows, d] (any order of heads and rows, so a
    transposed [rows, heads, d] projection too) by their position ids pos
    [pos_rows, rows] int32 (which may be one row, expanded).  q_out and k_out may be q and k; without them, new
    [heads, rows, d] tensors.  transpose (rope's by default) turns the other
    way: the gradient of the call, and with factor 1 its inverse.  Returns
    (q_out, k_out)."""
    some = q if q is not None else k
    if some is None:
        _fail(1, "neither q nor k")
    if (q is None and q_out is not None) or (k is None and k_out is not None):
        _fail(1, "an output without its input")
    if some.dim() != 3:
        _fail(2, "q and k must be [heads, rows, d]")
    used = [(t, n) for t, n in ((pos, "pos"), (q, "q"), (k, "k"), (q_out, "q_out"), (k_out, "k_out")) if t is not None]
    index = _on_device([t for t, _ in used], " ".join([n for _, n in used]))
    if transpose is not None and bool(transpose) != bool(rope.transpose):
        rope = Rope.from_buffer_copy(rope)
        rope.transpose = 1 if transpose else 0
    _, rows, d = some.shape
    dtype = some.dtype
    code = _code(dtype)
    p, ps = _positions(pos, rope, rows)
    hq = hk = hqo = hko = None
    if q is not None:
        hq = _heads(q, "q", dtype)
        if q_out is None:
            q_out = _like(stream, q)
        elif q_out.shape != q.shape:
            _fail(2, "q_out must have q's shape")
        hqo = _heads(q_out, "q_out", dtype)
    if k is not None:
        hk = _heads(k, "k", dtype)
        if k.shape[1:] != some.shape[1:]:
            _fail(2, "q and k must agree in rows and d")
        if k_out is None:
            k_out = _like(stream, k)
        elif k_out.shape != k.shape:
            _fail(2, "k_out must have k's shape")
        hko = _heads(k_out, "k_out", dtype)
    _check(library().apack_rotary(rope, rows, p, ps, code, d, hq, hqo, hk, hko, _stream_on(stream, index)))
    return q_out, k_out


def apack_pages_alloc(refs, n):
    """The n lowest free pages of a pool, ascending, as an int32 CPU tensor;
    refs (int32 CPU tensor, a count per page, 0 for a free one) counts them."""
    pages = _torch().empty(max(int(n), 0), dtype=_torch().int32)
    _check(library().apack_pages_alloc(refs.numel(), _int32_cpu(refs, "refs"), int(n), pages.data_ptr()))
    return pages


def apack_pages_free(refs, pages):
    """Gives up one reference to each page."""
    _check(library().apack_pages_free(refs.numel(), _int32_cpu(refs, "refs"), pages.numel(),
                                      _int32_cpu(pages, "pages")))


def apack_pages_fork(refs, page_rows, n_rows, parent, n_children):
    """Forks a sequence of n_rows rows in pages `parent` (int32 CPU tensor):
    (children [n_children, pages] int32, copies [n, 2] int32), CPU tensors.
    Full pages are shared; copies are the pairs that apack_pages_copy then
    copies (on the device) before anything is appended."""
    torch = _torch()
    page_rows, n_rows, n_children = int(page_rows), int(n_rows), int(n_children)
    n = -(-max(n_rows, 0) // page_rows) if page_rows > 0 else 0
    if parent.numel() < n:
        _fail(2, f"{n_rows} rows lie in {n} pages: parent has {parent.numel()}")
    children = torch.empty((max(n_children, 0), n), dtype=torch.int32)
    copies = torch.empty((max(n_children, 0), 2), dtype=torch.int32)
    got = _I64(0)
    _check(library().apack_pages_fork(refs.numel(), _int32_cpu(refs, "refs"), page_rows, n_rows,
                                      _int32_cpu(parent, "parent"), n_children, children.data_ptr(), copies.data_ptr(),
                                      ctypes.byref(got)))
    return children, copies[:got.value]


def apack_pages_copy(pairs, k_pages, v_pages=(), stream=None):
    """Copies page pairs[i, 0] to page pairs[i, 1] in every layer's K and V.
    pairs: int32 CUDA tensor [n, 2]; k_pages, v_pages: per layer [pages, heads,
    rows, d], or one tensor [layers, pages, heads, rows, d]."""
    first = _first(k_pages, "k_pages")
    index = _on_device((pairs, first, _first(v_pages, "v_pages") if _given(v_pages) else first), "pairs k_pages v_pages")
    p = _int32(pairs, "pairs", 2)
    if pairs.shape[1] != 2:
        _fail(2, "pairs must be [n, 2]")
    _check(library().apack_pages_copy(_pages(k_pages, v_pages), pairs.shape[0], p, _stream_on(stream, index)))


def apack_compact_kv_pages(src_rows, seqs, k_in, v_in, k_out, v_out, table_in=None, table_out=None, stream=None):
    """Gathers the kept rows of every sequence from pages or planes into pages
    or planes, in every layer.

    src_rows: int32 CUDA tensor of packed rows, sequence after sequence (a
    prune's kept_rows), or None to move each sequence's first rows; seqs: a
    (src_off, n_in, dst_off, n_out) per sequence.  With a table [n_seq, pages]
    a side's tensors are [pages, heads, rows, d] per layer, without one [heads,
    rows, d]; a list of layers or one tensor with layers first."""
    n = len(seqs)
    first = _first(k_in, "k_in")
    index = _on_device((first, _first(k_out, "k_out"), _first(v_in, "v_in") if _given(v_in) else first,
                        _first(v_out, "v_out") if _given(v_out) else first, first if src_rows is None else src_rows,
                        first if table_in is None else table_in, first if table_out is None else table_out),
                       "k_in k_out v_in v_out src_rows table_in table_out")
    moves = (Move * max(1, n))(*seqs)
    src = None
    if src_rows is not None:
        src = _int32(src_rows, "src_rows", 1)
        if src_rows.shape[0] != sum([m[3] for m in seqs]):
            _fail(2, "src_rows must hold sum n_out rows")
    pin = _pages(k_in, v_in, table_in, n, "in", planes=table_in is None)
    pout = _pages(k_out, v_out, table_out, n, "out", planes=table_out is None)
    _check(library().apack_compact_kv_pages(n, moves, src, pin, pout, _stream_on(stream, index)))


def apack_rotary_append(pos, rope, q, k, v, k_pages, v_pages, table, lens, q_out=None, stream=None):
    """One decode step's new token of each sequence: turns q [hq, n_seq, d] and
    k [hkv, n_seq, d] and writes k and v [hkv, n_seq, d] as row lens[s] - 1 of
    sequence s into one layer's pages [pages, hkv, rows, d].  Returns q_out (new
    if not given; it may be q)."""
    if q.dim() != 3:
        _fail(2, "q must be [hq, n_seq, d]")
    index = _on_device((q, pos, k, v, k_pages, v_pages, table, lens, q if q_out is None else q_out),
                       "q pos k v k_pages v_pages table lens q_out")
    _, n, d = q.shape
    dtype = q.dtype
    p, ps = _positions(pos, rope, n)
    pages = _one_layer(k_pages, v_pages, dtype, table, n, d)
    hq, hk, hv = _heads(q, "q", dtype), _heads(k, "k", dtype), _heads(v, "v", dtype)
    shape = (pages.hkv, n, d)
    if k.shape != shape or v.shape != shape:
        _fail(2, f"k and v must be [{pages.hkv}, {n}, {d}]")
    lp = _int32(lens, "lens", 1)
    if lens.shape[0] != n:
        _fail(2, f"lens must be [{n}]")
    if q_out is None:
        q_out = _like(stream, q)
    elif q_out.shape != q.shape:
        _fail(2, "q_out must have q's shape")
    _check(library().apack_rotary_append(rope, n, p, ps, lp, hq, _heads(q_out, "q_out", dtype), hk, hv, pages,
                                         _stream_on(stream, index)))
    return q_out


def apack_paged_attention_workspace(n_seq, hq, hkv, d, max_len):
    return int(library().apack_paged_attention_workspace(int(n_seq), int(hq), int(hkv), int(d), int(max_len)))


def apack_paged_attention(q, k_pages, v_pages, table, lens, max_len, mask=None, window=0, scale=None, out=None,
                          return_lse=False, lse=None, workspace=None, stream=None):
    """Attention of one query row per sequence, q [hq, n_seq, d], over its rows
    of one layer's paged cache ([pages, hkv, rows, d] tensors, table [n_seq,
    pages] int32, lens [n_seq] int32 of at most max_len rows).  mask: bool or
    uint8 [n_seq, max_len] (which may be one row, expanded), rows to attend to;
    window: only the last so many rows (0: all); scale: 1/sqrt(d) by default.
    Returns out [hq, n_seq, d] (new if not given), and with return_lse (out, lse
    [hq, n_seq] fp32)."""
    torch = _torch()
    if q.dim() != 3:
        _fail(2, "q must be [hq, n_seq, d]")
    index = _on_device((q, k_pages, v_pages, table, lens, q if mask is None else mask, q if out is None else out,
                        q if lse is None else lse, q if workspace is None else workspace),
                       "q k_pages v_pages table lens mask out lse workspace")
    hq, n, d = q.shape
    dtype, max_len = q.dtype, int(max_len)
    qh = _heads(q, "q", dtype)
    pages = _one_layer(k_pages, v_pages, dtype, table, n, d)
    lp = _int32(lens, "lens", 1)
    if lens.shape[0] != n:
        _fail(2, f"lens must be [{n}]")
    mp, ms = None, 0
    if mask is not None:
        if mask.dtype not in (torch.bool, torch.uint8):
            _fail(3, "mask must be bool or uint8")
        if mask.shape != (n, max_len) or (max_len > 1 and mask.stride(1) != 1):
            _fail(2, f"mask must be [{n}, {max_len}] with contiguous rows")
        mp, ms = mask.data_ptr(), mask.stride(0) if n > 1 else max_len
    if scale is not None and not scale > 0:
        _fail(1, "scale must be > 0")
    if out is None:
        out = _like(stream, q)
    elif out.shape != q.shape:
        _fail(2, "out must have q's shape")
    if return_lse and lse is None:
        lse = _new(stream, (hq, n), torch.float32, q.device)
    sp = None
    if lse is not None:
        if lse.dtype is not torch.float32:
            _fail(3, "lse must be float32")
        if lse.shape != (hq, n) or not lse.is_contiguous():
            _fail(2, f"lse must be a contiguous [{hq}, {n}] tensor")
        sp = lse.data_ptr()
    lib = library()
    if workspace is None:
        need = lib.apack_paged_attention_workspace(n, hq, pages.hkv, d, max_len)
        workspace = _new(stream, (max(need, 256),), torch.uint8, q.device)
    elif not workspace.is_contiguous():
        _fail(2, "workspace must be contiguous")
    _check(lib.apack_paged_attention(n, hq, qh, _heads(out, "out", dtype), sp, pages, lp, max_len, mp, ms, int(window),
                                     0.0 if scale is None else float(scale), workspace.data_ptr(),
                                     workspace.numel() * workspace.element_size(), _stream_on(stream, index)))
    return (out, lse) if return_lse else out

"""ctypes binding of the rotary, paged-cache and decode calls of include/apack.h
(argument marshalling only)."""

import contextlib
import ctypes

from . import _lib
from ._lib import ApackError, _alloc_on, _check, _stream, _torch, _workspace, library

ROPE_LAYOUTS = {"half": 0, "interleaved": 1}
ROPE_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "by_parts": 3}

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
                ("head_stride", _I64), ("row_stride", _I64), ("k", ctypes.POINTER(_P)), ("v", ctypes.POINTER(_P)),
                ("table", _P), ("table_stride", _I64)]


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


class _Device:
    """The device of a call: every tensor must lie on it, and it must be the current one."""

    def __init__(self):
        self.index = None

    def take(self, t, name, dtype=None):
        if not t.is_cuda:
            _fail(1, f"{name} must be a CUDA tensor")
        i = t.get_device()
        if self.index is None:
            self.index = i
            if i != _torch().cuda.current_device():
                _fail(1, f"{name} lies on device {i}, which is not the current one")
        elif i != self.index:
            _fail(1, f"{name} lies on device {i}, other tensors on {self.index}")
        if dtype is not None and t.dtype != dtype:
            _fail(3, f"{name} must be {dtype}, not {t.dtype}")
        return t.data_ptr()


def _heads(dev, t, name, dtype):
    """[heads, rows, d] with contiguous elements and any order of heads and rows."""
    p = dev.take(t, name, dtype)
    if t.dim() != 3:
        _fail(2, f"{name} must be [heads, rows, d]")
    sh, sr, se = t.stride()
    if se != 1 and t.shape[2] > 1:
        _fail(2, f"{name} must have contiguous elements")
    return Heads(p, t.shape[0], 0, sh, sr)


def _layers(dev, x, dims, name):
    """(pointers, shape, strides, dtype) of a tensor per layer: a list of them, or one tensor whose first dimension is
    the layer."""
    if isinstance(x, (list, tuple)):
        if not x:
            _fail(1, f"{name} needs one tensor per layer")
        first = x[0]
        shape, stride, dtype = first.shape, first.stride(), first.dtype
        ptrs = [dev.take(t, name, dtype) for t in x]
        if any(t.shape != shape or t.stride() != stride for t in x):
            _fail(2, f"the layers of {name} differ in shape or strides")
    else:
        base = dev.take(x, name)
        if x.dim() != dims + 1:
            _fail(2, f"{name} must be a list of layers or one tensor [layers, ...] of {dims + 1} dimensions")
        shape, stride, dtype = x.shape[1:], x.stride()[1:], x.dtype
        step = x.stride(0) * x.element_size()
        ptrs = [base + i * step for i in range(x.shape[0])]
    if len(shape) != dims:
        _fail(2, f"the layers of {name} must have {dims} dimensions")
    if stride[-1] != 1 and shape[-1] > 1:
        _fail(2, f"{name} must have contiguous elements")
    return ptrs, shape, stride, dtype


def _table(dev, t, n_seq):
    p = dev.take(t, "table", _torch().int32)
    if t.dim() != 2 or t.shape[0] != n_seq:
        _fail(2, f"table must be [{n_seq}, pages]")
    if t.stride(1) != 1 and t.shape[1] > 1:
        _fail(2, "table must have contiguous rows")
    return p, t.shape[1], max(t.stride(0), t.shape[1]) if n_seq < 2 else t.stride(0)


def _pages(dev, k, v, table=None, n_seq=0, name="pages", planes=False):
    """An apack_pages of [pages, heads, rows, d] tensors, or of planes [heads, rows, d]."""
    dims = 3 if planes else 4
    ptrs, shape, stride, dtype = _layers(dev, k, dims, f"k_{name}")
    n = len(ptrs)
    p = Pages()
    p.n_layers, p.dtype = n, _code(dtype)
    p.k = (_P * n)(*ptrs)
    if v is not None and len(v):
        vp, vshape, vstride, vdtype = _layers(dev, v, dims, f"v_{name}")
        if len(vp) != n or vshape != shape or vstride != stride:
            _fail(2, f"v_{name} must match k_{name} in layers, shape and strides")
        if vdtype != dtype:
            _fail(3, f"v_{name} must match k_{name} in dtype")
        p.v = (_P * n)(*vp)
    if planes:
        p.n_pages, p.hkv, p.page_rows, p.d = 1, shape[0], shape[1], shape[2]
        p.head_stride, p.row_stride = stride[0], stride[1]
    else:
        p.n_pages, p.hkv, p.page_rows, p.d = shape
        p.page_stride, p.head_stride, p.row_stride = stride[0], stride[1], stride[2]
    if table is not None:
        p.table, p.table_width, p.table_stride = _table(dev, table, n_seq)
    return p


def _code(dtype):
    torch = _torch()
    if dtype == torch.bfloat16:
        return _lib.APACK_BF16
    if dtype == torch.float32:
        return _lib.APACK_F32
    _fail(3, f"unsupported dtype {dtype}")


def _on(stream):
    return contextlib.nullcontext() if stream is None else _alloc_on(stream)


def _positions(dev, pos, rope, rows):
    """(pointer, row stride) of position ids [rows] or [pos_rows, rows]."""
    p = dev.take(pos, "pos", _torch().int32)
    shape = tuple(pos.shape)
    if shape != (rope.pos_rows, rows) and not (rope.pos_rows == 1 and shape == (rows,)):
        _fail(2, f"pos must be [{rope.pos_rows}, {rows}]")
    if rows > 1 and pos.stride(-1) != 1:
        _fail(2, "pos must have contiguous rows")
    return p, pos.stride(0) if rope.pos_rows > 1 else rows


def _int32_cpu(t, name, shape=None):
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
    [pos_rows, rows] int32.  q_out and k_out may be q and k; without them, new
    [heads, rows, d] tensors.  transpose (rope's by default) turns the other
    way: the gradient of the call, and with factor 1 its inverse.  Returns
    (q_out, k_out)."""
    torch = _torch()
    dev = _Device()
    some = q if q is not None else k
    if some is None:
        _fail(1, "neither q nor k")
    if some.dim() != 3:
        _fail(2, "q and k must be [heads, rows, d]")
    if k is not None and (k.dim() != 3 or k.shape[1:] != some.shape[1:]):
        _fail(2, "q and k must agree in rows and d")
    if (q is None and q_out is not None) or (k is None and k_out is not None):
        _fail(1, "an output without its input")
    if transpose is not None and bool(transpose) != bool(rope.transpose):
        rope = Rope.from_buffer_copy(rope)
        rope.transpose = 1 if transpose else 0
    _, rows, d = some.shape
    p, ps = _positions(dev, pos, rope, rows)
    dtype = some.dtype
    code = _code(dtype)
    pairs = []
    outs = []
    for x, y, name in ((q, q_out, "q"), (k, k_out, "k")):
        if x is None:
            pairs += [None, None]
            outs.append(None)
            continue
        hx = _heads(dev, x, name, dtype)
        if y is None:
            with _on(stream):
                y = torch.empty(x.shape, dtype=dtype, device=x.device)
        elif y.shape != x.shape:
            _fail(2, f"{name}_out must have {name}'s shape")
        pairs += [hx, _heads(dev, y, name + "_out", dtype)]
        outs.append(y)
    _check(library().apack_rotary(rope, rows, p, ps, code, d, *pairs, _stream(stream)))
    return outs[0], outs[1]


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
    dev = _Device()
    p = dev.take(pairs, "pairs", _torch().int32)
    if pairs.dim() != 2 or pairs.shape[1] != 2 or not pairs.is_contiguous():
        _fail(2, "pairs must be a contiguous [n, 2] tensor")
    _check(library().apack_pages_copy(_pages(dev, k_pages, v_pages), pairs.shape[0], p, _stream(stream)))


def apack_compact_kv_pages(src_rows, seqs, k_in, v_in, k_out, v_out, table_in=None, table_out=None, stream=None):
    """Gathers the kept rows of every sequence from pages or planes into pages
    or planes, in every layer.

    src_rows: int32 CUDA tensor of packed rows, sequence after sequence (a
    prune's kept_rows), or None to move each sequence's first rows; seqs: a
    (src_off, n_in, dst_off, n_out) per sequence.  With a table [n_seq, pages]
    a side's tensors are [pages, heads, rows, d] per layer, without one [heads,
    rows, d]; a list of layers or one tensor with layers first."""
    torch = _torch()
    dev = _Device()
    n = len(seqs)
    moves = (Move * max(1, n))(*seqs)
    src = None
    if src_rows is not None:
        src = dev.take(src_rows, "src_rows", torch.int32)
        if src_rows.numel() != sum(m[3] for m in seqs) or not src_rows.is_contiguous():
            _fail(2, "src_rows must be contiguous, with sum n_out rows")
    pin = _pages(dev, k_in, v_in, table_in, n, "in", planes=table_in is None)
    pout = _pages(dev, k_out, v_out, table_out, n, "out", planes=table_out is None)
    _check(library().apack_compact_kv_pages(n, moves, src, pin, pout, _stream(stream)))


def apack_rotary_append(pos, rope, q, k, v, k_pages, v_pages, table, lens, q_out=None, stream=None):
    """One decode step's new token of each sequence: turns q [hq, n_seq, d] and
    k [hkv, n_seq, d] and writes k and v [hkv, n_seq, d] as row lens[s] - 1 of
    sequence s into one layer's pages [pages, hkv, rows, d].  Returns q_out (new
    if not given; it may be q)."""
    torch = _torch()
    dev = _Device()
    if q.dim() != 3:
        _fail(2, "q must be [hq, n_seq, d]")
    n, dtype = q.shape[1], q.dtype
    p, ps = _positions(dev, pos, rope, n)
    hq = _heads(dev, q, "q", dtype)
    pages = _pages(dev, [k_pages], [v_pages], table, n)
    if pages.dtype != _code(dtype):
        _fail(3, "q and the pages must share a dtype")
    for x, name in ((k, "k"), (v, "v")):
        if tuple(x.shape) != (pages.hkv, n, pages.d):
            _fail(2, f"{name} must be [{pages.hkv}, {n}, {pages.d}]")
    if q.shape[2] != pages.d:
        _fail(2, "q and the pages differ in d")
    lp = dev.take(lens, "lens", torch.int32)
    if lens.shape != (n,) or not lens.is_contiguous():
        _fail(2, f"lens must be a contiguous [{n}] tensor")
    hk, hv = _heads(dev, k, "k", dtype), _heads(dev, v, "v", dtype)
    if q_out is None:
        with _on(stream):
            q_out = torch.empty(q.shape, dtype=dtype, device=q.device)
    elif q_out.shape != q.shape:
        _fail(2, "q_out must have q's shape")
    _check(library().apack_rotary_append(rope, n, p, ps, lp, hq, _heads(dev, q_out, "q_out", dtype), hk, hv, pages,
                                         _stream(stream)))
    return q_out


def apack_paged_attention_workspace(n_seq, hq, hkv, d, max_len):
    return int(library().apack_paged_attention_workspace(int(n_seq), int(hq), int(hkv), int(d), int(max_len)))


def apack_paged_attention(q, k_pages, v_pages, table, lens, max_len, mask=None, window=0, scale=None, out=None,
                          return_lse=False, lse=None, workspace=None, stream=None):
    """Attention of one query row per sequence, q [hq, n_seq, d], over its rows
    of one layer's paged cache ([pages, hkv, rows, d] tensors, table [n_seq,
    pages] int32, lens [n_seq] int32 of at most max_len rows).  mask: bool or
    uint8 [n_seq, max_len], rows to attend to; window: only the last so many
    rows (0: all); scale: 1/sqrt(d) by default.  Returns out [hq, n_seq, d] (new
    if not given), and with return_lse (out, lse [hq, n_seq] fp32)."""
    torch = _torch()
    dev = _Device()
    if q.dim() != 3:
        _fail(2, "q must be [hq, n_seq, d]")
    hq, n, d = q.shape
    dtype, max_len = q.dtype, int(max_len)
    qh = _heads(dev, q, "q", dtype)
    pages = _pages(dev, [k_pages], [v_pages], table, n)
    if pages.dtype != _code(dtype):
        _fail(3, "q and the pages must share a dtype")
    if d != pages.d:
        _fail(2, "q and the pages differ in d")
    lp = dev.take(lens, "lens", torch.int32)
    if lens.shape != (n,) or not lens.is_contiguous():
        _fail(2, f"lens must be a contiguous [{n}] tensor")
    mp = ms = 0
    if mask is not None:
        mp = dev.take(mask, "mask")
        if mask.dtype not in (torch.bool, torch.uint8):
            _fail(3, "mask must be bool or uint8")
        if tuple(mask.shape) != (n, max_len) or (max_len > 1 and mask.stride(1) != 1):
            _fail(2, f"mask must be [{n}, {max_len}] with contiguous rows")
        ms = mask.stride(0) if n > 1 else max_len
    if scale is not None and not scale > 0:
        _fail(1, "scale must be > 0")
    with _on(stream):
        if out is None:
            out = torch.empty(q.shape, dtype=dtype, device=q.device)
        if return_lse and lse is None:
            lse = torch.empty((hq, n), dtype=torch.float32, device=q.device)
        if workspace is None:
            workspace = _workspace(library().apack_paged_attention_workspace(n, hq, pages.hkv, d, max_len), q.device)
    if out.shape != q.shape:
        _fail(2, "out must have q's shape")
    sp = None
    if lse is not None:
        sp = dev.take(lse, "lse", torch.float32)
        if tuple(lse.shape) != (hq, n) or not lse.is_contiguous():
            _fail(2, f"lse must be a contiguous [{hq}, {n}] tensor")
    wp = dev.take(workspace, "workspace", torch.uint8)
    _check(library().apack_paged_attention(n, hq, qh, _heads(dev, out, "out", dtype), sp, pages, lp, max_len, mp, ms,
                                           int(window), 0.0 if scale is None else float(scale), wp, workspace.numel(),
                                           _stream(stream)))
    return (out, lse) if return_lse else out

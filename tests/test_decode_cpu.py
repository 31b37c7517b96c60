"""Rotary, paged-cache and decode calls on the CPU: pins of their oracle, the
bookkeeping of pages, and refusals (arguments are checked on the host before
anything is enqueued, so fake device addresses force every error path)."""

import ctypes
import math

import numpy as np
import pytest

import paper_2608_08794_amd as A
from oracle import decode as OD
from paper_2608_08794_amd import _decode as D

torch = pytest.importorskip("torch")

FAKE = 1 << 40


# -- the oracle ---------------------------------------------------------------

@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("transpose", [False, True])
def test_oracle_rotary_is_a_complex_product(layout, transpose):
    rng = np.random.default_rng(3)
    x, theta = rng.standard_normal((3, 5, 10)), rng.standard_normal((5, 4)) * 50
    y = OD.rotary(x, theta, layout, 1.5, transpose)
    a, b = (x[..., :4], x[..., 4:8]) if layout == "half" else (x[..., 0:8:2], x[..., 1:8:2])
    z = (a + 1j * b) * 1.5 * np.exp(-1j * theta if transpose else 1j * theta)
    ya, yb = (y[..., :4], y[..., 4:8]) if layout == "half" else (y[..., 0:8:2], y[..., 1:8:2])
    np.testing.assert_allclose(ya, z.real, rtol=0, atol=1e-13)
    np.testing.assert_allclose(yb, z.imag, rtol=0, atol=1e-13)
    np.testing.assert_array_equal(y[..., 8:], x[..., 8:])


def test_oracle_rotary_makes_products_of_differences():
    # <R(p) q, R(r) k> depends on p - r only.
    rng = np.random.default_rng(4)
    q, k = rng.standard_normal((2, 1, 1, 16))
    f, _ = OD.frequencies(16, 100.0)

    def at(x, p):
        return OD.rotary(x, np.array([[p]]) * f)[0, 0]

    assert abs(at(q, 70) @ at(k, 41) - at(q, 1029) @ at(k, 1000)) < 1e-10


def test_oracle_attention_is_torchs():
    rng = np.random.default_rng(5)
    q, k, v = rng.standard_normal((6, 8)), rng.standard_normal((2, 9, 8)), rng.standard_normal((2, 9, 8))
    o, lse, w, _ = OD.attention(q, k, v, 0.3)
    tq, tk, tv = (torch.from_numpy(x) for x in (q, k, v))
    want = torch.nn.functional.scaled_dot_product_attention(tq[None, :, None], tk[None], tv[None], scale=0.3,
                                                            enable_gqa=True)[0, :, 0]
    np.testing.assert_allclose(o, want.numpy(), atol=1e-13)
    x = 0.3 * (tk.repeat_interleave(3, 0) @ tq[..., None])[..., 0]
    np.testing.assert_allclose(lse, torch.logsumexp(x, -1).numpy(), atol=1e-13)
    assert (w >= np.abs(o) - 1e-15).all()
    o, lse, _, _ = OD.attention(q, k[:, :0], v[:, :0], 0.3)
    assert not o.any() and np.isneginf(lse).all()


def test_oracle_rows_seen():
    table = [3, -1, 7, 0]
    assert OD.rows_seen(table, 2, 5, 8, 100) == [(3, 0), (3, 1), (0, 0), (0, 1)]   # -1 and 7 are no pages of 5
    assert OD.rows_seen(table, 2, 8, 9, 100, window=3) == [(0, 0), (0, 1)]         # row 8 is beyond the table
    assert OD.rows_seen(table, 2, 8, 8, 5) == [(3, 0), (3, 1), (7, 0)]
    assert OD.rows_seen(table, 2, 8, 2, 5, mask=[0, 1]) == [(3, 1)]
    assert OD.rows_seen(table, 2, 8, -4, 5) == []


# -- frequencies --------------------------------------------------------------

@pytest.mark.parametrize("scaling", ["none", "linear", "ntk", "by_parts"])
@pytest.mark.parametrize("rot", [4, 36, 128, 256])
def test_rope_frequencies(rot, scaling):
    r = A.apack_rope(rot, base=1e6, scaling=scaling, factor=4.0, trained_len=32768)
    f, factor = OD.frequencies(rot, 1e6, scaling, 4.0, 32768)
    # pow and log are off by a few units in the last place of fp64.
    np.testing.assert_allclose(list(r.freq)[:rot // 2], f, rtol=1e-14)
    assert math.isclose(r.factor, factor, rel_tol=1e-15)
    assert r.pos_rows == 1 and r.sections[0] == rot // 2 and not any(list(r.freq)[rot // 2:])


def test_by_parts_keeps_fast_pairs_and_stretches_slow_ones():
    plain, scaled = A.apack_rope(128, base=1e6), A.apack_rope(128, base=1e6, scaling="by_parts", factor=8.0,
                                                              trained_len=4096)
    assert scaled.freq[0] == plain.freq[0]
    assert math.isclose(scaled.freq[63], plain.freq[63] / 8, rel_tol=1e-15)
    assert math.isclose(scaled.factor, 0.1 * math.log(8) + 1)


@pytest.mark.parametrize("kw", [
    dict(rot_dim=0), dict(rot_dim=7), dict(rot_dim=258), dict(rot_dim=64, base=1.0), dict(rot_dim=64, base=math.nan),
    dict(rot_dim=64, scaling="linear", factor=0.5), dict(rot_dim=64, scaling="by_parts", factor=2.0, trained_len=0),
    dict(rot_dim=2, scaling="ntk", factor=2.0), dict(rot_dim=64, layout="third"), dict(rot_dim=64, scaling="cubic"),
    dict(rot_dim=64, sections=(1, 2, 3, 4, 5)), dict(rot_dim=64, base=1e300, scaling="ntk", factor=1e300),
])
def test_rope_refusals(kw):
    with pytest.raises(A.ApackError):
        A.apack_rope(**kw)


# -- bookkeeping --------------------------------------------------------------

def _refs(*values):
    return torch.tensor(values, dtype=torch.int32)


def test_alloc_takes_the_lowest_free_pages():
    refs = _refs(1, 0, 2, 0, 0)
    assert A.apack_pages_alloc(refs, 2).tolist() == [1, 3]
    assert refs.tolist() == [1, 1, 2, 1, 0]
    with pytest.raises(A.ApackError, match="2 pages asked for, 1 free"):
        A.apack_pages_alloc(refs, 2)
    assert refs.tolist() == [1, 1, 2, 1, 0]
    assert A.apack_pages_alloc(refs, 0).numel() == 0
    with pytest.raises(A.ApackError):
        A.apack_pages_alloc(refs, -1)


def test_free_gives_up_references_or_nothing():
    refs = _refs(1, 2, 0)
    A.apack_pages_free(refs, _refs(1, 0, 1))
    assert refs.tolist() == [0, 0, 0]
    refs = _refs(1, 2, 0)
    for bad in (_refs(0, 0), _refs(1, 2), _refs(1, 3), _refs(0, -1)):
        with pytest.raises(A.ApackError):
            A.apack_pages_free(refs, bad)
        assert refs.tolist() == [1, 2, 0]


@pytest.mark.parametrize("n_rows", [0, 1, 15, 16, 17, 48])
def test_fork_shares_full_pages_and_copies_the_last(n_rows):
    refs = torch.zeros(20, dtype=torch.int32)
    refs[0] = 5
    parent = A.apack_pages_alloc(refs, 4)
    before = refs.clone()
    children, copies = A.apack_pages_fork(refs, 16, n_rows, parent, 3)
    full, n = n_rows // 16, -(-n_rows // 16)
    assert children.shape == (3, n)
    for c in range(3):
        assert children[c, :full].tolist() == parent[:full].tolist()
    assert (refs[parent[:full].long()] == before[parent[:full].long()] + 3).all()
    if n > full:
        assert copies.tolist() == [[int(parent[full]), int(children[c, full])] for c in range(3)]
        assert children[:, full].tolist() == [5, 6, 7] and (refs[5:8] == 1).all()
    else:
        assert copies.numel() == 0 and (refs[5:] == 0).all()
    # Freeing the children leaves the pool as it was.
    A.apack_pages_free(refs, children.flatten())
    assert refs.tolist() == before.tolist()


def test_fork_refusals_change_nothing():
    refs = _refs(1, 1, 0)
    for args in ((16, 20, _refs(0, 1), 2),        # two pages needed, one free
                 (16, 20, _refs(0, 2), 1),        # a page that nobody holds
                 (16, 20, _refs(0, 9), 1), (0, 20, _refs(0, 1), 1), (16, -1, _refs(0, 1), 1),
                 (16, 20, _refs(0, 1), -1), (16, 20, _refs(0), 1)):
        with pytest.raises(A.ApackError):
            A.apack_pages_fork(refs, *args)
        assert refs.tolist() == [1, 1, 0]
    children, copies = A.apack_pages_fork(refs, 16, 20, _refs(0, 1), 0)
    assert children.shape == (0, 2) and not copies.numel() and refs.tolist() == [1, 1, 0]


def test_bookkeeping_takes_host_int32_tensors():
    with pytest.raises(A.ApackError):
        A.apack_pages_alloc(torch.zeros(4, dtype=torch.int64), 1)
    with pytest.raises(A.ApackError):
        A.apack_pages_free(torch.zeros(8, dtype=torch.int32)[::2], _refs(0))


# -- refusals of the device calls ---------------------------------------------

def _pages(n_layers=1, n_pages=4, page_rows=16, hkv=2, d=64, dtype=0, table=FAKE + (9 << 34), width=4, v=True,
           k0=FAKE, v0=FAKE + (1 << 34), **kw):
    p = D.Pages()
    p.n_layers, p.n_pages, p.page_rows, p.hkv, p.d, p.dtype = n_layers, n_pages, page_rows, hkv, d, dtype
    p.row_stride, p.head_stride, p.page_stride = d, page_rows * d, hkv * page_rows * d
    n = max(1, min(n_layers, 100))
    p.pointers = [(ctypes.c_void_p * n)(*[x + (i << 28) for i in range(n)]) for x in (k0, v0)]
    p.k = ctypes.addressof(p.pointers[0])
    if v:
        p.v = ctypes.addressof(p.pointers[1])
    p.table, p.table_width, p.table_stride = table, width, width
    for name, x in kw.items():
        setattr(p, name, x)
    return p


def _heads(data, heads, rows, d, **kw):
    h = D.Heads(data, heads, 0, rows * d, d)
    for name, x in kw.items():
        setattr(h, name, x)
    return h


def _status(name, *args):
    st = getattr(A.library(), name)(*args)
    return st, A.library().apack_last_error().decode()


def _rope(rot=64, **kw):
    r = A.apack_rope(rot)
    for name, x in kw.items():
        setattr(r, name, x)
    return r


def _rotary(rope=None, rows=8, pos=FAKE + (5 << 34), stride=8, dtype=0, d=64, q=None, qo=None, k=None, ko=None):
    q = q or _heads(FAKE, 4, rows, d)
    qo = qo or _heads(FAKE + (1 << 34), 4, rows, d)
    return _status("apack_rotary", rope or _rope(), rows, pos, stride, dtype, d, q, qo, k, ko, None)


NAN_FREQ = (ctypes.c_double * 128)(*([math.nan] * 128))


@pytest.mark.parametrize("status,kw", [
    (3, dict(dtype=2)), (1, dict(pos=None)), (2, dict(rows=-1)), (7, dict(rows=1 << 31)), (7, dict(d=513)),
    (2, dict(d=62)), (1, dict(rope=_rope(layout=2))), (1, dict(rope=_rope(transpose=2))),
    (1, dict(rope=_rope(pos_rows=0))), (1, dict(rope=_rope(pos_rows=5))),
    (2, dict(rope=_rope(sections=(ctypes.c_int32 * 4)(31, 0, 0, 0)))),
    (2, dict(rope=_rope(pos_rows=2, sections=(ctypes.c_int32 * 4)(33, -1, 0, 0)))),
    (2, dict(rope=_rope(pos_rows=2, sections=(ctypes.c_int32 * 4)(16, 16, 0, 0)), stride=7)),
    (2, dict(rope=_rope(pos_rows=3, sections=(ctypes.c_int32 * 4)(16, 8, 8, 0)), stride=1 << 61)),
    (1, dict(rope=_rope(factor=math.inf))), (1, dict(rope=_rope(factor=1e300))), (1, dict(rope=_rope(freq=NAN_FREQ))),
    (2, dict(q=_heads(FAKE, 0, 8, 64))), (1, dict(q=_heads(None, 4, 8, 64))), (1, dict(q=_heads(FAKE, 4, 8, 64, reserved=1))),
    (2, dict(q=_heads(FAKE, 4, 8, 64, row_stride=63))), (2, dict(q=_heads(FAKE, 4, 8, 64, head_stride=0))),
    (2, dict(q=_heads(FAKE, 4, 8, 64, head_stride=-512))), (2, dict(q=_heads(FAKE, 4, 8, 64, head_stride=1 << 60))),
    (2, dict(q=_heads(FAKE, 3, 8, 64))), (1, dict(k=_heads(FAKE + (2 << 34), 1, 8, 64))),
    (5, dict(qo=_heads(FAKE + 128, 4, 8, 64))),                       # shifted onto its input
    (5, dict(qo=_heads(FAKE, 4, 8, 64, head_stride=64, row_stride=256))),   # its input in another order
    (5, dict(qo=_heads(FAKE + (5 << 34), 4, 8, 64))),                 # onto pos
    (5, dict(k=_heads(FAKE + (2 << 34), 4, 8, 64), ko=_heads(FAKE + (1 << 34) + 64, 4, 8, 64))),   # q_out and k_out
    (5, dict(k=_heads(FAKE + (1 << 34), 4, 8, 64), ko=_heads(FAKE + (3 << 34), 4, 8, 64))),         # q_out onto k
    (7, dict(q=_heads(FAKE, 1 << 17, 8, 64), qo=_heads(FAKE + (1 << 34), 1 << 17, 8, 64))),
])
def test_rotary_refusals(status, kw):
    st, msg = _rotary(**kw)
    assert st == status and msg


def test_rotary_of_more_rows_than_one_launch_takes():
    far = FAKE << 12                                          # rows of 511 single elements, one a workgroup
    st, msg = _rotary(rows=1 << 25, stride=1 << 25, d=511, pos=FAKE, q=_heads(far, 1, 1 << 25, 511),
                      qo=_heads(far << 1, 1, 1 << 25, 511))
    assert st == 7 and "too many rows" in msg


def test_rotary_of_no_rows_does_nothing():
    assert _rotary(rows=0, stride=0, pos=None)[0] == 0
    assert _status("apack_rotary", _rope(), 8, FAKE, 8, 0, 64, None, None, None, None, None)[0] == 0
    assert _status("apack_rotary", None, 8, FAKE, 8, 0, 64, None, None, None, None, None)[0] == 1


@pytest.mark.parametrize("status,kw", [
    (1, dict(n_layers=0)), (1, dict(n_layers=65)), (2, dict(n_pages=0)), (2, dict(page_rows=0)), (2, dict(hkv=0)),
    (2, dict(d=0)), (3, dict(dtype=7)), (1, dict(reserved=1)), (2, dict(row_stride=63)), (2, dict(head_stride=1023)),
    (2, dict(page_stride=0)), (2, dict(page_stride=-2048)), (2, dict(table_stride=3)), (2, dict(table_width=-1)),
    (1, dict(k0=0)), (2, dict(page_stride=1 << 62)),
])
def test_pool_refusals(status, kw):
    st, msg = _status("apack_pages_copy", _pages(**kw), 1, FAKE + (8 << 34), None)
    assert st == status and msg


def test_copy_refusals():
    assert _status("apack_pages_copy", None, 1, FAKE, None)[0] == 1
    assert _status("apack_pages_copy", _pages(), -1, FAKE, None)[0] == 1
    assert _status("apack_pages_copy", _pages(), 1, None, None)[0] == 1
    assert _status("apack_pages_copy", _pages(), 1, FAKE + 16, None)[0] == 5
    assert _status("apack_pages_copy", _pages(), 0, None, None)[0] == 0
    for pairs in (1 << 31, 1 << 24, 1 << 62):                # more threads than one launch takes
        assert _status("apack_pages_copy", _pages(k0=FAKE << 8, v0=(FAKE << 8) + (1 << 34)), pairs, FAKE, None)[0] == 7


def _compact(seqs, src=FAKE + (8 << 34), pin=None, pout=None):
    arr = (D.Move * max(1, len(seqs)))(*seqs)
    return _status("apack_compact_kv_pages", len(seqs), arr, src, pin or _pages(),
                   pout or _pages(k0=FAKE + (3 << 34), v0=FAKE + (4 << 34)), None)


def _planes(rows=64, **kw):
    return _pages(n_pages=1, page_rows=rows, table=None, width=0, **kw)


OUT = dict(k0=FAKE + (3 << 34), v0=FAKE + (4 << 34))


@pytest.mark.parametrize("status,seqs,kw", [
    (2, [(-1, 4, 0, 2)], {}), (2, [(0, 4, 0, -2)], {}), (2, [(0, -4, 0, 2)], {}), (2, [(0, 4, -1, 2)], {}),
    (7, [(1 << 31, 4, 0, 2)], {}), (7, [(0, 4, (1 << 31) - 1, 2)], {}),
    (2, [(0, 4, 0, 5)], dict(src=None)),
    (2, [(0, 64, 62, 3)], {}),                                  # past the output table's 64 rows
    (2, [(62, 3, 0, 2)], dict(pin=_planes())), (2, [(0, 64, 62, 3)], dict(pout=_planes(**OUT))),
    (2, [(0, 4, 0, 2)], dict(pin=_pages(n_layers=2))), (2, [(0, 4, 0, 2)], dict(pin=_pages(hkv=1))),
    (2, [(0, 4, 0, 2)], dict(pin=_pages(d=128))), (2, [(0, 4, 0, 2)], dict(pin=_pages(v=False))),
    (3, [(0, 4, 0, 2)], dict(pin=_pages(dtype=1))), (2, [(0, 4, 0, 2)], dict(pin=_pages(table=None))),
    (5, [(0, 4, 0, 2)], dict(pout=_pages(k0=FAKE + 64, v0=FAKE + (4 << 34)))),      # shifted onto the input
    (5, [(0, 4, 0, 2)], dict(pin=_planes(), pout=_planes())),                       # planes onto themselves
    (5, [(0, 4, 0, 2)], dict(pout=_pages(k0=FAKE + (1 << 34), v0=FAKE))),           # K onto V
    (5, [(0, 4, 0, 2)], dict(pout=_pages(k0=FAKE + (3 << 34), v0=FAKE + (3 << 34)))),
    (5, [(0, 4, 0, 2)], dict(src=FAKE + (3 << 34) + 4)),
    (5, [(0, 4, 0, 2)], dict(pout=_pages(table=FAKE + (3 << 34), **OUT))),
    (2, [(0, 4, 0, 2)] * 2, dict(pin=_pages(table_stride=1 << 62))),
])
def test_compact_pages_refusals(status, seqs, kw):
    st, msg = _compact(seqs, **kw)
    assert st == status and msg


def test_compact_pages_of_nothing():
    assert _compact([])[0] == 0
    assert _compact([(0, 4, 0, 0), (4, 0, 0, 0)])[0] == 0
    assert _compact([(0, 4, 0, 0)], src=None, pout=_pages())[0] == 0     # within one pool


def test_slices_of_one_tensor_are_apart():
    # K and V of each page side by side: page_stride covers both.
    kw = dict(page_stride=2 * 2 * 16 * 64)
    pin = _pages(v0=FAKE + 2 * 16 * 64 * 2, **kw)
    pout = _pages(k0=FAKE + (3 << 34), v0=FAKE + (3 << 34) + 2 * 16 * 64 * 2, **kw)
    assert _compact([(0, 4, 0, 0)], pin=pin, pout=pout)[0] == 0
    pout = _pages(k0=FAKE + (3 << 34), v0=FAKE + (3 << 34) + 2 * 16 * 64, **kw)      # half a page over
    assert _compact([(0, 4, 0, 0)], pin=pin, pout=pout)[0] == 5


def _append(n=3, pos=FAKE + (10 << 34), lens=FAKE + (11 << 34), q=None, qo=None, k=None, v=None, pages=None, rope=None):
    q = q or _heads(FAKE + (12 << 34), 4, n, 64)
    qo = qo or _heads(FAKE + (13 << 34), 4, n, 64)
    k = k or _heads(FAKE + (14 << 34), 2, n, 64)
    v = v or _heads(FAKE + (15 << 34), 2, n, 64)
    return _status("apack_rotary_append", rope or _rope(), n, pos, n, lens, q, qo, k, v, pages or _pages(), None)


@pytest.mark.parametrize("status,kw", [
    (1, dict(pos=None)), (1, dict(lens=None)), (2, dict(n=-1)), (1, dict(pages=_pages(n_layers=2))),
    (1, dict(pages=_pages(v=False))), (1, dict(pages=_planes())), (2, dict(k=_heads(FAKE + (14 << 34), 1, 3, 64))),
    (2, dict(qo=_heads(FAKE + (13 << 34), 3, 3, 64))), (2, dict(rope=_rope(66))), (5, dict(q=_heads(FAKE, 4, 3, 64))),
    (5, dict(qo=_heads(FAKE, 4, 3, 64))), (5, dict(k=_heads(FAKE + 64, 2, 3, 64))), (5, dict(lens=FAKE + 4)),
    (5, dict(qo=_heads(FAKE + (11 << 34), 4, 3, 64))), (5, dict(qo=_heads(FAKE + (12 << 34) + 64, 4, 3, 64))),
    (5, dict(v=_heads(FAKE + (13 << 34), 2, 3, 64))), (5, dict(pages=_pages(table=FAKE + 8))),
    (2, dict(pages=_pages(table_stride=1 << 61))),
])
def test_append_refusals(status, kw):
    st, msg = _append(**kw)
    assert st == status and msg


def _attend(n=3, hq=4, q=None, out=None, lse=FAKE + (16 << 34), pages=None, lens=FAKE + (11 << 34), max_len=64, mask=None,
            mask_stride=64, window=0, scale=0.0, ws=FAKE + (17 << 34), ws_bytes=1 << 30):
    q = q or _heads(FAKE + (12 << 34), hq, n, 64)
    out = out or _heads(FAKE + (13 << 34), hq, n, 64)
    return _status("apack_paged_attention", n, hq, q, out, lse, pages or _pages(), lens, max_len, mask, mask_stride,
                   window, scale, ws, ws_bytes, None)


@pytest.mark.parametrize("status,kw", [
    (2, dict(n=-1)), (2, dict(hq=3)), (2, dict(hq=0)), (2, dict(max_len=-1)), (1, dict(window=-1)), (1, dict(scale=-1.0)),
    (1, dict(scale=math.nan)), (1, dict(scale=math.inf)), (1, dict(scale=1e-60)), (1, dict(scale=1e31)),
    (1, dict(lens=None)), (7, dict(max_len=1 << 31)), (7, dict(max_len=(1 << 31) - (1 << 16) + 1)),
    (7, dict(n=60000, max_len=2000000, ws_bytes=1 << 40)), (7, dict(hq=4096, q=_heads(FAKE + (12 << 34), 4096, 3, 64))),
    (7, dict(n=65536)), (2, dict(pages=_pages(table_stride=1 << 61))), (2, dict(mask=FAKE + (18 << 34), mask_stride=1 << 62)),
    (2, dict(mask=FAKE + (18 << 34), mask_stride=63)), (7, dict(pages=_pages(d=96))),
    (1, dict(pages=_pages(v=False))), (1, dict(pages=_planes())), (1, dict(pages=_pages(n_layers=2))),
    (2, dict(q=_heads(FAKE + (12 << 34), 2, 3, 64))), (7, dict(q=_heads((FAKE + (12 << 34)) + 2, 4, 3, 64))),
    (7, dict(pages=_pages(row_stride=68, head_stride=16 * 68, page_stride=2 * 16 * 68))),
    (4, dict(max_len=1 << 20, ws=None)), (4, dict(max_len=1 << 20, ws=FAKE + (17 << 34) + 128)),
    (4, dict(max_len=1 << 20, ws_bytes=256)), (5, dict(out=_heads(FAKE, 4, 3, 64))),
    (5, dict(out=_heads(FAKE + (12 << 34), 4, 3, 64))), (5, dict(lse=FAKE + (13 << 34))), (5, dict(lse=FAKE + 64)),
    (5, dict(max_len=1 << 20, ws=FAKE)), (5, dict(lse=FAKE + (18 << 34), mask=FAKE + (18 << 34))),
])
def test_attention_refusals(status, kw):
    st, msg = _attend(**kw)
    assert st == status and msg


def test_attention_workspace_covers_shorter_calls():
    f = A.apack_paged_attention_workspace
    for n, hq, hkv in ((1, 28, 4), (3, 8, 8), (64, 28, 4), (1, 32, 1), (700, 4, 2)):
        sizes = [f(n, hq, hkv, 128, m) for m in (0, 1, 100, 1000, 1290, 5000, 94028, 1 << 20)]
        assert sizes == sorted(sizes) and sizes[0] > 0 and all(s % 256 == 0 for s in sizes)
    assert f(1, 3, 2, 128, 10) == 0 and f(1, 4, 2, 96, 10) == 0 and f(-1, 4, 2, 64, 10) == 0


def test_binding_refuses_host_tensors():
    x = torch.zeros(4, 8, 64)
    i = torch.zeros(8, dtype=torch.int32)
    t = torch.zeros(8, 1, dtype=torch.int32)
    p = torch.zeros(3, 2, 16, 64)
    kv = torch.zeros(2, 8, 64)
    rope = A.apack_rope(64)
    for call in (lambda: A.apack_rotary(i, rope, x), lambda: A.apack_rotary_append(i, rope, x, kv, kv, p, p, t, i),
                 lambda: A.apack_paged_attention(x, p, p, t, i, 16),
                 lambda: A.apack_pages_copy(torch.zeros(1, 2, dtype=torch.int32), [p], [p]),
                 lambda: A.apack_compact_kv_pages(None, [(0, 8, 0, 8)], [kv], [kv], [p], [p], table_out=t[:1])):
        with pytest.raises(A.ApackError, match="CUDA tensor"):
            call()
    with pytest.raises(A.ApackError):
        A.apack_rotary(i, rope)


# -- tables, masks and position ids at their edges ----------------------------

def _compact_of(pin, pout, seqs):
    return _status("apack_compact_kv_pages", len(seqs), (D.Move * len(seqs))(*seqs), None, pin, pout, None)


def test_table_without_entries_is_a_table():
    """torch gives a tensor of no elements no address, and a NULL table says that the tensors are planes."""
    x, y = (torch.zeros(1, 2, 16, 64) for _ in range(2))
    empty = torch.empty(1, 0, dtype=torch.int32)
    pages = D._pages([y], [], empty, 1)
    assert pages.table and pages.table_width == 0
    st, msg = _compact_of(D._pages([x[0]], [], planes=True), pages, [(0, 16, 0, 4)])
    assert st == 2 and "past the output table" in msg
    pages = D._one_layer(x, y, x.dtype, torch.zeros(3, 5, dtype=torch.int32)[:, 2:2], 3, 64)
    assert pages.table and pages.table_width == 0
    assert not D._pages([y[0]], [], planes=True).table


def _elements(k0, p):
    return {k0 // 2 + i * p.page_stride + h * p.head_stride + r * p.row_stride + e
            for i in range(p.n_pages) for h in range(p.hkv) for r in range(p.page_rows) for e in range(p.d)}


def test_overlap_is_found_and_slices_of_one_tensor_pass():
    """Pools of one to three dimensions at small strides: any element in common is an alias; slices of one dimension of
    a larger tensor are none.  Nothing is moved."""
    rng = np.random.default_rng(7)
    met = passed = 0
    for turn in range(4000):
        d, counts = int(rng.integers(1, 4)), rng.integers(1, 4, 3)
        order = rng.permutation(3)
        # A larger tensor of which both sides are slices: `extra` times as many of one dimension, or of the run.
        extra, where = int(rng.integers(1, 4)), int(rng.integers(0, 4))
        strides, at = np.zeros(3, dtype=int), d * (extra if where == 3 else 1)
        for i in order:
            strides[i] = at * (extra if where == i and rng.integers(0, 2) else 1) + int(rng.integers(0, 2))
            at = strides[i] * counts[i]
        kw = dict(n_pages=int(counts[0]), hkv=int(counts[1]), page_rows=int(counts[2]), d=d, v=False,
                  page_stride=int(strides[0]), head_stride=int(strides[1]), row_stride=int(strides[2]))
        shift = 2 * int(rng.integers(1, max(2, at + 2)))
        pin, pout = _pages(k0=FAKE, **kw), _pages(k0=FAKE + shift, **kw)
        if turn % 3 == 0:                                    # other counts at the same strides
            kw["page_rows"] = 1
            pout = _pages(k0=FAKE + shift, **kw)
        st, _ = _compact([(0, 1, 0, 0)], src=None, pin=pin, pout=pout)
        if _elements(FAKE, pin) & _elements(FAKE + shift, pout):
            assert st == 5, (kw, shift)
            met += 1
        else:
            passed += st == 0
            assert st == 0 or turn % 3 == 0, (kw, shift)     # all three strides alike: exact
    assert met > 500 and passed > 500


def test_slices_within_the_heads_are_apart():
    # [pages][heads][K and V][rows][d].
    kw = dict(hkv=4, head_stride=2 * 16 * 64, page_stride=4 * 2 * 16 * 64)
    pin = _pages(v0=FAKE + 16 * 64 * 2, **kw)
    pout = _pages(k0=FAKE + (3 << 34), v0=FAKE + (3 << 34) + 16 * 64 * 2, **kw)
    assert _compact([(0, 4, 0, 0)], pin=pin, pout=pout)[0] == 0
    pout = _pages(k0=FAKE + (3 << 34), v0=FAKE + (3 << 34) + 16 * 64, **kw)      # half the rows over
    assert _compact([(0, 4, 0, 0)], pin=pin, pout=pout)[0] == 5
    # A projection [rows][heads][q, k and v][d], turned in place: refused only further on, for its many rows.
    rows, d, far = 1 << 25, 511, FAKE << 12
    q, k = (_heads(far + 2 * i * d, 2, rows, d, head_stride=3 * d, row_stride=6 * d) for i in range(2))
    st, msg = _rotary(rows=rows, stride=rows, d=d, pos=FAKE, q=q, qo=q, k=k, ko=k)
    assert st == 7 and "too many rows" in msg
    k = _heads(far + d, 2, rows, d, head_stride=3 * d, row_stride=6 * d)
    assert _rotary(rows=rows, stride=rows, d=d, pos=FAKE, q=q, qo=q, k=k, ko=k)[0] == 5


@pytest.mark.parametrize("hq,hkv", [(28, 4), (4, 2), (8, 8), (32, 1), (16, 16)])
def test_attention_workspace_covers_smaller_batches(hq, hkv):
    """A batch that shrinks, as sequences end, decodes on with the workspace of the whole."""
    f = A.apack_paged_attention_workspace
    heads = dict(hq=hq, q=_heads(FAKE + (12 << 34), hq, 64, 64), out=_heads(FAKE + (13 << 34), hq, 64, 64))
    for longest in (0, 1, 512, 513, 700, 1290, 1408, 2047, 2048, 2049, 9454):
        sizes = [f(n, hq, hkv, 64, longest) for n in range(0, 65)]
        assert sizes == sorted(sizes)
        for n in (1, 2, 3, 7, 16, 40, 64):
            for shorter in (longest, longest // 2, 513):
                # Refused for its outputs, which are looked at after the workspace.
                st, _ = _attend(n=n, pages=_pages(hkv=hkv), max_len=min(longest, shorter), lse=FAKE + 64,
                                ws_bytes=sizes[64], **heads)
                assert st == 5


def test_one_row_of_position_ids_for_all():
    # A row stride of 0; refused further on, q_out lying on its input (q's and lens' overlap for the append).
    rope = _rope(pos_rows=3, sections=(ctypes.c_int32 * 4)(16, 8, 8, 0))
    assert _rotary(rope=rope, stride=0, qo=_heads(FAKE + 128, 4, 8, 64))[0] == 5
    args = [_heads(FAKE + (i << 34), h, 3, 64) for i, h in ((12, 4), (11, 4), (14, 2), (15, 2))]
    assert _status("apack_rotary_append", rope, 3, FAKE + (10 << 34), 0, FAKE + (11 << 34), *args, _pages(), None)[0] == 5
    for stride in (1, 7, -8):
        assert _rotary(rope=rope, stride=stride)[0] == 2
    # Onto the last of the ids.
    far = _heads(FAKE + (5 << 34) + 4 * 8, 4, 8, 64)
    assert _rotary(rope=rope, stride=0, q=far, qo=_heads(FAKE + (5 << 34) + 4 * 7, 4, 8, 64))[0] == 5


def test_one_mask_for_all_sequences():
    # A row stride of 0; refused further on, lse lying on the mask's row.
    mask = FAKE + (18 << 34)
    assert _attend(mask=mask, mask_stride=0, lse=mask + 60)[0] == 5
    for stride in (1, 63, -64):
        assert _attend(mask=mask, mask_stride=stride)[0] == 2


def test_one_table_for_all_sequences():
    # A row stride of 0; refused further on: an output lies on the table's row, or (moved nothing) not at all.
    table = FAKE + (9 << 34)
    assert _attend(pages=_pages(table_stride=0), lse=table + 12)[0] == 5
    assert _append(pages=_pages(table_stride=0), lens=table, qo=_heads(table, 4, 3, 64))[0] == 5
    assert _compact([(0, 4, 0, 0)] * 2, pout=_pages(table_stride=0, **OUT))[0] == 0
    for stride in (1, 3, -4):
        assert _compact([(0, 4, 0, 0)] * 2, pout=_pages(table_stride=stride, **OUT))[0] == 2

"""GPU parity of the rotary, paged-cache and decode calls against the fp64 oracle.

Tolerances count roundings.  u is half a step of fp32 (2^-24), h half a step of
the tensors' type.  A turned element is a c - b s with sines and cosines within
4 u of their values (a series, of an angle reduced in fp64), so it is within
8 u factor (|a| + |b|) of the formula, then rounded once (h); both sides form the
angle itself in fp64, within 2^-51 of |theta| together.

A logit is a sum of d products in fp32, within (d + 2) u scale sum |q k| of the
formula; call the largest such error e.  Probabilities then differ by a factor of
1 + 2 e, the exponential's argument (|x - m| <= 60 where it counts, two
roundings) adds 2^7 u, and sums over n rows n u.  With bf16 tensors the result is
rounded once more (h); probabilities keep 16 bits, for which most tests allow one
whole rounding (h) and the test of those bits 2^-16.
"""

import numpy as np
import pytest

from oracle import decode as OD
from tests.gpu_util import bits, log

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2608_08794_amd as A
    A.library()


def _dt(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _half(dtype):
    return torch.finfo(_dt(dtype)).eps / 2


def _f64(t):
    return t.detach().double().cpu().numpy()


def _rand(gen, dtype, *shape):
    return torch.randn(*shape, generator=gen, device="cuda").to(_dt(dtype))


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


# ---------------------------------------------------------------------------
# Rotary positions
# ---------------------------------------------------------------------------

def _rope(rot, layout="half", sections=None, **kw):
    import paper_2608_08794_amd as A
    return A.apack_rope(rot, base=1e6, layout=layout, sections=sections, **kw)


def _check_turned(got, x, pos, rope, layout, dtype, transpose=False):
    rot = rope.rot_dim
    freq = np.array(list(rope.freq)[:rot // 2])
    theta = OD.angles(np.atleast_2d(pos.cpu().numpy()), freq, list(rope.sections)[:rope.pos_rows])
    xx, got = _f64(x), _f64(got)
    want = OD.rotary(xx, theta, layout, rope.factor, transpose)
    size = OD.rotary(np.abs(xx), np.full_like(theta, np.pi / 4), layout, np.sqrt(2), True)   # |a| + |b| in the first half
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    size[..., b] = size[..., a]
    turn = np.zeros_like(want)
    turn[..., a] = turn[..., b] = np.abs(theta) * 2.0 ** -51
    tol = rope.factor * size * (8 * U + turn) + _half(dtype) * np.abs(want)
    assert (np.abs(got - want)[..., :rot] <= tol[..., :rot]).all(), np.abs(got - want)[..., :rot].max()
    np.testing.assert_array_equal(got[..., rot:], xx[..., rot:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rows,heads,d,rot,sections", [
    (1, (1, 1), 128, 128, None), (33, (28, 4), 128, 128, (16, 24, 24)), (64, (8, 2), 64, 32, None),
    (257, (3, 1), 64, 36, None), (5, (2, 2), 9, 8, (1, 2, 0, 1)), (7, (5, 1), 2, 2, None), (300, (1, 1), 512, 256, None),
    (1000, (70, 2), 80, 80, (0, 40)),
])
def test_rotary(dtype, layout, rows, heads, d, rot, sections):
    import paper_2608_08794_amd as A
    g = _gen(rows * d)
    rope = _rope(rot, layout, sections)
    q, k = (_rand(g, dtype, h, rows, d) for h in heads)
    shape = (rope.pos_rows, rows) if sections else (rows,)
    pos = torch.randint(-5000, 100000, shape, generator=g, device="cuda", dtype=torch.int32)
    keep = q.clone(), k.clone()
    qo, ko = A.apack_rotary(pos, rope, q, k)
    _check_turned(qo, q, pos, rope, layout, dtype)
    _check_turned(ko, k, pos, rope, layout, dtype)
    assert torch.equal(q, keep[0]) and torch.equal(k, keep[1])
    # The other way, one tensor alone, and in place: the same bits.
    to, none = A.apack_rotary(pos, rope, q=q, transpose=True)
    assert none is None and rope.transpose == 0
    _check_turned(to, q, pos, rope, layout, dtype, transpose=True)
    k2 = k.clone()
    A.apack_rotary(pos, rope, k=k2, k_out=k2)
    np.testing.assert_array_equal(bits(k2), bits(ko))


@pytest.mark.parametrize("scaling", ["linear", "ntk", "by_parts"])
def test_rotary_far_positions_and_scalings(scaling):
    import paper_2608_08794_amd as A
    g = _gen(9)
    rope = _rope(64, scaling=scaling, factor=8.0, trained_len=4096)
    x = _rand(g, "f32", 4, 6, 64)
    pos = torch.tensor([0, 1, -1, 1 << 20, 2**31 - 1, -2**31], dtype=torch.int32, device="cuda")
    y, _ = A.apack_rotary(pos, rope, x)
    _check_turned(y, x, pos, rope, "half", "f32")
    if scaling != "by_parts":
        assert torch.equal(y[:, 0], x[:, 0])


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 36), ("f32", 64)])
def test_rotary_strides(dtype, d):
    """A fused projection [rows][q heads | k heads | v heads][d]: slices in, planes out; and in place."""
    import paper_2608_08794_amd as A
    g = _gen(11)
    rope = _rope(d)
    fused = _rand(g, dtype, 37, 6 + 2 + 2, d)
    pos = torch.arange(37, dtype=torch.int32, device="cuda")
    q, k = fused[:, :6].transpose(0, 1), fused[:, 6:8].transpose(0, 1)
    qo, ko = A.apack_rotary(pos, rope, q, k)
    assert qo.is_contiguous()
    _check_turned(qo, q, pos, rope, "half", dtype)
    _check_turned(ko, k, pos, rope, "half", dtype)
    v = fused[:, 8:].clone()
    A.apack_rotary(pos, rope, q, k, q_out=q, k_out=k)
    np.testing.assert_array_equal(bits(q), bits(qo))
    np.testing.assert_array_equal(bits(k), bits(ko))
    assert torch.equal(fused[:, 8:], v)
    # Rows past the call's stay as they were.
    big = torch.full((6, 50, d), 7.0, dtype=_dt(dtype), device="cuda")
    A.apack_rotary(pos, rope, qo, q_out=big[:, 5:42])
    assert (big[:, :5] == 7).all() and (big[:, 42:] == 7).all()


def test_rotary_offsets_past_32_bits():
    import paper_2608_08794_amd as A
    base = torch.empty((2 << 30) + 4096, dtype=torch.bfloat16, device="cuda")
    x = base.as_strided((2, 3, 128), (256, 1 << 30, 1))
    x.copy_(_rand(_gen(12), "bf16", 2, 3, 128))
    pos = torch.tensor([3, 4, 5], dtype=torch.int32, device="cuda")
    rope = _rope(128)
    want, _ = A.apack_rotary(pos, rope, x.contiguous())
    _check_turned(want, x, pos, rope, "half", "bf16")
    A.apack_rotary(pos, rope, x, q_out=x)
    np.testing.assert_array_equal(bits(x), bits(want))


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotary_transposed_is_the_gradient(layout):
    """Against the formula's gradient, and against differences of the call itself: it is linear, so a difference of any
    size is exact but for rounding, and <R x, w> = <x, R' w>."""
    import paper_2608_08794_amd as A
    g = _gen(13)
    rope = _rope(48, layout, scaling="by_parts", factor=3.0, trained_len=100)
    x, w, dx = (_rand(g, "f32", 3, 20, 64) for _ in range(3))
    pos = torch.randint(0, 5000, (20,), generator=g, device="cuda", dtype=torch.int32)
    grad, _ = A.apack_rotary(pos, rope, w, transpose=True)
    theta = torch.tensor(OD.angles(pos.cpu().numpy()[None], np.array(list(rope.freq)[:24]), [24]))
    leaf = x.double().cpu().requires_grad_()
    a, b = (leaf[..., :24], leaf[..., 24:48]) if layout == "half" else (leaf[..., 0:48:2], leaf[..., 1:48:2])
    c, s = rope.factor * theta.cos(), rope.factor * theta.sin()
    ya, yb = a * c - b * s, a * s + b * c
    y = torch.cat([ya, yb] if layout == "half" else [torch.stack([ya, yb], -1).flatten(-2)], -1)
    (torch.cat([y, leaf[..., 48:]], -1) * w.double().cpu()).sum().backward()
    np.testing.assert_allclose(_f64(grad), leaf.grad.numpy(), rtol=0, atol=16 * U * 2 * float(w.abs().max()) * rope.factor)
    up, _ = A.apack_rotary(pos, rope, x + dx)
    at, _ = A.apack_rotary(pos, rope, x)
    lhs = ((up - at).double() * w.double()).sum().item()
    rhs = (dx.double() * grad.double()).sum().item()
    bound = 40 * U * rope.factor * 2 * float(((x.abs() + dx.abs()).double().sum() * w.abs().max().double()).item())
    assert abs(lhs - rhs) <= bound


# ---------------------------------------------------------------------------
# Pages
# ---------------------------------------------------------------------------

def _pool(gen, dtype, layers, pages, hkv, pr, d, how="heads"):
    """[layers, pages, hkv, pr, d] K and V of a pool, laid out as `how` says."""
    if how == "heads":
        return _rand(gen, dtype, layers, pages, hkv, pr, d), _rand(gen, dtype, layers, pages, hkv, pr, d)
    if how == "rows":                                     # [pages][rows][heads][d]
        return tuple(_rand(gen, dtype, layers, pages, pr, hkv, d).transpose(2, 3) for _ in range(2))
    if how == "pairs":                                    # K and V of a page side by side
        kv = _rand(gen, dtype, layers, pages, 2, hkv, pr, d)
        return kv[:, :, 0], kv[:, :, 1]
    if how == "padded":                                   # rows of d in longer ones
        return tuple(_rand(gen, dtype, layers, pages, hkv, pr, d + 3)[..., :d] for _ in range(2))
    raise AssertionError(how)


@pytest.mark.parametrize("dtype,layers,hkv,pr,d,how", [
    ("bf16", 3, 4, 16, 128, "heads"), ("bf16", 1, 2, 16, 128, "rows"), ("f32", 2, 2, 5, 64, "pairs"),
    ("bf16", 2, 3, 7, 9, "heads"), ("bf16", 1, 3, 7, 33, "padded"), ("f32", 1, 1, 1, 3, "rows"),
    ("bf16", 40, 1, 300, 64, "heads"),
])
def test_pages_copy(dtype, layers, hkv, pr, d, how):
    import paper_2608_08794_amd as A
    g = _gen(layers * pr)
    k, v = _pool(g, dtype, layers, 12, hkv, pr, d, how)
    want_k, want_v = k.clone(), v.clone()
    pairs = torch.tensor([[3, 1], [3, 0], [5, 11], [12, 2], [-1, 4], [6, 12], [7, -3]], dtype=torch.int32, device="cuda")
    for a, b in ((3, 1), (3, 0), (5, 11)):
        want_k[:, b], want_v[:, b] = k[:, a], v[:, a]
    A.apack_pages_copy(pairs, k, v)
    assert torch.equal(k, want_k) and torch.equal(v, want_v)
    # A list of layers, K alone.
    want_k[:, 8] = k[:, 9]
    A.apack_pages_copy(torch.tensor([[9, 8]], dtype=torch.int32, device="cuda"), list(k.unbind(0)))
    assert torch.equal(k, want_k) and torch.equal(v, want_v)
    A.apack_pages_copy(torch.empty((0, 2), dtype=torch.int32, device="cuda"), k, v)
    assert torch.equal(k, want_k)


def _random_table(gen, n, width, pages):
    t = torch.randperm(pages, generator=gen, device="cuda")[:n * width].int().view(n, width)
    return t.contiguous()


def _check_move(src_rows, seqs, k_in, k_out, before, table_in, table_out):
    """k_out (any layout) after a move of k_in against a loop over its rows; `before`: k_out's contents before."""
    want = before.clone()
    at = 0
    ti = table_in.cpu().numpy() if table_in is not None else None
    to = table_out.cpu().numpy() if table_out is not None else None
    rows = src_rows.cpu().tolist() if src_rows is not None else None
    for s, (so, n_in, do, n_out) in enumerate(seqs):
        for i in range(n_out):
            r = rows[at + i] - so if rows is not None else i
            if not 0 <= r < n_in:
                continue
            if ti is None:
                x = k_in[:, :, so + r]
            else:
                p = OD.place(ti[s], k_in.shape[3], r, k_in.shape[1])
                if p is None:
                    continue
                x = k_in[:, p[0], :, p[1]]
            if to is None:
                want[:, :, do + i] = x
            else:
                p = OD.place(to[s], k_out.shape[3], do + i, k_out.shape[1])
                if p is not None:
                    want[:, p[0], :, p[1]] = x
        at += n_out
    assert torch.equal(k_out, want)


@pytest.mark.parametrize("dtype,layers,hkv,d,pr_in,pr_out,how", [
    ("bf16", 2, 4, 128, 16, 16, "heads"), ("bf16", 1, 2, 128, 16, 48, "rows"), ("f32", 2, 2, 64, 5, 16, "pairs"),
    ("bf16", 1, 3, 33, 7, 1, "padded"), ("bf16", 30, 1, 64, 1, 32, "heads"), ("f32", 1, 1, 2048, 16, 16, "heads"),
    ("bf16", 1, 1, 2, 4, 4, "heads"),
])
@pytest.mark.parametrize("paged", [(True, True), (False, True), (True, False)])
def test_compact_pages(dtype, layers, hkv, d, pr_in, pr_out, how, paged):
    import paper_2608_08794_amd as A
    g = _gen(d + pr_in)
    sizes, outs = [70, 1, 0, 33], [41, 1, 0, 33]
    off = [0, 70, 71, 71]
    total = sum(sizes)
    rows = [torch.randperm(n, generator=g, device="cuda")[:m].sort().values.int() + o for n, m, o in zip(sizes, outs, off)]
    rows[0][3] = total + 5            # no row of the sequence: nothing is copied
    rows[0][7] = -1
    src = torch.cat(rows)
    table_in = table_out = None
    if paged[0]:
        table_in = _random_table(g, 4, -(-70 // pr_in), 4 * -(-70 // pr_in) + 2)
        k_in, v_in = _pool(g, dtype, layers, 4 * -(-70 // pr_in) + 2, hkv, pr_in, d, how)
        table_in[3, 0] = -1
        if table_in.shape[1] > 1:
            table_in[0, 1] = 1 << 20
    else:
        k_in, v_in = (_rand(g, dtype, layers, hkv, total + 9, d) for _ in range(2))
    if paged[1]:
        width = -(-50 // pr_out)
        dst = [5, 0, 0, 3]
        table_out = _random_table(g, 4, width, 4 * width + 1)
        k_out, v_out = _pool(g, dtype, layers, 4 * width + 1, hkv, pr_out, d, how)
        table_out[1, 0] = -7
    else:
        dst = [0, 41, 42, 44]
        k_out, v_out = (_rand(g, dtype, layers, hkv, 80, d) for _ in range(2))
    seqs = list(zip(off, sizes, dst, outs))
    k0, v0 = k_out.clone(), v_out.clone()
    A.apack_compact_kv_pages(src, seqs, k_in, v_in, k_out, v_out, table_in=table_in, table_out=table_out)
    _check_move(src, seqs, k_in, k_out, k0, table_in, table_out)
    _check_move(src, seqs, v_in, v_out, v0, table_in, table_out)
    # All first rows, K alone, layers as a list.
    k0 = k_out.clone()
    seqs = [(o, n, t, min(n, m)) for o, n, t, m in seqs]
    A.apack_compact_kv_pages(None, seqs, list(k_in.unbind(0)), [], list(k_out.unbind(0)), [], table_in=table_in,
                             table_out=table_out)
    _check_move(None, seqs, k_in, k_out, k0, table_in, table_out)


def test_compact_pages_of_many_sequences_within_one_pool():
    """More sequences than travel in one launch, out of and into pages of one pool."""
    import paper_2608_08794_amd as A
    g = _gen(21)
    n, pr = 131, 4
    k, v = _pool(g, "bf16", 2, 2 * n * 3, 2, pr, 64)
    t = _random_table(g, 2 * n, 3, 2 * n * 3)
    tin, tout = t[:n], t[n:]
    sizes = [(i * 7) % 13 for i in range(n)]
    off = np.concatenate([[0], np.cumsum(sizes)])[:-1].tolist()
    kept = [[r for r in range(s) if (r * 5 + i) % 3] for i, s in enumerate(sizes)]
    src = torch.tensor([o + r for o, x in zip(off, kept) for r in x], dtype=torch.int32, device="cuda")
    seqs = [(o, s, 0, len(x)) for o, s, x in zip(off, sizes, kept)]
    k0, v0 = k.clone(), v.clone()
    A.apack_compact_kv_pages(src, seqs, k, v, k, v, table_in=tin, table_out=tout)
    _check_move(src, seqs, k0, k, k0, tin, tout)
    _check_move(src, seqs, v0, v, v0, tin, tout)


def test_compact_pages_offsets_past_32_bits():
    import paper_2608_08794_amd as A
    base = torch.empty((2 << 30) + (1 << 20), dtype=torch.bfloat16, device="cuda")
    pool = base.as_strided((1, 3, 2, 16, 128), (0, 1 << 30, 2048, 128, 1))
    small = _rand(_gen(22), "bf16", 1, 3, 2, 16, 128)
    table = torch.tensor([[2, 0, 1]], dtype=torch.int32, device="cuda")
    A.apack_compact_kv_pages(None, [(0, 48, 0, 48)], list(small.unbind(0)), [], list(pool.unbind(0)), [], table_in=table,
                             table_out=table)
    assert torch.equal(pool, small)
    A.apack_pages_copy(torch.tensor([[2, 1]], dtype=torch.int32, device="cuda"), list(pool.unbind(0)))
    assert torch.equal(pool[:, 1], small[:, 2])


# ---------------------------------------------------------------------------
# Append
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,hq,hkv,d,rot,pr,how,layout", [
    ("bf16", 28, 4, 128, 128, 16, "heads", "half"), ("f32", 8, 2, 64, 32, 5, "rows", "interleaved"),
    ("bf16", 3, 1, 34, 18, 16, "padded", "half"), ("bf16", 4, 4, 64, 64, 1, "pairs", "interleaved"),
])
def test_rotary_append(dtype, hq, hkv, d, rot, pr, how, layout):
    import paper_2608_08794_amd as A
    g = _gen(hq * d)
    n, width = 9, 4
    kp, vp = (x[0] for x in _pool(g, dtype, 1, n * width + 1, hkv, pr, d, how))
    table = _random_table(g, n, width, n * width + 1)
    lens = torch.tensor([1, pr, pr + 1, 4 * pr, 4 * pr + 1, 0, -3, 2, 2**31 - 1], dtype=torch.int32, device="cuda")
    table[7, 0] = -1
    q, k, v = (_rand(g, dtype, n, h, d).transpose(0, 1) for h in (hq, hkv, hkv))
    pos = torch.randint(0, 9000, (3, n), generator=g, device="cuda", dtype=torch.int32)
    rope = _rope(rot, layout, (1, rot // 2 - 2, 1))
    k0, v0 = kp.clone(), vp.clone()
    qo = A.apack_rotary_append(pos, rope, q, k, v, kp, vp, table, lens)
    qw, kw = A.apack_rotary(pos, rope, q, k)
    _check_turned(qw, q, pos, rope, layout, dtype)
    assert torch.equal(qo, qw)
    for s in range(n):
        at = OD.place(table[s].tolist(), pr, int(lens[s]) - 1, kp.shape[0])
        assert (at is None) == (s in (4, 5, 6, 8) or (s == 7 and pr > 1))   # row 1 of sequence 7: page 0 or 1
        if at is not None:
            k0[at[0], :, at[1]], v0[at[0], :, at[1]] = kw[:, s], v[:, s]
    assert torch.equal(kp, k0) and torch.equal(vp, v0)
    q2 = q.contiguous()
    A.apack_rotary_append(pos, rope, q2, k, v, kp, vp, table, lens, q_out=q2)
    assert torch.equal(q2, qw) and torch.equal(kp, k0)


# ---------------------------------------------------------------------------
# Attention
# ---------------------------------------------------------------------------

def _check_attention(o, lse, q, kp, vp, table, lens, max_len, mask=None, window=0, scale=None, dtype="bf16", only=None):
    hq, n, d = q.shape
    scale = scale or d ** -0.5
    kk, vv, qq = _f64(kp), _f64(vp), _f64(q)
    o, lse = _f64(o), (None if lse is None else _f64(lse))
    h = _half(dtype) if dtype == "bf16" else 0.0
    tab, m = table.cpu().numpy(), (None if mask is None else mask.cpu().numpy())
    for s in range(n) if only is None else only:
        at = OD.rows_seen(tab[s], kp.shape[2], kp.shape[0], int(lens[s]), max_len, window, None if m is None else m[s])
        p, r = (np.array([x[i] for x in at], dtype=int) for i in range(2))
        want, wl, w, size = OD.attention(qq[:, s], kk[p, :, r].transpose(1, 0, 2), vv[p, :, r].transpose(1, 0, 2), scale)
        if not at:
            assert not o[:, s].any() and (lse is None or np.isneginf(lse[:, s]).all())
            continue
        if np.isnan(want).any():                        # a NaN among the rows attended to is not hidden
            assert np.isnan(want).all() and np.isnan(o[:, s]).all() and (lse is None or np.isnan(lse[:, s]).all())
            continue
        e = (d + 2) * U * size[:, None]
        rel = 2 * e + 2 ** 7 * U + 3 * len(at) * U
        tol = w * (rel + h) + (h + 4 * U) * np.abs(want)
        assert (np.abs(o[:, s] - want) <= tol).all(), (s, len(at), np.abs(o[:, s] - want).max(), tol.min())
        if lse is not None:
            assert (np.abs(lse[:, s] - wl) <= rel[:, 0] + 8 * U * np.abs(wl)).all(), (s, len(at))


def _paged(gen, dtype, lens, hkv, pr, d, how="heads", spare=2):
    """A pool with NaN wherever no sequence has a row, and the table."""
    counts = [-(-max(x, 0) // pr) for x in lens]
    width = max(max(counts), 1)
    kp, vp = (x[0] for x in _pool(gen, dtype, 1, sum(counts) + spare, hkv, pr, d, how))
    ids = torch.randperm(sum(counts) + spare, generator=gen, device="cuda").int()
    table = torch.full((len(lens), width), -1, dtype=torch.int32, device="cuda")
    used = torch.zeros(kp.shape[0], pr, dtype=torch.bool, device="cuda")
    at = 0
    for s, c in enumerate(counts):
        table[s, :c] = ids[at:at + c]
        u = used[table[s, :c].long()].flatten()
        u[:max(lens[s], 0)] = True
        used[table[s, :c].long()] = u.view(c, pr)
        at += c
    for x in (kp, vp):
        x.copy_(torch.where(used[:, None, :, None], x, float("nan")))
    return kp, vp, table, torch.tensor(lens, dtype=torch.int32, device="cuda")


CASES = [
    # hq, hkv, d, page rows, layout, lens
    (28, 4, 128, 16, "heads", [1, 0, 2, 15, 16, 17, 31, 32, 33, 127, 128, 129, 500]),
    (16, 2, 128, 16, "rows", [3000]),
    (8, 2, 64, 1, "pairs", [5, 300, 1]),
    (8, 8, 128, 48, "heads", [100, 2049, 7]),
    (32, 1, 64, 5, "heads", [333, 64]),
    (17, 1, 128, 7, "rows", [40, 257]),
    (1, 1, 64, 16, "heads", [0]),
    (28, 4, 128, 4096, "heads", [4000, 50]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,pr,how,lens", CASES)
def test_paged_attention(dtype, hq, hkv, d, pr, how, lens):
    import paper_2608_08794_amd as A
    g = _gen(hq + d + pr)
    kp, vp, table, n = _paged(g, dtype, lens, hkv, pr, d, how)
    q = _rand(g, dtype, len(lens), hq, d).transpose(0, 1)
    longest = max(lens)
    o, lse = A.apack_paged_attention(q, kp, vp, table, n, longest, return_lse=True)
    _check_attention(o, lse, q, kp, vp, table, n, longest, dtype=dtype)
    # A larger bound splits the rows otherwise; the same call twice gives the same bits.
    wide = A.apack_paged_attention(q, kp, vp, table, n, 40 * longest + 5000)
    _check_attention(wide, None, q, kp, vp, table, n, 40 * longest + 5000, dtype=dtype)
    again, lse2 = A.apack_paged_attention(q, kp, vp, table, n, longest, return_lse=True)
    np.testing.assert_array_equal(bits(again), bits(o))
    np.testing.assert_array_equal(bits(lse2), bits(lse))
    # Rows past max_len are left out.
    short = max(1, longest // 3)
    o, lse = A.apack_paged_attention(q, kp, vp, table, n, short, return_lse=True, scale=0.3)
    _check_attention(o, lse, q, kp, vp, table, n, short, scale=0.3, dtype=dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [1, 16, 100, 5000])
@pytest.mark.parametrize("bound", [700, 9000])
def test_paged_attention_window(dtype, window, bound):
    import paper_2608_08794_amd as A
    g = _gen(window)
    kp, vp, table, n = _paged(g, dtype, [700, 99, 100, 101, 1, 0], 2, 16, 128)
    # Rows that the window leaves out may hold anything.
    for s, x in enumerate(n.tolist()):
        for page in table[s, :max(0, x - window) // 16].tolist():
            kp[page], vp[page] = float("nan"), float("inf")
    q = _rand(g, dtype, 12, 6, 128)
    o, lse = A.apack_paged_attention(q, kp, vp, table, n, bound, window=window, return_lse=True)
    _check_attention(o, lse, q, kp, vp, table, n, bound, window=window, dtype=dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_paged_attention_masks_and_missing_pages(dtype):
    import paper_2608_08794_amd as A
    g = _gen(31)
    lens = [600, 40, 17, 300, 1]
    kp, vp, table, n = _paged(g, dtype, lens, 2, 16, 64)
    mask = torch.rand(5, 640, generator=g, device="cuda") < 0.4
    mask[1] = False                                      # nothing to attend to
    mask[2, :16] = False
    mask[4, 0] = True
    for s in range(5):                                   # masked rows hold NaN and infinities
        for r in (~mask[s, :lens[s]]).nonzero().flatten().tolist():
            page, at = int(table[s, r // 16]), r % 16
            kp[page, :, at], vp[page, :, at] = float("inf"), float("nan")
    table[3, 2], table[3, 5], table[3, 18] = -1, kp.shape[0], 2**31 - 1
    q = _rand(g, dtype, 5, 8, 64).transpose(0, 1)
    wide = torch.ones(5, 999, dtype=torch.uint8, device="cuda")
    wide[:, :640] = mask.to(torch.uint8) * 200
    for m in (mask, wide[:, :640]):
        o, lse = A.apack_paged_attention(q, kp, vp, table, n, 640, mask=m, return_lse=True)
        _check_attention(o, lse, q, kp, vp, table, n, 640, mask=mask, dtype=dtype)
    o, lse = A.apack_paged_attention(q, kp, vp, torch.full_like(table, -1), n, 640, return_lse=True)
    assert not o.any() and torch.isneginf(lse).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_paged_attention_of_large_logits(dtype):
    """One row takes all; then equal rows; logits of a few thousand."""
    import paper_2608_08794_amd as A
    g = _gen(33)
    kp, vp, table, n = _paged(g, dtype, [777, 333], 2, 16, 128)
    q = _rand(g, dtype, 4, 2, 128)
    kp.mul_(200)
    o, lse = A.apack_paged_attention(q, kp, vp, table, n, 777, return_lse=True)
    _check_attention(o, lse, q, kp, vp, table, n, 777, dtype=dtype)
    kp.copy_(torch.where(kp.isnan(), kp, torch.ones_like(kp)))
    o, lse = A.apack_paged_attention(q, kp, vp, table, n, 777, return_lse=True)
    _check_attention(o, lse, q, kp, vp, table, n, 777, dtype=dtype)


def test_paged_attention_outputs_and_their_surroundings():
    import paper_2608_08794_amd as A
    g = _gen(34)
    kp, vp, table, n = _paged(g, "bf16", [300, 20, 5], 2, 16, 64)
    q = _rand(g, "bf16", 6, 3, 64)
    want = A.apack_paged_attention(q, kp, vp, table, n, 300)
    room = torch.full((5, 7, 70), 3.0, dtype=torch.bfloat16, device="cuda")     # [seqs][heads][d] and more
    out = room[1:4, :6, :64].transpose(0, 1)
    k0 = kp.clone()
    A.apack_paged_attention(q, kp, vp, table, n, 300, out=out)
    assert torch.equal(out, want)
    out.fill_(3.0)
    assert (room == 3).all()
    np.testing.assert_array_equal(bits(kp), bits(k0))
    empty = A.apack_paged_attention(q[:, :0], kp, vp, table[:0], n[:0], 300)
    assert empty.shape == (6, 0, 64)
    A.apack_compact_kv_pages(None, [], [kp], [vp], [kp], [vp], table_in=table[:0], table_out=table[:0])
    A.apack_rotary_append(n[:0], A.apack_rope(64), q[:, :0], q[:2, :0], q[:2, :0], kp, vp, table[:0], n[:0])
    zero, lse = A.apack_paged_attention(q, kp, vp, table, n, 0, return_lse=True)
    assert not zero.any() and torch.isneginf(lse).all()


def test_paged_attention_joins_by_lse():
    """Attention over all rows is that over two parts, weighed by their exponentials."""
    import paper_2608_08794_amd as A
    g = _gen(35)
    kp, vp, table, n = _paged(g, "f32", [640], 2, 16, 64)
    q = _rand(g, "f32", 4, 1, 64)
    mask = (torch.arange(640, device="cuda") % 3 == 0)[None]
    o, lse = A.apack_paged_attention(q, kp, vp, table, n, 640, return_lse=True)
    o1, l1 = A.apack_paged_attention(q, kp, vp, table, n, 640, mask=mask, return_lse=True)
    o2, l2 = A.apack_paged_attention(q, kp, vp, table, n, 640, mask=~mask, return_lse=True)
    w = torch.softmax(torch.stack([l1, l2]).double(), 0)[..., None]
    torch.testing.assert_close((w[0] * o1 + w[1] * o2).float(), o, rtol=0, atol=2e-5)
    torch.testing.assert_close(torch.logaddexp(l1, l2), lse, rtol=0, atol=2e-5)


def test_paged_attention_far_pages_and_many_sequences():
    import paper_2608_08794_amd as A
    g = _gen(36)
    base = torch.empty((2 << 30) + (1 << 20), dtype=torch.bfloat16, device="cuda")
    kp = base.as_strided((3, 2, 16, 128), (1 << 30, 2048, 128, 1))
    vp = base.as_strided((3, 2, 16, 128), (1 << 30, 2048, 128, 1), 1 << 16)
    kp.copy_(_rand(g, "bf16", 3, 2, 16, 128))
    vp.copy_(_rand(g, "bf16", 3, 2, 16, 128))
    table = torch.tensor([[2, 0, 1], [1, 2, 0]], dtype=torch.int32, device="cuda")
    n = torch.tensor([48, 41], dtype=torch.int32, device="cuda")
    q = _rand(g, "bf16", 4, 2, 128)
    o, lse = A.apack_paged_attention(q, kp, vp, table, n, 48, return_lse=True)
    _check_attention(o, lse, q, kp, vp, table, n, 48)
    # Thousands of sequences that share pages.
    seqs = 3001
    table = table[torch.randint(0, 2, (seqs,), generator=g, device="cuda")].contiguous()
    n = torch.randint(0, 49, (seqs,), generator=g, device="cuda", dtype=torch.int32)
    q = _rand(g, "bf16", 4, seqs, 128)
    o, lse = A.apack_paged_attention(q, kp, vp, table, n, 48, return_lse=True)
    _check_attention(o, lse, q, kp, vp, table, n, 48, only=range(0, seqs, 97))


def test_paged_attention_long_cache():
    import paper_2608_08794_amd as A
    g = _gen(37)
    kp, vp, table, n = _paged(g, "bf16", [94028, 3], 4, 16, 128)
    q = _rand(g, "bf16", 2, 28, 128).transpose(0, 1)
    o, lse = A.apack_paged_attention(q, kp, vp, table, n, 94028, return_lse=True)
    _check_attention(o, lse, q, kp, vp, table, n, 94028)


# ---------------------------------------------------------------------------
# Together
# ---------------------------------------------------------------------------

class Decoder:
    """A two-layer cache after a prune, decoded a token at a time; `truth` holds each sequence's rows in fp64."""

    hq, hkv, d, pr, dtype = 8, 2, 64, 16, "bf16"

    def __init__(self, seed=41):
        import paper_2608_08794_amd as A
        self.A, self.g = A, _gen(seed)
        self.rope = A.apack_rope(self.d, base=1e4, sections=(8, 12, 12))

    def rand(self, *shape):
        return _rand(self.g, self.dtype, *shape)

    def step(self, kp, vp, table, lens, pos, layer, max_len):
        n = table.shape[0]
        q, k, v = (self.rand(n, h, self.d).transpose(0, 1) for h in (self.hq, self.hkv, self.hkv))
        qt = self.A.apack_rotary_append(pos, self.rope, q, k, v, kp[layer], vp[layer], table, lens)
        o, lse = self.A.apack_paged_attention(qt, kp[layer], vp[layer], table, lens, max_len, return_lse=True)
        _check_turned(qt, q, pos, self.rope, "half", self.dtype)
        _check_attention(o, lse, qt, kp[layer], vp[layer], table, lens, max_len, dtype=self.dtype)
        return k, v


def test_prune_compact_fork_and_decode():
    """Prefill, rotate, prune, compact into pages, fork, decode the children, compact the pages again."""
    D = Decoder()
    A, d, pr = D.A, D.d, D.pr
    sizes = [300, 130]
    off, total = [0, 300], 430
    pos = torch.stack([torch.arange(total, device="cuda"), torch.arange(total, device="cuda") // 3,
                       torch.arange(total, device="cuda") % 7]).int()
    proj = [D.rand(total, D.hq + 2 * D.hkv, d) for _ in range(2)]      # two layers' fused projections
    planes_k, planes_v = [], []
    for x in proj:
        q, k, v = x[:, :D.hq].transpose(0, 1), x[:, D.hq:-D.hkv].transpose(0, 1), x[:, -D.hkv:].transpose(0, 1)
        qt, kt = A.apack_rotary(pos, D.rope, q, k)
        planes_k.append(kt)
        planes_v.append(v.contiguous())
    seqs = [dict(tok_off=o, n_tokens=n, spans=[(0, n // 2, 1), (n // 2, n // 2 - 10, 2)], q_off=o + n - 8, q_len=8,
                 keep=(0.4, 0.3)) for o, n in zip(off, sizes)]
    _, kept, n_kept = A.apack_prune_layer(qt, planes_k[1], seqs)
    # Pages for what each keeps and for what it will say.
    refs = torch.zeros(80, dtype=torch.int32)
    kp, vp = (D.rand(2, 80, D.hkv, pr, d) for _ in range(2))
    tables = [A.apack_pages_alloc(refs, -(-(n + 4) // pr)) for n in n_kept]
    table = torch.full((2, 24), -1, dtype=torch.int32)
    for s, t in enumerate(tables):
        table[s, :t.numel()] = t
    table = table.cuda()
    moves = [(o, n, 0, m) for o, n, m in zip(off, sizes, n_kept)]
    before = kp.clone()
    A.apack_compact_kv_pages(kept, moves, planes_k, planes_v, kp, vp, table_out=table)
    _check_move(kept, moves, torch.stack(planes_k), kp, before, None, table)
    kept_pos = torch.empty(3, sum(n_kept), dtype=torch.int32, device="cuda")
    A.apack_compact_kv(kept, total, pos_in=pos, pos_out=kept_pos)
    assert torch.equal(kept_pos, pos[:, kept.long()])
    # Decode four tokens of both sequences.
    lens = torch.tensor(n_kept, dtype=torch.int32, device="cuda")
    for t in range(4):
        lens += 1
        for layer in range(2):
            D.step(kp, vp, table, lens, torch.full((3, 2), total + t, dtype=torch.int32, device="cuda"), layer, 24 * pr)
    # Fork the first into three; the parent's last page is copied for each.
    n0 = int(lens[0])
    children, copies = A.apack_pages_fork(refs, pr, n0, tables[0], 3)
    assert copies.shape[0] == (3 if n0 % pr else 0)
    A.apack_pages_copy(copies.cuda(), kp, vp)
    parent_rows = [kp[layer][table[0, :children.shape[1]].long()].clone() for layer in range(2)]
    more = [A.apack_pages_alloc(refs, 1) for _ in range(3)]
    ctable = torch.cat([children, torch.stack(more)], 1).cuda()
    clens = torch.full((3,), n0, dtype=torch.int32, device="cuda")
    for t in range(pr):
        clens += 1
        for layer in range(2):
            D.step(kp, vp, ctable, clens, torch.randint(0, 999, (3, 3), dtype=torch.int32, device="cuda"), layer, 24 * pr)
    for layer in range(2):
        assert torch.equal(kp[layer][table[0, :children.shape[1]].long()], parent_rows[layer])
    # Compact a child within the pool, free its old pages, decode on.
    keep = torch.arange(0, n0 + pr, 2, dtype=torch.int32, device="cuda")
    fresh = A.apack_pages_alloc(refs, -(-(keep.numel() + 1) // pr))
    ftable = fresh[None].cuda()
    before = kp.clone()
    A.apack_compact_kv_pages(keep, [(0, n0 + pr, 0, keep.numel())], kp, vp, kp, vp, table_in=ctable[1:2], table_out=ftable)
    _check_move(keep, [(0, n0 + pr, 0, keep.numel())], before, kp, before, ctable[1:2], ftable)
    A.apack_pages_free(refs, torch.cat([children[1], more[1]]))
    flens = torch.tensor([keep.numel() + 1], dtype=torch.int32, device="cuda")
    for layer in range(2):
        D.step(kp, vp, ftable, flens, torch.full((3, 1), 2000, dtype=torch.int32, device="cuda"), layer, 24 * pr)
    # Back to planes, for a prune of a layer that lives in pages.
    plane = torch.empty(D.hkv, int(flens[0]), d, dtype=torch.bfloat16, device="cuda")
    A.apack_compact_kv_pages(None, [(0, int(flens[0]), 0, int(flens[0]))], [kp[1]], [], [plane], [], table_in=ftable)
    q = D.rand(D.hq, 1, d)
    rows = int(flens[0])
    _, again, n_again = A.apack_prune_layer(q, plane, [dict(tok_off=0, n_tokens=rows, spans=[(0, rows - 1, 2)], q_off=0,
                                                            q_len=1, keep=(0.0, 0.5))])
    assert n_again == [again.numel()]
    for t in (tables[0], tables[1], torch.cat([children[0], more[0]]), torch.cat([children[2], more[2]]), fresh):
        A.apack_pages_free(refs, t)
    assert not refs.any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_several_new_tokens_of_one_sequence(dtype):
    """Four tokens of one sequence and two of another in one call of each, tables as columns of a wider one."""
    import paper_2608_08794_amd as A
    g = _gen(61)
    kp, vp = (_rand(g, dtype, 9, 2, 16, 64) for _ in range(2))
    wide = torch.full((6, 11), 77, dtype=torch.int32, device="cuda")
    table = wide[:, 2:6]
    table.copy_(torch.tensor([[3, 1, 8, -1]] * 4 + [[0, 5, 2, 4]] * 2, dtype=torch.int32))
    lens = torch.tensor([15, 16, 17, 18, 50, 51], dtype=torch.int32, device="cuda")
    q, k, v = (_rand(g, dtype, h, 6, 64) for h in (8, 2, 2))
    rope = A.apack_rope(64, layout="interleaved")
    k0, v0 = kp.clone(), vp.clone()
    qt = A.apack_rotary_append(lens, rope, q, k, v, kp, vp, table, lens)
    _, kt = A.apack_rotary(lens, rope, q, k)
    for s, n in enumerate(lens.tolist()):
        page, row = OD.place(table[s].tolist(), 16, n - 1, 9)
        k0[page, :, row], v0[page, :, row] = kt[:, s], v[:, s]
    assert torch.equal(kp, k0) and torch.equal(vp, v0)
    o, lse = A.apack_paged_attention(qt, kp, vp, table, lens, 64, return_lse=True)
    _check_attention(o, lse, qt, kp, vp, table, lens, 64, dtype=dtype)


def test_calls_of_no_rows():
    import paper_2608_08794_amd as A
    rope = A.apack_rope(64)
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    x = torch.empty(4, 0, 64, device="cuda")
    q, k = A.apack_rotary(none, rope, x, x[:2])
    assert q.shape == (4, 0, 64) and k.shape == (2, 0, 64)
    p = torch.ones(1, 3, 2, 16, 64, device="cuda")
    A.apack_compact_kv_pages(none, [(0, 5, 0, 0)], p, [], torch.zeros(1, 2, 7, 64, device="cuda"), [],
                             table_in=torch.zeros(1, 1, dtype=torch.int32, device="cuda"))
    assert (p == 1).all()


def _decode_once(A, rope, st):
    qt = A.apack_rotary_append(st["pos"], rope, st["q"], st["k"], st["v"], st["kp"], st["vp"], st["table"], st["lens"],
                               q_out=st["qt"])
    A.apack_paged_attention(qt, st["kp"], st["vp"], st["table"], st["lens"], st["max_len"], out=st["o"], lse=st["lse"],
                            workspace=st["ws"])
    return st["o"]


def _state(A, g, lens, max_len, hq=28, hkv=4, d=128):
    kp, vp, table, n = _paged(g, "bf16", [max_len] * len(lens), hkv, 16, d)
    b = len(lens)
    return dict(kp=kp, vp=vp, table=table, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), max_len=max_len,
                pos=torch.tensor(lens, dtype=torch.int32, device="cuda"),
                q=_rand(g, "bf16", hq, b, d), k=_rand(g, "bf16", hkv, b, d), v=_rand(g, "bf16", hkv, b, d),
                qt=torch.empty(hq, b, d, dtype=torch.bfloat16, device="cuda"),
                o=torch.empty(hq, b, d, dtype=torch.bfloat16, device="cuda"),
                lse=torch.empty(hq, b, dtype=torch.float32, device="cuda"),
                ws=torch.empty(A.apack_paged_attention_workspace(b, hq, hkv, d, max_len), dtype=torch.uint8, device="cuda"))


def test_captured_decode_step_is_replayed_as_lengths_grow():
    """Two graphs of decode steps, replayed in turn with the program's own work between; each replay against eager."""
    import paper_2608_08794_amd as A
    g = _gen(51)
    rope = A.apack_rope(128)
    states = [_state(A, g, [5, 900, 1, 2000], 3000), _state(A, g, [40], 700)]
    graphs = []
    for st in states:
        _decode_once(A, rope, st)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            _decode_once(A, rope, st)
        graphs.append(graph)
    for turn in range(4):
        for st, graph in zip(states, graphs):
            st["lens"] += 1 + 97 * turn
            st["pos"] += 1
            for x in ("q", "k", "v"):
                st[x].copy_(_rand(g, "bf16", *st[x].shape))
            st["o"].fill_(9)
            graph.replay()
            torch.cuda.synchronize()
            got, lse = st["o"].clone(), st["lse"].clone()
            want = _decode_once(A, rope, st)
            torch.cuda.synchronize()
            np.testing.assert_array_equal(bits(got), bits(want))
            np.testing.assert_array_equal(bits(lse), bits(st["lse"]))
            _check_attention(got, lse, st["qt"], st["kp"], st["vp"], st["table"], st["lens"], st["max_len"])


def test_two_graphs_share_a_workspace():
    """Replayed in turn on one stream: each call writes what it reads."""
    import paper_2608_08794_amd as A
    g = _gen(54)
    rope = A.apack_rope(128)
    states = [_state(A, g, [900, 30, 2000], 3000), _state(A, g, [2500], 3000)]
    for st in states:
        st["ws"] = states[0]["ws"]
    want, graphs = [], []
    for st in states:
        want.append(_decode_once(A, rope, st).clone())
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            _decode_once(A, rope, st)
        graphs.append(graph)
    states[0]["ws"].fill_(255)                             # NaN in every part
    for _ in range(3):
        for st in states:
            st["o"].fill_(9)
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for st, w in zip(states, want):
            np.testing.assert_array_equal(bits(st["o"]), bits(w))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_paged_attention_with_far_bounds(dtype):
    """Bounds and windows near the largest that a call takes, over short sequences."""
    import paper_2608_08794_amd as A
    g = _gen(55)
    most = 2**31 - 2**16
    kp, vp, table, n = _paged(g, dtype, [700, 0, 33], 2, 16, 64)
    q = _rand(g, dtype, 6, 3, 64)
    for window in (0, most, 2**62):
        o, lse = A.apack_paged_attention(q, kp, vp, table, n, most, window=window, return_lse=True)
        _check_attention(o, lse, q, kp, vp, table, n, most, window=window, dtype=dtype)
    # Lengths beyond the bound and the table, none, and one that takes in rows of NaN.
    n = torch.tensor([2**31 - 1, -2**31, 40], dtype=torch.int32, device="cuda")
    for bound, window in ((700, 0), (33, 0), (most, 50)):
        o, lse = A.apack_paged_attention(q, kp, vp, table, n, bound, window=window, return_lse=True)
        _check_attention(o, lse, q, kp, vp, table, n, bound, window=window, dtype=dtype)


def test_entry_points_on_side_streams():
    """Every call on a stream of its own, two of them at once, with default outputs and workspaces."""
    import paper_2608_08794_amd as A
    g = _gen(52)
    rope = A.apack_rope(128)
    states = [_state(A, g, [300, 900, 1], 1000) for _ in range(2)]
    want = []
    for st in states:
        kp, vp = st["kp"].clone(), st["vp"].clone()
        qt = A.apack_rotary_append(st["pos"], rope, st["q"], st["k"], st["v"], kp, vp, st["table"], st["lens"])
        o = A.apack_paged_attention(qt, kp, vp, st["table"], st["lens"], 1000)
        plane = torch.zeros(4, 900, 128, dtype=torch.bfloat16, device="cuda")
        A.apack_compact_kv_pages(None, [(0, 0, 0, 0), (0, 900, 0, 900)], [kp], [], [plane], [], table_in=st["table"][:2])
        r, _ = A.apack_rotary(torch.arange(900, dtype=torch.int32, device="cuda"), rope, plane)
        kp[7] = kp[3]
        want.append((o, r, kp))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    pos = torch.arange(900, dtype=torch.int32, device="cuda")
    pairs = torch.tensor([[3, 7]], dtype=torch.int32, device="cuda")
    planes = [torch.zeros(4, 900, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for st, s, plane in zip(states, streams, planes):
        qt = A.apack_rotary_append(st["pos"], rope, st["q"], st["k"], st["v"], st["kp"], st["vp"], st["table"], st["lens"],
                                   stream=s)
        o = A.apack_paged_attention(qt, st["kp"], st["vp"], st["table"], st["lens"], 1000, stream=s)
        A.apack_compact_kv_pages(None, [(0, 0, 0, 0), (0, 900, 0, 900)], [st["kp"]], [], [plane], [],
                                 table_in=st["table"][:2], stream=s)
        r, _ = A.apack_rotary(pos, rope, plane, stream=s.cuda_stream)
        A.apack_pages_copy(pairs, [st["kp"]], stream=s)
        got.append((o, r, st["kp"]))
    for s in streams:
        s.synchronize()
    for a, b in zip(got, want):
        for x, y in zip(a, b):
            np.testing.assert_array_equal(bits(x), bits(y))


def test_binding_refusals():
    import paper_2608_08794_amd as A
    g = _gen(53)
    kp, vp, table, n = _paged(g, "bf16", [30, 4], 2, 16, 64)
    q = _rand(g, "bf16", 4, 2, 64)
    k = _rand(g, "bf16", 2, 2, 64)
    pos = torch.zeros(2, dtype=torch.int32, device="cuda")
    rope = A.apack_rope(64)
    bad = [
        lambda: A.apack_paged_attention(q.float(), kp, vp, table, n, 30),
        lambda: A.apack_paged_attention(q, kp, vp, table.long(), n, 30),
        lambda: A.apack_paged_attention(q, kp, vp, table[:1], n, 30),
        lambda: A.apack_paged_attention(q, kp, vp, table, n[:1], 30),
        lambda: A.apack_paged_attention(q, kp, vp[:1], table, n, 30),
        lambda: A.apack_paged_attention(q, kp, vp, table, n, 30, mask=torch.ones(2, 29, dtype=torch.bool, device="cuda")),
        lambda: A.apack_paged_attention(q, kp, vp, table, n, 30, mask=torch.ones(2, 30, device="cuda")),
        lambda: A.apack_paged_attention(q, kp, vp, table, n, 30, scale=0.0),
        lambda: A.apack_paged_attention(q[..., ::2], kp, vp, table, n, 30),
        lambda: A.apack_paged_attention(q, kp, vp, table, n, 30, out=q),
        lambda: A.apack_paged_attention(q, kp, vp, table, n, 30, lse=torch.empty(4, 3, device="cuda")),
        lambda: A.apack_paged_attention(q[:, :, :48], kp, vp, table, n, 30),
        lambda: A.apack_paged_attention(q.cpu(), kp, vp, table, n, 30),
        lambda: A.apack_rotary(pos.long(), rope, q),
        lambda: A.apack_rotary(pos[:1], rope, q),
        lambda: A.apack_rotary(pos, rope, q, k[:, :1]),
        lambda: A.apack_rotary(pos, rope, q.half()),
        lambda: A.apack_rotary(pos, rope, q, q_out=torch.empty(4, 3, 64, dtype=torch.bfloat16, device="cuda")),
        lambda: A.apack_rotary(pos, rope, q[..., ::2]),
        lambda: A.apack_rotary(pos, rope, q, k_out=k),
        lambda: A.apack_rotary(pos, A.apack_rope(64, sections=(16, 16)), q),
        lambda: A.apack_rotary_append(pos, rope, q, k[:1], k, kp, vp, table, n),
        lambda: A.apack_rotary_append(pos, rope, q, k, k, kp.float(), vp.float(), table, n),
        lambda: A.apack_pages_copy(pos, [kp], [vp]),
        lambda: A.apack_pages_copy(torch.zeros(1, 2, dtype=torch.int32, device="cuda"), [kp, kp[:1]], [vp, vp[:1]]),
        lambda: A.apack_compact_kv_pages(pos, [(0, 9, 0, 3)], [kp], [vp], [kp], [vp], table_in=table[:1], table_out=table[1:]),
    ]
    k0 = kp.clone()
    for i, call in enumerate(bad):
        with pytest.raises(A.ApackError):
            call()
            log(f"call {i} was not refused")
    torch.cuda.synchronize()
    np.testing.assert_array_equal(bits(kp), bits(k0))


def test_layers_as_a_list_and_as_one_tensor():
    """K a list of layers and V one tensor, and the other way round."""
    import paper_2608_08794_amd as A
    g = _gen(59)
    kv = _rand(g, "bf16", 3, 2, 5, 2, 8, 16)
    pairs = torch.tensor([[1, 4], [0, 2]], dtype=torch.int32, device="cuda")
    want = kv.clone()
    want[:, :, 4], want[:, :, 2] = kv[:, :, 1], kv[:, :, 0]
    for k_list, v_list in ((True, False), (False, True), (True, True), (False, False)):
        got = kv.clone()
        k, v = got[:, 0], got[:, 1]
        A.apack_pages_copy(pairs, list(k) if k_list else k, list(v) if v_list else v)
        np.testing.assert_array_equal(bits(got), bits(want))
    for k, v in ((list(kv[:, 0]), kv[:2, 1]), (kv[:, 0], list(kv[:, 1].float())), (kv[:, 0], kv[:, 1, :, :1])):
        with pytest.raises(A.ApackError):
            A.apack_pages_copy(pairs, k, v)


def test_workspace_with_gaps_is_refused():
    import paper_2608_08794_amd as A
    g = _gen(61)
    kp, vp, table, n = _paged(g, "bf16", [30, 4], 2, 16, 64)
    q = _rand(g, "bf16", 4, 2, 64)
    need = max(256, A.apack_paged_attention_workspace(2, 4, 2, 64, 30))
    for ws in (torch.empty(1, dtype=torch.uint8, device="cuda").expand(need),
               torch.empty(2 * need, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(A.ApackError):
            A.apack_paged_attention(q, kp, vp, table, n, 30, workspace=ws)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_paged_attention_of_infinities(dtype):
    """Logits of -inf weigh nothing, one of +inf gives NaN; an infinite element of V stays in its element."""
    import paper_2608_08794_amd as A
    g = _gen(67)
    kp, vp, table, n = _paged(g, dtype, [100, 700], 2, 16, 64)
    kp, vp = kp.nan_to_num(0.0), vp.nan_to_num(0.0)
    q = _rand(g, dtype, 4, 2, 64).abs() + 1
    row = lambda s, j: (int(table[s, j // 16]), slice(None), j % 16)
    want, lse = A.apack_paged_attention(q, kp, vp, table, n, 700, return_lse=True)
    vi = vp.clone()
    for s, j in ((0, 40), (1, 600)):
        vi[row(s, j)][:, 7] = float("inf")
    got = A.apack_paged_attention(q, kp, vi, table, n, 700)
    assert not torch.isfinite(got[..., 7]).any()
    rest = [e for e in range(64) if e != 7]
    np.testing.assert_array_equal(bits(got[..., rest].contiguous()), bits(want[..., rest].contiguous()))
    ki = kp.clone()
    for j in range(100):
        ki[row(0, j)] = float("-inf")
    got, l = A.apack_paged_attention(q, ki, vp, table, n, 700, return_lse=True)
    assert not got[:, 0].any() and torch.isneginf(l[:, 0]).all()
    np.testing.assert_array_equal(bits(got[:, 1].contiguous()), bits(want[:, 1].contiguous()))
    np.testing.assert_array_equal(bits(l[:, 1].contiguous()), bits(lse[:, 1].contiguous()))
    ki = kp.clone()
    ki[row(1, 333)] = float("inf")
    got = A.apack_paged_attention(q, ki, vp, table, n, 700)
    assert got[:, 1].isnan().all()
    np.testing.assert_array_equal(bits(got[:, 0].contiguous()), bits(want[:, 0].contiguous()))


@pytest.mark.parametrize("dtype,hkv,lens,window", [
    ("bf16", 1, [0, 1, 5000, 31, 33, 0, 2500] * 10, 0),
    ("bf16", 4, [900, 0, 4001], 0),
    ("f32", 2, [3000, 2999, 1, 640, 0, 17], 0),
    ("bf16", 2, [5000, 4000, 700, 3, 0], 2049),
    ("f32", 8, [700, 513], 0)])
def test_paged_attention_of_few_ragged_sequences(dtype, hkv, lens, window):
    """Long spans of few sequences: every key head of a sequence is split on its own."""
    import paper_2608_08794_amd as A
    g = _gen(71)
    kp, vp, table, n = _paged(g, dtype, lens, hkv, 16, 128)
    q = _rand(g, dtype, 2 * hkv, len(lens), 128)
    o, lse = A.apack_paged_attention(q, kp, vp, table, n, 5000, window=window, return_lse=True)
    _check_attention(o, lse, q, kp, vp, table, n, 5000, window=window, dtype=dtype)
    again = A.apack_paged_attention(q, kp, vp, table, n, 5000, window=window)
    np.testing.assert_array_equal(bits(again), bits(o))


# ---------------------------------------------------------------------------
# Tables, masks and position ids at their edges
# ---------------------------------------------------------------------------

def test_tables_without_entries():
    """Every row is beyond such a table, also where the pool is one page."""
    import paper_2608_08794_amd as A
    g = _gen(81)
    kp, vp = (_rand(g, "bf16", 1, 2, 16, 64) for _ in range(2))
    k0, v0 = kp.clone(), vp.clone()
    q, k, v = (_rand(g, "bf16", h, 3, 64) for h in (4, 2, 2))
    n = torch.tensor([1, 5, 16], dtype=torch.int32, device="cuda")
    rope = A.apack_rope(64)
    for table in (torch.empty(3, 0, dtype=torch.int32, device="cuda"),
                  torch.zeros(3, 4, dtype=torch.int32, device="cuda")[:, 2:2]):
        o, lse = A.apack_paged_attention(q, kp, vp, table, n, 16, return_lse=True)
        assert not o.any() and torch.isneginf(lse).all()
        o, lse = A.apack_paged_attention(q, kp, vp, table, n, 5000, return_lse=True)
        assert not o.any() and torch.isneginf(lse).all()
        qt = A.apack_rotary_append(n, rope, q, k, v, kp, vp, table, n)
        assert torch.equal(qt, A.apack_rotary(n, rope, q)[0])
        plane = torch.full((2, 16, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        A.apack_compact_kv_pages(None, [(0, 16, 0, 16), (0, 0, 0, 0), (0, 0, 0, 0)], [kp], [], [plane], [], table_in=table)
        assert (plane == 7).all()
        with pytest.raises(A.ApackError, match="past the output table"):
            A.apack_compact_kv_pages(None, [(0, 16, 0, 1)] + [(0, 0, 0, 0)] * 2, [plane], [], [kp], [], table_out=table)
        assert torch.equal(kp, k0) and torch.equal(vp, v0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_slices_within_the_heads(dtype):
    """A projection [rows][heads][q, k and v][d] turned in place, and pools [pages][heads][K and V][rows][d]."""
    import paper_2608_08794_amd as A
    g = _gen(82)
    rope = _rope(64)
    fused = _rand(g, dtype, 40, 2, 3, 64)
    q, k, v = (x.transpose(0, 1) for x in fused.unbind(2))
    pos = torch.randint(0, 9000, (40,), generator=g, device="cuda", dtype=torch.int32)
    v0 = v.clone()
    qw, kw = A.apack_rotary(pos, rope, q.contiguous(), k.contiguous())
    A.apack_rotary(pos, rope, q, k, q_out=q, k_out=k)
    assert torch.equal(q, qw) and torch.equal(k, kw) and torch.equal(v, v0)
    pool, other = (_rand(g, dtype, 6, 2, 2, 16, 64) for _ in range(2))
    (kp, vp), (ko, vo) = pool.unbind(2), other.unbind(2)
    k1, v1 = kp.clone(), vp.clone()
    table = torch.tensor([[4, 1, 5]], dtype=torch.int32, device="cuda")
    A.apack_compact_kv_pages(None, [(0, 40, 0, 40)], [k], [v], [kp], [vp], table_out=table)
    for j in range(40):
        page, row = int(table[0, j // 16]), j % 16
        k1[page, :, row], v1[page, :, row] = k[:, j], v[:, j]
    assert torch.equal(kp, k1) and torch.equal(vp, v1)
    n = torch.tensor([41], dtype=torch.int32, device="cuda")
    new = _rand(g, dtype, 1, 2, 3, 64)
    q, k, v = (x.transpose(0, 1) for x in new.unbind(2))
    qt = A.apack_rotary_append(n, rope, q, k, v, kp, vp, table, n, q_out=q)
    k1[5, :, 8], v1[5, :, 8] = A.apack_rotary(n, rope, k=k)[1][:, 0], v[:, 0]
    assert torch.equal(kp, k1) and torch.equal(vp, v1)
    o, lse = A.apack_paged_attention(qt, kp, vp, table, n, 48, return_lse=True)
    _check_attention(o, lse, qt, kp, vp, table, n, 48, dtype=dtype)
    table_out = torch.tensor([[2, 0, 3]], dtype=torch.int32, device="cuda")
    A.apack_compact_kv_pages(None, [(0, 41, 0, 41)], [kp], [vp], [ko], [vo], table_in=table, table_out=table_out)
    A.apack_pages_copy(torch.tensor([[2, 4], [0, 1], [3, 5]], dtype=torch.int32, device="cuda"), [ko], [vo])
    assert torch.equal(ko[[4, 1]], k1[[4, 1]]) and torch.equal(vo[5, :, :9], v1[5, :, :9])


@pytest.mark.parametrize("rows", [1, 37])
def test_position_ids_expanded_from_one_row(rows):
    """Text tokens have the same id in every row."""
    import paper_2608_08794_amd as A
    g = _gen(83)
    rope = _rope(64, sections=(16, 8, 8))
    pos = torch.randint(0, 9000, (1, rows), generator=g, device="cuda", dtype=torch.int32).expand(3, rows)
    q, k, v = (_rand(g, "bf16", h, rows, 64) for h in (4, 2, 2))
    qt, kt = A.apack_rotary(pos, rope, q, k)
    _check_turned(qt, q, pos, rope, "half", "bf16")
    assert torch.equal(kt, A.apack_rotary(pos.contiguous(), rope, k=k)[1])
    kp, vp = (torch.zeros(rows, 2, 16, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.arange(rows, dtype=torch.int32, device="cuda")[:, None]
    assert torch.equal(A.apack_rotary_append(pos, rope, q, k, v, kp, vp, table, torch.full_like(pos[0], 4)), qt)
    assert torch.equal(kp[:, :, 3], kt.transpose(0, 1)) and torch.equal(vp[:, :, 3], v.transpose(0, 1))


@pytest.mark.parametrize("dtype,pr,longest", [("bf16", 16, 700), ("f32", 16, 5000), ("bf16", 7, 300)])
def test_mask_expanded_from_one_row(dtype, pr, longest):
    import paper_2608_08794_amd as A
    g = _gen(84)
    kp, vp, table, n = _paged(g, dtype, [longest, 40, 0, longest // 2], 2, pr, 64)
    q = _rand(g, dtype, 4, 4, 64)
    one = torch.rand(1, longest, generator=g, device="cuda") < 0.5
    for kind in (torch.bool, torch.uint8):
        mask = one.to(kind).expand(4, longest)
        o, lse = A.apack_paged_attention(q, kp, vp, table, n, longest, mask=mask, return_lse=True)
        _check_attention(o, lse, q, kp, vp, table, n, longest, mask=mask, dtype=dtype)
        again = A.apack_paged_attention(q, kp, vp, table, n, longest, mask=mask.contiguous())
        np.testing.assert_array_equal(bits(o), bits(again))


def test_table_expanded_from_one_row():
    """Several new tokens of one sequence, and moves into several parts of one."""
    import paper_2608_08794_amd as A
    g = _gen(85)
    kp, vp = (_rand(g, "bf16", 8, 2, 16, 64) for _ in range(2))
    k0, v0 = kp.clone(), vp.clone()
    one = torch.tensor([[6, 2, 3, 7]], dtype=torch.int32, device="cuda")
    table = one.expand(3, 4)
    lens = torch.tensor([32, 33, 34], dtype=torch.int32, device="cuda")
    q, k, v = (_rand(g, "bf16", h, 3, 64) for h in (4, 2, 2))
    rope = _rope(64)
    qt = A.apack_rotary_append(lens, rope, q, k, v, kp, vp, table, lens)
    kt = A.apack_rotary(lens, rope, k=k)[1]
    for s, (page, row) in enumerate([(2, 15), (3, 0), (3, 1)]):
        k0[page, :, row], v0[page, :, row] = kt[:, s], v[:, s]
    assert torch.equal(kp, k0) and torch.equal(vp, v0)
    o, lse = A.apack_paged_attention(qt, kp, vp, table, lens, 64, return_lse=True)
    _check_attention(o, lse, qt, kp, vp, table, lens, 64)
    plane = _rand(g, "bf16", 2, 30, 64)
    moves = [(0, 10, 20, 10), (10, 20, 35, 20), (30, 0, 0, 0)]
    A.apack_compact_kv_pages(None, moves, [plane], [], [kp], [], table_out=table)
    _check_move(None, moves, plane[None], kp[None], k0[None], None, table)
    back = torch.zeros_like(plane)
    A.apack_compact_kv_pages(torch.arange(20, 30, dtype=torch.int32, device="cuda").repeat(3),
                             [(0, 64, 10 * i, 10) for i in range(3)], [kp], [], [back], [], table_in=table)
    assert torch.equal(back, plane[:, :10].repeat(1, 3, 1))


# ---------------------------------------------------------------------------
# Probabilities in two bf16 parts
# ---------------------------------------------------------------------------

def _one_part(q, k, v, scale):
    """The oracle's output with each probability (of the largest) rounded once to bf16, in the products with V alone."""
    out = np.zeros_like(q)
    for h in range(q.shape[0]):
        g = h // (q.shape[0] // k.shape[0])
        x = scale * (k[g] @ q[h])
        p = np.exp(x - x.max())
        out[h] = torch.tensor(p).bfloat16().double().numpy() @ v[g] / p.sum()
    return out


@pytest.mark.parametrize("hq,hkv,d,pr", [(8, 2, 128, 16), (4, 4, 64, 5), (20, 1, 64, 32)])
def test_paged_attention_keeps_16_bits_of_probabilities(hq, hkv, d, pr):
    """Neighbouring rows have nearly the same K and opposite V, so that the output is small beside sum p |v| and its one
    rounding h |o| hides little.  The first part leaves at most h p, the second h of that: 2^-16 of each probability.
    Dropping the second part, as the oracle does here on the CPU, is out of this bound."""
    import paper_2608_08794_amd as A
    g = _gen(hq * d)
    lens = [2, 4, 8, 16, 64]
    kp, vp, table, n = _paged(g, "bf16", lens, hkv, pr, d)
    for s, rows in enumerate(lens):
        at = lambda j: (table[s, j // pr].long(), slice(None), j % pr)
        for j in range(1, rows, 2):
            kp[at(j)] = (kp[at(j - 1)].float() + 0.05 * torch.randn(hkv, d, generator=g, device="cuda")).bfloat16()
            vp[at(j)] = -vp[at(j - 1)]
    q = (0.25 * torch.randn(hq, len(lens), d, generator=g, device="cuda")).bfloat16()
    scale, h = d ** -0.5, _half("bf16")
    for bound in (64, 5000):                              # taken whole, and in shares
        o = _f64(A.apack_paged_attention(q, kp, vp, table, n, bound))
        for s, rows in enumerate(lens):
            page, row = (np.array([f(j) for j in range(rows)]) for f in (lambda j: int(table[s, j // pr]), lambda j: j % pr))
            qs, k, v = _f64(q[:, s]), *(_f64(x)[page, :, row].transpose(1, 0, 2) for x in (kp, vp))
            want, _, w, size = OD.attention(qs, k, v, scale)
            rel = 2 * (d + 2) * U * size[:, None] + 2 ** 7 * U + 3 * rows * U + 2.0 ** -16
            tol = w * rel + (h + 4 * U) * np.abs(want)
            assert (np.abs(o[:, s] - want) <= tol).all(), (rows, (np.abs(o[:, s] - want) / tol).max())
            assert (np.abs(_one_part(qs, k, v, scale) - want) > tol).any()


# ---------------------------------------------------------------------------
# How rows are dealt to workgroups
# ---------------------------------------------------------------------------

def _dealt(hq, hkv, d, lens, max_len, window):
    """("whole", "tiles": a share of one tile each, "own": in parts of each item's own, or "equal": equal shares of all
    tiles; tiles a share): as the kernel decides it, from the lengths, for these sizes."""
    import paper_2608_08794_amd as A
    n, group = len(lens), hq // hkv
    items = hkv * -(-group // 16)
    span = min(window, max_len) if window else max_len
    if span <= max(512, min(2048, 11 * n * items)):
        return "whole", 0
    shares = min(512, n * items * -(-span // 32))
    up = lambda x: -(-x // 256) * 256
    need = up(12 * n * items) + up(8 * shares * min(16, group) * (d + 4))
    if not window:                                        # the count of shares shows in the workspace
        assert A.apack_paged_attention_workspace(n, hq, hkv, d, max_len) == need
    tiles = 0
    for x in lens:
        lo = max(0, x - window) if window else 0
        tiles += max(1, -(-(min(x, max_len) - lo // 16 * 16) // 32)) if min(x, max_len) > lo else 1
    total, pieces = tiles * items, n * items
    shares = min(shares, total)
    if total <= shares:
        return "tiles", 1
    if n > 1 and pieces < shares and total * pieces <= 2 * shares * (shares - pieces):
        return "own", total / shares
    return "equal", total / shares


RAGGED = [(i * 2719) % 6001 if i % 7 else i % 34 for i in range(64)]   # 0 to 6000 rows; every seventh of 33 at most

DEALT = [
    # how, dtype, hq, hkv, d, page rows, window, masked, lens
    ("equal", "bf16", 28, 4, 128, 16, 0, False, [20011]),
    ("equal", "f32", 4, 2, 64, 16, 0, False, [20480]),
    ("equal", "bf16", 8, 4, 128, 16, 0, False, RAGGED),
    ("equal", "f32", 4, 4, 64, 16, 0, False, RAGGED),
    ("equal", "bf16", 8, 4, 64, 16, 0, True, RAGGED),
    ("equal", "bf16", 4, 4, 128, 7, 0, False, RAGGED),
    ("equal", "f32", 8, 8, 128, 1, 0, True, [5, 700, 1301, 0, 33, 2049] * 6),
    ("equal", "bf16", 20, 1, 64, 32, 0, False, [17000]),
    ("equal", "bf16", 8, 4, 128, 16, 2500, False, RAGGED),
    ("equal", "f32", 8, 8, 64, 5, 4097, True, [19999]),
    ("own", "bf16", 8, 4, 128, 16, 4097, False, [9000, 5000, 700, 3, 0]),
    ("own", "f32", 8, 8, 128, 16, 0, False, [3000, 2999, 640, 0]),
    ("own", "f32", 4, 4, 64, 16, 2600, False, [6000, 5000, 2700, 40]),
    ("own", "bf16", 8, 4, 64, 16, 0, True, [4100, 0, 3001, 555]),
    ("own", "f32", 8, 4, 64, 48, 0, True, [4100, 0, 3001, 555]),
    ("own", "bf16", 8, 4, 128, 5, 0, False, [3999, 17, 2500]),
    ("own", "f32", 4, 4, 128, 7, 0, True, [3999, 17, 2500]),
    ("own", "bf16", 6, 2, 64, 9, 4500, True, [9001, 8000, 5000]),
    ("own", "bf16", 40, 2, 64, 16, 0, False, [3999, 0, 2500]),
]


@pytest.mark.parametrize("how,dtype,hq,hkv,d,pr,window,masked,lens", DEALT)
def test_paged_attention_as_rows_are_dealt(how, dtype, hq, hkv, d, pr, window, masked, lens):
    import paper_2608_08794_amd as A
    longest = max(lens)
    got, share = _dealt(hq, hkv, d, lens, longest, window)
    assert got == how and share > 1
    g = _gen(91)
    kp, vp, table, n = _paged(g, dtype, lens, hkv, pr, d)
    mask = None
    if masked:
        mask = torch.rand(len(lens), longest + 3, generator=g, device="cuda")[:, :longest] < 0.5
        mask[0, :min(lens[0], longest) // 2] = False      # whole tiles and parts without a row
    q = _rand(g, dtype, hq, len(lens), d)
    args = dict(mask=mask, window=window)
    o, lse = A.apack_paged_attention(q, kp, vp, table, n, longest, return_lse=True, **args)
    _check_attention(o, lse, q, kp, vp, table, n, longest, dtype=dtype, **args)
    again, lse2 = A.apack_paged_attention(q, kp, vp, table, n, longest, return_lse=True, **args)
    np.testing.assert_array_equal(bits(again), bits(o))
    np.testing.assert_array_equal(bits(lse2), bits(lse))


def test_paged_attention_shares_hold_several_items():
    """The equal shares above: some hold parts of three items or more, some begin or end inside one."""
    items, tiles = 4, [max(1, -(-x // 32)) for x in RAGGED]
    ends = np.cumsum([t for t in tiles for _ in range(items)])
    starts = np.array([w * int(ends[-1]) // 512 for w in range(513)])
    first, last = (np.searchsorted(ends, x, side="right") for x in (starts[:-1], starts[1:] - 1))
    assert (last - first >= 2).any() and (last == first).any() and (last - first == 1).any()
    assert not np.isin(starts[1:-1], ends).all()

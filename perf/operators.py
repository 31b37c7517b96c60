"""Rotary positions, a cache of pages and the decode step over it: the cases they are timed on.

What follows a prune in a decoder: queries and keys are turned by their position ids, kept rows move into pages, pages
are copied when a sequence is forked, and each new token is turned, appended to its sequence's pages and attends to
them.  Shapes are those of the library's other workloads: the 3B thinker's heads (16 query / 2 key), the 7B thinker's
(28 / 4, 28 layers), head dim 128, three rows of position ids, clips of 30 s to 5 minutes, and the small fp32 context
(8 / 2 heads, head dim 64).

`own` chooses between the plain form in torch operations and the library's entry points.
"""

import math

import torch

own = False

SECTIONS = {128: (16, 24, 24), 64: (8, 12, 12)}   # frequencies turned by each of three position rows, by rotated width


# ---------------------------------------------------------------------------
# The cases
# ---------------------------------------------------------------------------

def _rotary(name, dtype, hq, hkv, d, rows, rot, layout, pos_rows, transpose, projected, scaling, first):
    return dict(name=name, kind="rotary", dtype=dtype, hq=hq, hkv=hkv, d=d, rows=rows, rot=rot, layout=layout,
                pos_rows=pos_rows, transpose=transpose, projected=projected, scaling=scaling, first=first)


def _append(name, dtype, hq, hkv, d, seqs, page_rows, longest, pos_rows):
    return dict(name=name, kind="append", dtype=dtype, hq=hq, hkv=hkv, d=d, seqs=seqs, page_rows=page_rows,
                longest=longest, pos_rows=pos_rows)


def _copy(name, dtype, hkv, d, layers, page_rows, pages, pairs):
    return dict(name=name, kind="copy", dtype=dtype, hkv=hkv, d=d, layers=layers, page_rows=page_rows, pages=pages,
                pairs=pairs)


def _compact(name, dtype, hkv, d, layers, rows, keep, page_rows, paged_in, paged_out):
    return dict(name=name, kind="compact", dtype=dtype, hkv=hkv, d=d, layers=layers, rows=rows, keep=keep,
                page_rows=page_rows, paged_in=paged_in, paged_out=paged_out)


def _attend(name, dtype, hq, hkv, d, seqs, shortest, longest, page_rows, masked, window):
    return dict(name=name, kind="attend", dtype=dtype, hq=hq, hkv=hkv, d=d, seqs=seqs, shortest=shortest,
                longest=longest, page_rows=page_rows, masked=masked, window=window)


def listed():
    return [
        # The 64 text-query rows that a prune scores with, at the 7B shape: the call's latency.
        _rotary("rotary_query_7b", "bf16", 28, 4, 128, 64, 128, "half", 3, False, True, "none", 9390),
        # Prefill of a 5-minute clip at the 7B shape: projections [rows][heads][d] to the head-major planes of the cache.
        _rotary("rotary_prefill_7b", "bf16", 28, 4, 128, 94028, 128, "half", 3, False, True, "by_parts", 0),
        # Full precision, interleaved pairs in half of the head, the other way round (the gradient).
        _rotary("rotary_gradient_f32", "f32", 16, 2, 128, 9454, 64, "interleaved", 1, True, False, "none", 0),
        # One sequence's new token.
        _append("append_7b_1", "bf16", 28, 4, 128, 1, 16, 9454, 3),
        # The new tokens of a large batch.
        _append("append_7b_256", "bf16", 28, 4, 128, 256, 16, 1024, 3),
        # A sequence forked into eight: each child's copy of the last, partial page.
        _copy("fork_7b_8", "bf16", 4, 128, 28, 16, 600, 8),
        # A whole prompt's pages copied (60 s clip after the pre-LLM stage).
        _copy("copy_7b_prompt", "bf16", 4, 128, 28, 16, 1200, 591),
        # The kept rows of one 30 s clip, one layer, contiguous planes to pages.
        _compact("compact_3b_30s", "bf16", 2, 128, 1, "9454", 0.42, 16, False, True),
        # The kept rows of a 5-minute clip, all layers, from pages to pages.
        _compact("compact_7b_5min", "bf16", 4, 128, 28, "94028", 0.5, 16, True, True),
        # Decoding in a small fp32 context.
        _attend("attend_tiny_f32", "f32", 8, 2, 64, 4, 1, 1312, 16, False, 0),
        # A ragged batch of pruned 30 s to 60 s clips, decoding.
        _attend("attend_7b_64", "bf16", 28, 4, 128, 64, 700, 9454, 16, False, 0),
        # One token over a full 5-minute clip.
        _attend("attend_7b_5min", "bf16", 28, 4, 128, 1, 94028, 94028, 16, False, 0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotary", "rotary", "append", "copy", "compact", "compact", "attend", "attend", "attend"])
    hq, hkv = rng.choice([(28, 4), (16, 2), (8, 2), (8, 8), (32, 1)])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    d = rng.choice([128, 128, 64])
    page_rows = rng.choice([16, 16, 32, 64, 48, 1])
    if kind == "rotary":
        rot = rng.choice([d, d, d // 2, 36])
        case = _rotary("", dtype, hq, hkv, d, _log(rng, 1, 94028 if dtype == "bf16" else 40000), rot,
                       rng.choice(["half", "half", "interleaved"]), 3 if rot in SECTIONS and rng.random() < 0.6 else 1,
                       rng.random() < 0.3, rng.random() < 0.5, rng.choice(["none", "linear", "ntk", "by_parts"]),
                       rng.choice([0, 0, 5000, 1000003]))
    elif kind == "append":
        case = _append("", dtype, hq, hkv, d, _log(rng, 1, 256), page_rows, _log(rng, 20, 1200),
                       rng.choice([1, 3]))
    elif kind == "copy":
        pairs = _log(rng, 1, 500)
        case = _copy("", dtype, hkv if hkv < 8 else 4, d, rng.choice([1, 28, 36]), rng.choice([16, 16, 8, 32]),
                     2 * pairs + rng.randint(1, 60), pairs)
    elif kind == "compact":
        layers = rng.choice([1, 1, 28])
        rows = [_log(rng, 1, 90000 // (4 if layers > 1 else 1)) for _ in range(rng.choice([1, 1, 3, 8]))]
        rows = rows if sum(rows) <= 90000 else rows[:1]
        paged = rng.choice([(True, True), (True, True), (False, True), (True, False)])
        case = _compact("", dtype, hkv if hkv < 8 else 4, d, layers, ",".join(str(x) for x in rows),
                        round(rng.uniform(0.2, 1.0), 2), page_rows, paged[0], paged[1])
    else:
        seqs = _log(rng, 1, 128)
        longest = _log(rng, 1, min(94028, 500000 // seqs) // (1 if hkv < 8 else 2))
        case = _attend("", dtype, hq, hkv, d, seqs, 0 if rng.random() < 0.3 else max(1, longest // 8), longest,
                       page_rows, rng.random() < 0.3, rng.choice([0, 0, 0, 1, 100, 4097]))
    del case["name"]
    return case


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _dt(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _normal(g, c, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=_dt(c))


def _pool(g, c, layers, pages):
    """K and V pages of every layer: [layers][2][pages][heads][rows of a page][d]; K and V of them."""
    kv = _normal(g, c, layers, 2, pages, c["hkv"], c["page_rows"], c["d"])
    return kv, kv[:, 0], kv[:, 1]


def _planes(g, c, layers, rows):
    kv = _normal(g, c, layers, 2, c["hkv"], rows, c["d"])
    return kv, kv[:, 0], kv[:, 1]


def _table(pages, counts):
    """A page table of sequences with so many pages each, from a shuffled list of page ids; -1 where there is none."""
    n = torch.tensor(counts, device="cuda")
    at = torch.arange(max(counts), device="cuda")[None]
    t = pages[((n.cumsum(0) - n)[:, None] + at).clamp(max=pages.numel() - 1)]
    return torch.where(at < n[:, None], t, -1).int().contiguous()


def _positions(g, rows, pos_rows, first):
    t = torch.arange(first, first + rows, dtype=torch.int32, device="cuda")
    h = torch.randint(0, 64, (pos_rows - 1, rows), generator=g, device="cuda", dtype=torch.int32)
    return torch.cat([t[None], t[None] // 2 + h])


def _lens(g, seqs, shortest, longest):
    """Lengths of a ragged batch; one of them is the longest."""
    n = torch.randint(shortest, longest + 1, (seqs,), generator=g, device="cuda", dtype=torch.int32)
    n[seqs // 2] = longest
    return n


def prepare(case, seed):
    c, g = case, _gen(seed)
    s = dict(case=c)
    if c["kind"] in ("rotary", "append"):
        # Which row of the position ids turns each frequency.
        n = c["rot"] if c["kind"] == "rotary" else c["d"]
        sections = SECTIONS[n] if c["pos_rows"] == 3 else (n // 2,)
        s["which"] = torch.arange(len(sections), device="cuda").repeat_interleave(torch.tensor(sections, device="cuda"))
    if c["kind"] == "rotary":
        s["pos"] = _positions(g, c["rows"], c["pos_rows"], c["first"])
        for name, h in (("q", c["hq"]), ("k", c["hkv"])):
            shape = (c["rows"], h, c["d"]) if c["projected"] else (h, c["rows"], c["d"])
            x = _normal(g, c, *shape)
            s[name] = x.transpose(0, 1) if c["projected"] else x
        return s
    pr = c["page_rows"] if "page_rows" in c else 0
    if c["kind"] == "append":
        n = c["seqs"]
        s["lens"] = _lens(g, n, 1, c["longest"])
        per = -(-c["longest"] // pr)
        s["table"] = _table(torch.randperm(n * per, generator=g, device="cuda"), [per] * n)
        s["kv"], k, v = _pool(g, c, 1, n * per)
        s["k_pages"], s["v_pages"] = k[0], v[0]
        s["pos"] = _positions(g, n, c["pos_rows"], c["longest"])
        s["q"], s["k"], s["v"] = (_normal(g, c, n, h, c["d"]).transpose(0, 1) for h in (c["hq"], c["hkv"], c["hkv"]))
    elif c["kind"] == "copy":
        s["kv"], s["k_pages"], s["v_pages"] = _pool(g, c, c["layers"], c["pages"])
        s["pairs"] = torch.randperm(c["pages"], generator=g, device="cuda")[:2 * c["pairs"]].view(-1, 2).int()
    elif c["kind"] == "compact":
        rows = [int(x) for x in c["rows"].split(",")]
        out = [max(1, int(c["keep"] * x)) for x in rows]
        off = [sum(rows[:i]) for i in range(len(rows))]
        s["kept"] = torch.cat([torch.randperm(n, generator=g, device="cuda")[:m].sort().values + o
                               for n, m, o in zip(rows, out, off)]).int()
        # What a decoder knows of each sequence: its first row and rows, the first row and rows it moves to.
        s["seqs"] = [(o, n, 0 if c["paged_out"] else sum(out[:i]), m)
                     for i, (o, n, m) in enumerate(zip(off, rows, out))]
        for side, paged, sizes in (("in", c["paged_in"], rows), ("out", c["paged_out"], out)):
            counts = [-(-x // pr) for x in sizes]
            if paged:
                s["table_" + side] = _table(torch.randperm(sum(counts), generator=g, device="cuda"), counts)
                s["kv_" + side], s["k_" + side], s["v_" + side] = _pool(g, c, c["layers"], sum(counts))
            else:
                s["table_" + side] = None
                s["kv_" + side], s["k_" + side], s["v_" + side] = _planes(g, c, c["layers"], sum(sizes))
        # Sequence of each kept row, and its first kept row, as indices.
        s["of"] = torch.arange(len(rows), device="cuda").repeat_interleave(torch.tensor(out, device="cuda"))
        s["first_in"] = torch.tensor(off, device="cuda")
        s["first_out"] = torch.tensor([sum(out[:i]) for i in range(len(out))], device="cuda")
    else:
        n, longest = c["seqs"], c["longest"]
        s["lens"] = _lens(g, n, c["shortest"], longest)
        counts = [-(-x // pr) for x in s["lens"].tolist()]
        # A pool with some pages more than are in use; short rows of the table end in -1.
        s["table"] = _table(torch.randperm(sum(counts) + 3, generator=g, device="cuda"), counts)
        _, k, v = _pool(g, c, 1, sum(counts) + 3)
        s["k_pages"], s["v_pages"] = k[0], v[0]
        s["q"] = _normal(g, c, n, c["hq"], c["d"]).transpose(0, 1)
        s["mask"] = (torch.rand(n, longest, generator=g, device="cuda") < 0.6).to(torch.uint8) if c["masked"] else None
    return s


# ---------------------------------------------------------------------------
# The plain form
# ---------------------------------------------------------------------------

BASE, FACTOR, TRAINED = 1e6, 4.0, 32768   # base of the frequencies; the factor and length that scaled ones use


def _frequencies(rot, scaling):
    """([rot / 2] radians a position in 64 bits, factor on the turned elements)."""
    i = torch.arange(rot // 2, device="cuda", dtype=torch.float64)
    base = BASE * FACTOR ** (rot / (rot - 2)) if scaling == "ntk" else BASE
    f = torch.exp(i * (-2.0 * math.log(base) / rot))
    if scaling == "linear":
        return f / FACTOR, 1.0
    if scaling == "by_parts":
        turns = TRAINED * f / (2 * math.pi)
        g = ((turns - 1) / 31).clamp(0, 1)
        return (1 - g) * f / FACTOR + g * f, 0.1 * math.log(FACTOR) + 1
    return f, 1.0


def _angles(s, rot, scaling):
    """Angles [rows][rot / 2] of the position ids, in 64 bits: far positions times a frequency lose what matters in 32."""
    f, factor = _frequencies(rot, scaling)
    return s["pos"].double()[s["which"]].t() * f, factor


def _turn(x, theta, factor, layout, transpose):
    """x [heads][rows][d] turned by theta [rows][rot / 2], in theta's type."""
    rot = 2 * theta.shape[1]
    cos, sin = factor * theta.cos(), (-factor if transpose else factor) * theta.sin()
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    y = x.to(theta.dtype)
    y = y.clone() if y.data_ptr() == x.data_ptr() else y
    xa, xb = y[..., a], y[..., b]
    ya, yb = xa * cos - xb * sin, xa * sin + xb * cos
    y[..., a], y[..., b] = ya, yb
    return y


def _turn32(x, s, rot, layout="half", transpose=False, scaling="none"):
    """The same with the angles reduced to one turn in 64 bits and the rest in 32, rounded once at the end."""
    theta, factor = _angles(s, rot, scaling)
    theta = torch.remainder(theta, 2 * math.pi).float()
    return _turn(x, theta, factor, layout, transpose).to(x.dtype).contiguous()


def _rows_of(pool, table, pr):
    """Pages [pages][heads][rows][d] of a table [seqs][pages], as rows [seqs][heads][pages * rows][d]; a page that is not
    there as page 0."""
    x = pool[table.long().clamp(min=0)]
    return x.permute(0, 2, 1, 3, 4).reshape(table.shape[0], pool.shape[1], -1, pool.shape[3])


def _seen(s, c):
    """Which rows [seqs][rows] each sequence attends to."""
    lens = s["lens"][:, None]
    at = torch.arange(s["table"].shape[1] * c["page_rows"], device="cuda")[None]
    seen = at < lens
    if c["window"]:
        seen = seen & (at >= lens - c["window"])
    if s["mask"] is not None:
        seen = seen & torch.nn.functional.pad(s["mask"] != 0, (0, at.shape[1] - s["mask"].shape[1]))
    return seen


def _attend_plain(s, c, dtype):
    pr, hkv, d = c["page_rows"], c["hkv"], c["d"]
    k = _rows_of(s["k_pages"], s["table"], pr).to(dtype)
    q = s["q"].to(dtype).view(hkv, -1, c["seqs"], d).permute(2, 0, 3, 1).contiguous()      # [seqs][hkv][d][group]
    x = torch.matmul(k, q).transpose(2, 3) / math.sqrt(d)                                # [seqs][hkv][group][rows]
    del k
    x = x.masked_fill(~_seen(s, c)[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, 0, top))
    total = p.sum(-1, keepdim=True)
    v = _rows_of(s["v_pages"], s["table"], pr).to(dtype)
    o = torch.matmul(p.contiguous(), v) / torch.where(total == 0, 1, total)
    lse = torch.log(total) + top
    o = o.reshape(c["seqs"], c["hq"], d).transpose(0, 1)
    return o, lse.reshape(c["seqs"], c["hq"]).t()


def _places(s, c, side, local, packed):
    """(page, row in it) of rows of a side that has pages, or (None, packed row)."""
    if s["table_" + side] is None:
        return None, packed
    return s["table_" + side].long()[s["of"], local // c["page_rows"]], local % c["page_rows"]


def _plain(s, c):
    if c["kind"] == "rotary":
        how = dict(rot=c["rot"], layout=c["layout"], transpose=c["transpose"], scaling=c["scaling"])
        return dict(q=_turn32(s["q"], s, **how), k=_turn32(s["k"], s, **how))
    if c["kind"] == "append":
        at = s["lens"].long() - 1
        pr = c["page_rows"]
        page = s["table"].long().gather(1, (at // pr)[:, None])[:, 0]
        s["k_pages"][page, :, at % pr] = _turn32(s["k"], s, c["d"]).transpose(0, 1)
        s["v_pages"][page, :, at % pr] = s["v"].transpose(0, 1)
        return dict(q=_turn32(s["q"], s, c["d"]), kv=s["kv"])
    if c["kind"] == "copy":
        src, dst = s["pairs"].long().unbind(1)
        s["kv"][:, :, dst] = s["kv"][:, :, src]
        return dict(kv=s["kv"])
    if c["kind"] == "compact":
        kept = s["kept"].long()
        i = torch.arange(kept.numel(), device="cuda")
        page, row = _places(s, c, "in", kept - s["first_in"][s["of"]], kept)
        x = s["kv_in"][:, :, :, row].permute(3, 0, 1, 2, 4) if page is None else s["kv_in"][:, :, page, :, row]
        page, row = _places(s, c, "out", i - s["first_out"][s["of"]], i)
        if page is None:
            s["kv_out"][:, :, :, row] = x.permute(1, 2, 3, 0, 4)
        else:
            s["kv_out"][:, :, page, :, row] = x
        return dict(kv=s["kv_out"])
    o, lse = _attend_plain(s, c, torch.float32)
    return dict(o=o.to(s["q"].dtype).contiguous(), lse=lse.contiguous())


# ---------------------------------------------------------------------------
# The library's entry points
# ---------------------------------------------------------------------------

def _own(s, c):
    import paper_2608_08794_amd as A

    if c["kind"] == "rotary":
        rope = A.apack_rope(c["rot"], base=BASE, layout=c["layout"], scaling=c["scaling"], factor=FACTOR,
                            trained_len=TRAINED, sections=SECTIONS[c["rot"]] if c["pos_rows"] == 3 else None)
        q, k = A.apack_rotary(s["pos"], rope, s["q"], s["k"], transpose=c["transpose"])
        return dict(q=q, k=k)
    if c["kind"] == "append":
        rope = A.apack_rope(c["d"], base=BASE, sections=SECTIONS[c["d"]] if c["pos_rows"] == 3 else None)
        q = A.apack_rotary_append(s["pos"], rope, s["q"], s["k"], s["v"], s["k_pages"], s["v_pages"], s["table"],
                                  s["lens"])
        return dict(q=q, kv=s["kv"])
    if c["kind"] == "copy":
        A.apack_pages_copy(s["pairs"], s["k_pages"], s["v_pages"])
        return dict(kv=s["kv"])
    if c["kind"] == "compact":
        A.apack_compact_kv_pages(s["kept"], s["seqs"], s["k_in"], s["v_in"], s["k_out"], s["v_out"],
                                 table_in=s["table_in"], table_out=s["table_out"])
        return dict(kv=s["kv_out"])
    o, lse = A.apack_paged_attention(s["q"], s["k_pages"], s["v_pages"], s["table"], s["lens"], c["longest"],
                                     mask=s["mask"], window=c["window"], return_lse=True)
    return dict(o=o, lse=lse)


def run(state):
    c = state["case"]
    if own:
        return _own(state, c)
    return _plain(state, c)


# ---------------------------------------------------------------------------
# What a pass cannot do without, and what it should give
# ---------------------------------------------------------------------------

def work(case):
    c = case
    es = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "rotary":
        n = c["rows"] * (c["hq"] + c["hkv"])
        return dict(bytes=2 * n * c["d"] * es + 4 * c["pos_rows"] * c["rows"], flops=3 * n * c["rot"])
    if c["kind"] == "append":
        n = c["seqs"]
        return dict(bytes=2 * n * (c["hq"] + 2 * c["hkv"]) * c["d"] * es + 4 * n * (c["pos_rows"] + 2),
                    flops=3 * n * (c["hq"] + c["hkv"]) * c["d"])
    if c["kind"] == "copy":
        page = c["hkv"] * c["page_rows"] * c["d"] * es
        return dict(bytes=c["pairs"] * (8 + 4 * c["layers"] * page), flops=0)
    if c["kind"] == "compact":
        rows = sum(max(1, int(c["keep"] * int(x))) for x in c["rows"].split(","))
        return dict(bytes=rows * (4 + 4 * c["layers"] * c["hkv"] * c["d"] * es), flops=0)
    # Lengths are drawn evenly between the shortest and the longest, and one is the longest.
    mean = lambda top: (min(c["shortest"], top) + top) / 2  # noqa: E731
    top = min(c["longest"], c["window"] or c["longest"])
    rows = top + (c["seqs"] - 1) * (mean(c["longest"]) if not c["window"] else min(top, mean(c["longest"])))
    rows = rows * (0.6 if c["masked"] else 1.0)
    return dict(bytes=rows * 2 * c["hkv"] * c["d"] * es + 2 * c["seqs"] * c["hq"] * c["d"] * es,
                flops=4 * rows * c["hq"] * c["d"])


def _exact_turn(x, pos, rot, layout, transpose, scaling):
    """Each pair as a complex number, times e^(i theta)."""
    i = torch.arange(rot // 2, device="cuda", dtype=torch.float64)
    base, factor = BASE, 1.0
    if scaling == "ntk":
        base = BASE * FACTOR ** (rot / (rot - 2))
    f = torch.pow(torch.tensor(base, dtype=torch.float64, device="cuda"), -2 * i / rot)
    if scaling == "linear":
        f = f / FACTOR
    if scaling == "by_parts":
        g = torch.clip((TRAINED * f / (2 * math.pi) - 1) / (32 - 1), 0, 1)
        f, factor = f * ((1 - g) / FACTOR + g), 1 + math.log(FACTOR) / 10
    p = pos.double()
    if pos.shape[0] == 3:
        n = SECTIONS[rot]
        theta = torch.cat([p[0, :, None] * f[:n[0]], p[1, :, None] * f[n[0]:n[0] + n[1]], p[2, :, None] * f[-n[2]:]], 1)
    else:
        theta = p[0, :, None] * f
    w = torch.polar(torch.full_like(theta, factor), -theta if transpose else theta)
    y = x.double().contiguous()
    turned = y[..., :rot].unflatten(-1, (rot // 2, 2) if layout == "interleaved" else (2, rot // 2))
    turned = turned if layout == "interleaved" else turned.transpose(-1, -2).contiguous()
    z = torch.view_as_real(torch.view_as_complex(turned) * w)
    z = z if layout == "interleaved" else z.transpose(-1, -2)
    return torch.cat([z.flatten(-2), y[..., rot:]], -1)


def exact(case, seed):
    c = case
    if c["kind"] in ("copy", "compact"):
        return None                                     # moved, not computed
    s = prepare(case, seed)
    if c["kind"] == "rotary":
        return {x: _exact_turn(s[x], s["pos"], c["rot"], c["layout"], c["transpose"], c["scaling"]) for x in ("q", "k")}
    if c["kind"] == "append":
        kv = s["kv"].double()
        k = _exact_turn(s["k"], s["pos"], c["d"], "half", False, "none")
        for i, n in enumerate(s["lens"].tolist()):
            page, row = int(s["table"][i, (n - 1) // c["page_rows"]]), (n - 1) % c["page_rows"]
            kv[0, 0, page, :, row], kv[0, 1, page, :, row] = k[:, i], s["v"][:, i].double()
        return dict(q=_exact_turn(s["q"], s["pos"], c["d"], "half", False, "none"), kv=kv)
    o = torch.zeros(c["hq"], c["seqs"], c["d"], dtype=torch.float64, device="cuda")
    lse = torch.full((c["hq"], c["seqs"]), -math.inf, dtype=torch.float64, device="cuda")
    for i, n in enumerate(s["lens"].tolist()):
        at = torch.arange(max(0, n - c["window"]) if c["window"] else 0, n, device="cuda")
        at = at if s["mask"] is None else at[s["mask"][i, at] != 0]
        if not at.numel():
            continue
        page, row = s["table"][i].long()[at // c["page_rows"]], at % c["page_rows"]
        k, v = (x[page, :, row].double().repeat_interleave(c["hq"] // c["hkv"], 1) for x in (s["k_pages"], s["v_pages"]))
        x = (k * s["q"][:, i].double()[None]).sum(-1) / c["d"] ** 0.5
        lse[:, i] = torch.logsumexp(x, 0)
        o[:, i] = (torch.softmax(x, 0)[..., None] * v).sum(0)
    return dict(o=o, lse=lse)

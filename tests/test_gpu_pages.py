"""Paged caches: page_bounds, select_pages and attend_pages against 64-bit definitions (GB300).

Boxes and choices are whole numbers and powers of two: they have to be equal.

Tolerances of the attention (before any run):
  fp32 queries  as for the attention over contiguous records: scores are fp32 sums far
      within 2^-12 scale ||q|| max ||k^||, a score error e moves the softmax weights by at most
      2e, so |out - ref| <= (2^-11 scale ||q|| max ||k^|| + 2^-16) max |v^|.
  bf16 queries  decoded values may be fp16 numbers times a factor of the record (the bin
      centre, the norm and their product rounded, the norm's exponential good to 2^-9.9): a key
      within 2^-9 of its length, so a score within 2^-9 scale ||q|| ||k^||, the weights within twice
      that; a value and its weight, likewise, within 2^-8 of its length; and the output's
      rounding: |out - ref| <= (2^-8 scale ||q|| max ||k^|| + 2^-16) max |v^| + 2^-8 max ||v^|| + ulp/2.
A wrong page, bin, norm, sign or weight gives errors of the order of max |v^|.
"""
import math

import numpy as np
import pytest

import pages_ref as ref
import parity
import workloads

pytestmark = pytest.mark.gpu


def _dtype(name):
    import torch
    return torch.bfloat16 if name == "bf16" else torch.float32


def _gen(seed):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _table(lens, page, spare, seed, width=None):
    """(table with pages in random order, pages of the pool)."""
    import torch
    per = [-(-n // page) for n in lens]
    width = max([1] + per) if width is None else width
    pages = sum(per) + spare
    order = np.random.default_rng(seed).permutation(pages)
    t = np.full((len(lens), width), -1, dtype=np.int32)
    at = 0
    for s, n in enumerate(per):
        t[s, :n] = order[at: at + n]
        at += n
    return torch.from_numpy(t).cuda(), pages


# ---------------------------------------------------------------------------
# boxes
# ---------------------------------------------------------------------------
def _check_bounds(tac, keys, bounds, table, start, first, page):
    import torch
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    want = ref.bounds(bounds.codes.cpu().numpy(), bounds.scales.cpu().numpy(), parity.to_f64(keys), table.cpu().numpy(),
                      start, first if first is not None else range(len(start) + 1), page)
    tac.page_bounds(bounds, keys, table, i32(start), None if first is None else i32(first))
    torch.cuda.synchronize()
    assert np.array_equal(bounds.codes.cpu().numpy().astype(np.int64), want[0])
    assert np.array_equal(bounds.scales.cpu().numpy().astype(np.float64), want[1])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page,heads", [(16, 3), (48, 8), (64, 1), (256, 2)])
def test_bounds_prompts_and_steps(tac_gpu, dtype, d, page, heads):
    """Prompts of odd lengths, a second chunk that starts inside a page, then single tokens."""
    import torch
    tac = tac_gpu
    lens = [1, page - 1, page, page + 1, 3 * page + 7, 0, 517]
    table, pages = _table([n + 2 * page for n in lens], page, 2, 5)
    g = _gen(d + page)
    bounds = tac.PageBounds.empty(pages, heads, d, page)
    bounds.codes.fill_(99)                       # what reused pages held
    bounds.scales.fill_(4.0)
    sigma = torch.exp(2 * torch.randn((heads, d), generator=g, device="cuda"))

    def keys(n):
        return (torch.randn((n, heads, d), generator=g, device="cuda") * sigma).to(_dtype(dtype))

    first = np.concatenate([[0], np.cumsum(lens)])
    _check_bounds(tac, keys(int(first[-1])), bounds, table, [0] * len(lens), first, page)
    more = [page // 2, 0, 3, 1, page, 5, 2 * page - 1]
    first = np.concatenate([[0], np.cumsum(more)])
    _check_bounds(tac, keys(int(first[-1])) * 8, bounds, table, lens, first, page)
    now = [a + b for a, b in zip(lens, more)]
    for step in range(2):
        _check_bounds(tac, keys(len(lens)) * 4.0**step, bounds, table, [n + step for n in now], None, page)


def test_bounds_hold_the_keys_and_do_not_depend_on_how_they_come(tac_gpu):
    """A prompt at once, in chunks, and token by token: the same boxes, which hold every key."""
    import torch
    tac = tac_gpu
    page, heads, d, n = 32, 2, 128, 101
    table, pages = _table([n], page, 0, 1)
    x = (torch.randn((n, heads, d), generator=_gen(3), device="cuda") * 3).to(torch.bfloat16)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    got = []
    for cuts in ([0, n], [0, 1, 40, 64, n], list(range(n + 1))):
        b = tac.PageBounds.empty(pages, heads, d, page)
        for a, e in zip(cuts, cuts[1:]):
            tac.page_bounds(b, x[a:e], table, i32([a]), i32([0, e - a]))
        got.append(b)
    for b in got[1:]:
        # scales only grow by the largest key: equal; codes rounded outward step by step may be wider by the steps
        assert torch.equal(b.scales, got[0].scales)
    for b in got:
        box = b.codes.double() * b.scales.double()[..., None, None]
        for t in range(n):
            p = int(table[0, t // page])
            assert bool((box[p, :, 0] <= x[t].double()).all()) and bool((x[t].double() <= box[p, :, 1]).all())


def test_bounds_nonfinite_zero_and_extreme_keys(tac_gpu):
    import torch
    tac = tac_gpu
    page, heads, d = 16, 2, 64
    lens = [40, 40, 40]
    table, pages = _table([64] * 3, page, 1, 2)
    for dtype in ("bf16", "fp32"):
        bounds = tac.PageBounds.empty(pages, heads, d, page)
        x = torch.randn((120, heads, d), generator=_gen(9), device="cuda").to(_dtype(dtype))
        x[3, 0, 5], x[50, 1, 0], x[90, 0, 63] = math.nan, math.inf, -math.inf
        x[16:32] = 0
        x[56:60, 0] = 3e38
        x[60:64, 0] = -3e38
        x[104:120, 1] = 1e-40
        x[110, 1, 7] = -2e-39
        first = [0, 40, 80, 120]
        _check_bounds(tac, x, bounds, table, [0, 0, 0], first, page)
        assert bool(torch.isinf(bounds.scales).any()) and bool((bounds.scales == 2.0**-126).any())
        # on: an unbounded page stays so until it starts afresh
        y = torch.randn((3, heads, d), generator=_gen(10), device="cuda").to(_dtype(dtype))
        _check_bounds(tac, y, bounds, table, lens, None, page)
        _check_bounds(tac, x[16:64], bounds, table, [0, 0, 0], [0, 16, 32, 48], page)


def test_bounds_outward_where_products_underflow(tac_gpu):
    """A key of -1e-30 beside one of 1e30: its bound is one step below zero, not zero."""
    import torch
    tac = tac_gpu
    table = torch.zeros((1, 1), dtype=torch.int32, device="cuda")
    x = torch.zeros((2, 1, 64), device="cuda")
    x[0, 0, 0], x[0, 0, 1], x[1, 0, 2] = -1e-30, 1e-30, 1e30
    b = tac.PageBounds.empty(1, 1, 64, 16)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    tac.page_bounds(b, x[:1], table, i32([0]))
    tac.page_bounds(b, x[1:], table, i32([1]))
    c = b.codes[0, 0].cpu()
    assert c[0, 0] == -1 and c[1, 0] == 0 and c[0, 1] == 0 and c[1, 1] == 1 and c[1, 2] > 60
    tac.page_bounds(b, x, table, i32([0]), i32([0, 2]))
    c = b.codes[0, 0].cpu()
    assert c[0, 0] == -1 and c[1, 1] == 1


def test_bounds_rows_outside_are_left_out(tac_gpu):
    """Negative positions, positions beyond the table, no page, row ranges beyond k, strided k."""
    import torch
    tac = tac_gpu
    page, heads, d = 16, 2, 64
    table = torch.tensor([[0, 1], [-1, 2], [9, 3], [4, 1000000]], dtype=torch.int32, device="cuda")
    bounds = tac.PageBounds.empty(5, heads, d, page)
    big = torch.randn((90, heads + 1, 2 * d), generator=_gen(4), device="cuda").to(torch.bfloat16)
    x = big[:80, :heads, :d]
    _check_bounds(tac, x, bounds, table, [-5, 8, 10, 3], [0, 20, 40, 62, 200], page)
    _check_bounds(tac, x, bounds, table, [31, 32, 40, -3], [5, 10, 20, 30, 34], page)
    _check_bounds(tac, x[:4], bounds, table, [-1, 16, 3, 31], None, page)


# ---------------------------------------------------------------------------
# choice of pages
# ---------------------------------------------------------------------------
def _boxes(tac, pages, heads, d, page, seed, levels=127, exps=4):
    import torch
    g = _gen(seed)
    a = torch.randint(-levels, levels + 1, (2, pages, heads, d), generator=g, device="cuda")
    codes = torch.stack([torch.minimum(a[0], a[1]), torch.maximum(a[0], a[1])], dim=2).to(torch.int8).contiguous()
    scales = torch.exp2(torch.randint(-exps, exps + 1, (pages, heads), generator=g, device="cuda").float())
    return tac.PageBounds(codes, scales, page)


def _check_select(tac, q, bounds, table, lens, budget, kf=1, kl=1):
    import torch
    lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
    sel, cnt = tac.select_pages(q, bounds, table, lengths, budget, kf, kl)
    torch.cuda.synchronize()
    want, counts = ref.select(parity.to_f64(q), bounds.codes.cpu().numpy(), bounds.scales.cpu().numpy().astype(np.float64),
                              table.cpu().numpy(), lens, bounds.page_tokens, budget, kf, kl)
    assert np.array_equal(cnt.cpu().numpy(), counts)
    assert np.array_equal(sel.cpu().numpy(), want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,heads,group", [(64, 1, 1), (64, 3, 5), (128, 2, 3), (128, 2, 4), (128, 1, 8), (64, 2, 8)])
def test_select_small(tac_gpu, dtype, d, heads, group):
    """Lengths around the page and the budget, every keep; ragged, empty and negative lengths."""
    import torch
    tac = tac_gpu
    page = 16
    lens = [0, 1, 15, 16, 17, 7 * 16, 8 * 16, 8 * 16 + 1, 33 * 16 + 5, 1000, -4, 10**6]
    table, pages = _table([max(0, min(n, 1600)) for n in lens], page, 4, d + group, width=100)
    bounds = _boxes(tac, pages, heads, d, page, 11 * d + group)
    q = torch.randn((len(lens), heads * group, d), generator=_gen(group), device="cuda").to(_dtype(dtype))
    for budget, kf, kl in ((1, 0, 0), (1, 1, 0), (8, 0, 0), (8, 1, 1), (8, 3, 5), (33, 0, 4), (128, 2, 2)):
        _check_select(tac, q, bounds, table, lens, budget, kf, kl)


@pytest.mark.parametrize("n", [700, 2049, 9001])
def test_select_long_tables_and_ties(tac_gpu, n):
    """Tables that several CTAs share; few distinct scores, so that ties decide."""
    import torch
    tac = tac_gpu
    page, heads, d, group = 16, 2, 64, 4
    lens = [n * page, (n - 3) * page - 5]
    table, pages = _table(lens, page, 0, n)
    g = _gen(n)
    for levels, exps in ((127, 3), (1, 0), (0, 0)):
        bounds = _boxes(tac, pages, heads, d, page, n + levels, levels, exps)
        q = torch.randn((2, heads * group, d), generator=g, device="cuda")
        if levels == 1:                          # whole scores in a small range
            q = torch.zeros_like(q)
            q[..., :3] = 1.0
        for budget in (2, 64, n // 2, n - 4):
            _check_select(tac, q, bounds, table, lens, budget)


def test_select_special_values(tac_gpu):
    """NaN and inf queries, pages without a bound, no page, zero queries, extreme scales."""
    import torch
    tac = tac_gpu
    page, heads, d, group, n = 16, 2, 128, 4, 90
    lens = [n * page] * 6
    table, pages = _table(lens, page, 0, 3)
    bounds = _boxes(tac, pages, heads, d, page, 77)
    bounds.scales[::7] = math.inf
    bounds.scales[3::11] = 2.0**110
    bounds.scales[5::13] = 2.0**-126
    table[0, 10:20] = -1
    table[1, 5] = pages
    table[1, 0] = -7
    q = torch.randn((6, heads * group, d), generator=_gen(1), device="cuda")
    q[1, 2, 5], q[1, 3], q[2, 0, 1], q[2, 1, 2] = math.nan, math.nan, math.inf, -math.inf
    q[3] = 0
    q[4] *= 2.0**100
    q[5] *= 1e-42
    for budget in (3, 20, 80, 89):
        _check_select(tac, q, bounds, table, lens, budget)


def test_select_strides_and_given_outputs(tac_gpu):
    import torch
    tac = tac_gpu
    page, heads, d, group = 32, 2, 64, 2
    lens = [3000, 1777, 64]
    wide, pages = _table(lens, page, 0, 8, width=128)
    table = torch.full((3, 300), -3, dtype=torch.int32, device="cuda")
    table[:, 50:178] = wide
    table = table[:, 50:178]
    bounds = _boxes(tac, pages, heads, d, page, 5)
    big = torch.randn((3, 2 * heads * group, 2 * d), generator=_gen(2), device="cuda").to(torch.bfloat16)
    q = big[:, 1::2, :d]
    _check_select(tac, q, bounds, table, lens, 9)
    sel = torch.full((3, heads, 9), 55, dtype=torch.int32, device="cuda")
    cnt = torch.full((3, heads), 55, dtype=torch.int32, device="cuda")
    lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
    a, b = tac.select_pages(q, bounds, table, lengths, 9, selected=sel, counts=cnt)
    c, e = tac.select_pages(q.contiguous(), bounds, table.contiguous(), lengths, 9)
    assert a is sel and b is cnt and torch.equal(a, c) and torch.equal(b, e)


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
K8, V4 = (8, 0), (4, 1)


def _pools(tac, d, heads, page, lens, seed, kbook, vbook, spare=1, dtype="bf16", width=None):
    """A cache of random rows in random pages; every other slot is filled with ones' bytes: NaN headers, the largest codes."""
    import torch
    table, pages = _table(lens, page, spare, seed, width)
    cfgs = [tac.layer_cfg(d, *book, 0, 3, kv) for kv, book in enumerate((kbook, vbook))]
    cache = tac.PagedCache.empty(cfgs[0], cfgs[1], pages, heads, page)
    for c in (cache.k, cache.v):
        c.codes.fill_(255)
        c.norms.fill_(255)
    seq = torch.tensor(np.repeat(np.arange(len(lens)), lens), device="cuda")
    pos = torch.tensor(np.concatenate([np.arange(n) for n in lens] + [np.zeros(0)]).astype(np.int64), device="cuda")
    w = workloads.CONFIGS["mistral7b" if d == 128 else "llama1b"]
    if len(pos):
        slot = cache.slots(table, pos, seq)
        jobs = []
        for kv, c in enumerate((cache.k, cache.v)):
            n = len(pos) * heads
            x = workloads.block(w, 2, kv, tokens=-(-n // w.heads), seed=seed, device="cuda")[:n].contiguous()
            jobs.append(tac.EncodeJob(c.cfg, x, c, slot))
        tac.encode_multi(jobs)
    return cache, table


def _queries(seqs, rows, d, dtype, seed):
    import torch
    return (0.5 * torch.randn((seqs, rows, d), generator=_gen(seed), device="cuda")).to(_dtype(dtype))


def _check_attend(tac, orc, cache, table, lens, q, selected=None, counts=None, out=None, rows=None):
    import torch
    d, heads = cache.k.cfg.d, cache.kv_heads
    scale = 1.0 / math.sqrt(d)
    lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
    got = tac.attend_pages(q, cache, table, lengths, scale, selected, counts, out=out)
    torch.cuda.synchronize()
    krows, vrows = rows or (ref.pool_rows(orc, cache.k), ref.pool_rows(orc, cache.v))
    q64 = parity.to_f64(q)
    sel = None if selected is None else selected.cpu().numpy()
    cnt = None if counts is None else counts.cpu().numpy()
    want, kmax, vnorm, vel = ref.attend(orc, q64, krows, vrows, table.cpu().numpy(), lens, cache.page_tokens, heads, scale, sel, cnt)
    qn = np.linalg.norm(q64, axis=-1)
    bf = q.dtype == torch.bfloat16
    tol = (2.0**(-8 if bf else -11) * scale * qn * kmax + 2.0**-16) * vel
    tol = np.broadcast_to(tol[..., None], want.shape)
    if bf:
        tol = tol + 2.0**-8 * vnorm[..., None] + parity.bf16_half_ulp(want)
    g64 = parity.to_f64(got)
    assert np.isfinite(g64).all()
    err = np.abs(g64 - want)
    assert np.all(err <= tol), float((err / np.maximum(tol, 1e-300)).max())
    empty = kmax == 0
    assert np.all(g64[empty] == 0)
    return got, want


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,heads,group", [(64, 2, 1), (64, 3, 4), (64, 1, 8), (128, 2, 2), (128, 2, 4), (128, 1, 5), (128, 1, 8)])
def test_attend_ragged(tac_gpu, orc, dtype, d, heads, group):
    """Lengths around tile, batch and page; empty sequences first, between and last."""
    tac = tac_gpu
    lens = [0, 1, 15, 16, 17, 31, 32, 33, 0, 47, 48, 49, 96, 97, 200, 0]
    cache, table = _pools(tac, d, heads, 48, lens, d + group, (64, *K8), (64, *V4))
    q = _queries(len(lens), heads * group, d, dtype, group)
    _check_attend(tac, orc, cache, table, lens, q)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kbook,vbook", [
    ((256, 8, 0), (256, 4, 1)), ((128, 8, 0), (64, 8, 0)), ((56, 32, 2), (48, 32, 2)), ((48, 4, 0), (256, 4, 0)),
    ((2, 8, 1), (4, 8, 1)), ((32, 4, 1), (16, 8, 0)), ((8, 32, 2), (128, 4, 1)), ((256, 32, 2), (256, 32, 2))])
@pytest.mark.parametrize("d", [64, 128])
def test_attend_codebooks(tac_gpu, orc, dtype, kbook, vbook, d):
    """Every norm storage on both sides, code widths 1 to 8, bins that are no power of two."""
    tac = tac_gpu
    lens = [77, 130, 5]
    cache, table = _pools(tac, d, 2, 32, lens, d + kbook[0], kbook, vbook)
    q = _queries(3, 2 * 3, d, dtype, 5)
    _check_attend(tac, orc, cache, table, lens, q)


@pytest.mark.parametrize("page", [16, 32, 80, 256, 1024])
@pytest.mark.parametrize("seqs,heads,length", [(1, 1, 5000), (2, 2, 3001), (1, 8, 700), (9, 1, 333)])
def test_attend_split_over_ctas(tac_gpu, orc, page, seqs, heads, length):
    """One long sequence over many CTAs, and parts that end inside a warp's or a CTA's tiles."""
    tac = tac_gpu
    lens = [length - 7 * s for s in range(seqs)]
    cache, table = _pools(tac, 128, heads, page, lens, page + length, (64, *K8), (64, *V4))
    for dtype in ("bf16", "fp32"):
        _check_attend(tac, orc, cache, table, lens, _queries(seqs, heads * 4, 128, dtype, 1))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("page", [16, 64])
def test_attend_selected(tac_gpu, orc, dtype, page):
    """Selections: short, in any order, with entries that name no column, nothing, or a page twice."""
    import torch
    tac = tac_gpu
    heads, d, group = 2, 128, 4
    lens = [1000, 1, 0, 640, 333]
    cache, table = _pools(tac, d, heads, page, lens, 6, (64, *K8), (64, *V4))
    width = table.shape[1]
    g = np.random.default_rng(3)
    budget = 7
    sel = np.full((5, heads, budget), -1, dtype=np.int32)
    cnt = np.zeros((5, heads), dtype=np.int32)
    for s, n in enumerate(lens):
        cols = -(-n // page)
        for h in range(heads):
            k = min(budget, cols)
            sel[s, h, :k] = g.permutation(cols)[:k]
            cnt[s, h] = k
    sel[0, 0] = [width, -5, 0, 0, 2**31 - 1, (1000 - 1) // page, 1]
    cnt[0, 0] = 100                              # above the budget: clamped
    cnt[3, 1] = -2                               # below zero: no token
    cnt[2] = 3
    sel[2] = 0                                   # a sequence without a token
    q = _queries(5, heads * group, d, dtype, 2)
    _check_attend(tac, orc, cache, table, lens, q, torch.from_numpy(sel).cuda(), torch.from_numpy(cnt).cuda())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attend_missing_pages_and_lengths_outside(tac_gpu, orc, dtype):
    """Table entries that name no page, lengths below zero and beyond the table."""
    tac = tac_gpu
    heads, d, page = 2, 64, 32
    lens = [320, 320, 64, 320]
    cache, table = _pools(tac, d, heads, page, lens, 12, (64, *K8), (64, *V4))
    table[0, 3] = -1
    table[0, 9] = cache.pages
    table[1, ::2] = 2**31 - 1
    table[2] = -2**31
    q = _queries(4, heads * 3, d, dtype, 4)
    _check_attend(tac, orc, cache, table, [320, 299, 64, 10**9], q)
    _check_attend(tac, orc, cache, table, [-1, 31, 0, -2**31], q)


def test_attend_many_short_sequences(tac_gpu, orc):
    """More (sequence, head)s than warps: whole ones inside a warp, several in a row."""
    tac = tac_gpu
    g = np.random.default_rng(0)
    lens = [int(v) for v in g.integers(0, 70, size=700)]
    cache, table = _pools(tac, 64, 8, 16, lens, 1, (64, *K8), (64, *V4))
    rows = ref.pool_rows(orc, cache.k), ref.pool_rows(orc, cache.v)
    for dtype in ("bf16", "fp32"):
        _check_attend(tac, orc, cache, table, lens, _queries(700, 8 * 2, 64, dtype, 3), rows=rows)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attend_strided_and_given_output(tac_gpu, orc, dtype):
    import torch
    tac = tac_gpu
    heads, d, group, lens = 2, 128, 2, [90, 33, 200]
    cache, table = _pools(tac, d, heads, 16, lens, 4, (64, *K8), (64, *V4))
    big = _queries(3, 3 * heads * group, 2 * d, dtype, 8)
    q = big[:, 2::3, d:]
    out = torch.full((3, 2 * heads * group, d), 7.0, dtype=q.dtype, device="cuda")
    got, _ = _check_attend(tac, orc, cache, table, lens, q, out=out[:, ::2])
    assert got.data_ptr() == out.data_ptr() and bool((out[:, 1::2] == 7).all())


@pytest.mark.parametrize("dtype,limit", [("bf16", 1.5), ("fp32", 1.5)])
@pytest.mark.parametrize("d,books", [(128, ((64, *K8), (64, *V4))), (64, ((128, *K8), (64, *V4))), (128, ((64, 8, 0), (64, 8, 0))),
                                     (128, ((128, 32, 2), (64, 32, 2)))])
def test_attend_precision(tac_gpu, orc, dtype, limit, d, books):
    """The error against 64 bits, 2-norm over all rows, is at most 1.5 times that of fp32 arithmetic on
    the decoded rows, rounded once to the queries' type."""
    import torch
    tac = tac_gpu
    lens = [1, 3, 40, 300, 1500, 1500, 1500]
    heads, group = 4, 4
    cache, table = _pools(tac, d, heads, 64, lens, 21, *books)
    q = _queries(len(lens), heads * group, d, dtype, 9)
    got, want = _check_attend(tac, orc, cache, table, lens, q)
    krows, vrows = (torch.from_numpy(ref.pool_rows(orc, c)).float() for c in (cache.k, cache.v))
    plain = torch.zeros(q.shape)
    t = table.cpu().numpy()
    for s in range(len(lens)):
        for h in range(heads):
            tok = ref.tokens_of(s, h, t, lens, 64, cache.pages)
            slot = torch.tensor([(p * heads + h) * 64 + x % 64 for x, p in tok])
            sc = (q[s, h * group: (h + 1) * group].cpu().float() @ krows[slot].T) * (1.0 / math.sqrt(d))
            e = torch.exp(sc - sc.amax(dim=1, keepdim=True))
            plain[s, h * group: (h + 1) * group] = (e @ vrows[slot]) / e.sum(dim=1, keepdim=True)
    plain = parity.to_f64(plain.to(q.dtype))
    err, base = np.linalg.norm(parity.to_f64(got) - want), np.linalg.norm(plain - want)
    assert err <= limit * base, (err, base)


def test_attend_nan_records_and_queries_stay_in_their_rows(tac_gpu):
    """A NaN key makes its own (sequence, head) NaN and no other; a NaN query its own row."""
    import torch
    tac = tac_gpu
    heads, d, group, lens, page = 2, 64, 2, [50, 40], 16
    for dtype in ("bf16", "fp32"):
        cache, table = _pools(tac, d, heads, page, lens, 4, (64, *K8), (64, *V4))
        lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
        q = _queries(2, heads * group, d, dtype, 8)
        q[0, 1, 3] = math.nan
        row = torch.full((1, d), math.nan, device="cuda")
        slot = cache.slots(table, torch.tensor([7], device="cuda"), torch.tensor([1], device="cuda"))[1:2]
        tac.encode_multi([tac.EncodeJob(cache.k.cfg, row, cache.k, slot)])
        out = tac.attend_pages(q, cache, table, lengths, 0.125)
        bad = torch.isnan(out).any(dim=-1).cpu()
        assert bad.tolist() == [[False, True, False, False], [False, False, True, True]]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_calls_on_another_stream_and_captured(tac_gpu, dtype):
    """The three calls of a decode step on a side stream, and in a CUDA graph whose replay sees
    the lengths, tables and queries of the moment."""
    import torch
    tac = tac_gpu
    heads, d, group, page, lens = 2, 128, 4, 16, [400, 123, 0]
    cache, table = _pools(tac, d, heads, page, [n + 32 for n in lens], 14, (64, *K8), (64, *V4))
    bounds = _boxes(tac, cache.pages, heads, d, page, 3)
    lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
    start = torch.tensor(lens, dtype=torch.int32, device="cuda")
    keys = torch.randn((3, heads, d), generator=_gen(2), device="cuda").to(_dtype(dtype))
    q = _queries(3, heads * group, d, dtype, 1)
    codes, scales = bounds.codes.clone(), bounds.scales.clone()

    def step(stream=None, **kw):
        tac.page_bounds(bounds, keys, table, start, stream=stream)
        sel, cnt = tac.select_pages(q, bounds, table, lengths, 6, stream=stream)
        return sel, cnt, tac.attend_pages(q, cache, table, lengths, 0.088, sel, cnt, stream=stream, **kw)

    want = [t.clone() for t in step()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    bounds.codes.copy_(codes)
    bounds.scales.copy_(scales)
    side.wait_stream(torch.cuda.current_stream())
    got = step(side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(held, want))
    lengths.copy_(torch.tensor([77, 16, 30], dtype=torch.int32))
    start.copy_(lengths)
    q.mul_(0.5)
    bounds.codes.copy_(codes)
    bounds.scales.copy_(scales)
    graph.replay()
    torch.cuda.synchronize()
    after = [t.clone() for t in held]
    bounds.codes.copy_(codes)
    bounds.scales.copy_(scales)
    assert all(torch.equal(a, b) for a, b in zip(step(), after))


def test_same_call_same_bits(tac_gpu):
    import torch
    tac = tac_gpu
    lens = [3000, 10, 777, 2048]
    cache, table = _pools(tac, 128, 4, 64, lens, 2, (64, *K8), (64, *V4))
    lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
    for dtype in ("bf16", "fp32"):
        q = _queries(4, 16, 128, dtype, 5)
        a = tac.attend_pages(q, cache, table, lengths, 0.088)
        assert all(torch.equal(a, tac.attend_pages(q, cache, table, lengths, 0.088)) for _ in range(3))


def test_long_pool_offsets_pass_32_bits(tac_gpu, orc):
    """Record and box offsets above 2^32 bytes: the last pages of a pool of 5 GB a plane."""
    import torch
    tac = tac_gpu
    heads, d, page = 8, 128, 256
    pages = 38_000                               # 77.8 M slots: 4.98 GB of K norms, 3.7 GB of angles
    cfgs = [tac.layer_cfg(d, 64, b, m, 0, 3, kv) for kv, (b, m) in enumerate((K8, (8, 0)))]
    cache = tac.PagedCache.empty(cfgs[0], cfgs[1], pages, heads, page)
    lens = [600, 300]
    table = torch.tensor([[pages - 1, 0, pages - 2], [pages - 3, pages // 2, -1]], dtype=torch.int32, device="cuda")
    small, t2 = _pools(tac, d, heads, page, lens, 3, (64, *K8), (64, 8, 0), spare=0)
    for a, b in ((cache.k, small.k), (cache.v, small.v)):
        ab, nb = tac.angle_row_bytes(a.cfg), tac.norm_row_bytes(a.cfg)
        for s in range(2):
            for j in range(-(-lens[s] // page)):
                n = heads * page
                src, dst = int(t2[s, j]) * n, int(table[s, j]) * n
                a.codes[dst * ab: (dst + n) * ab] = b.codes[src * ab: (src + n) * ab]
                a.norms[dst * nb: (dst + n) * nb] = b.norms[src * nb: (src + n) * nb]
                ho, hs = tac.header_offset(a.cfg, a.capacity), tac.header_offset(b.cfg, b.capacity)
                a.norms[ho + 8 * dst: ho + 8 * (dst + n)] = b.norms[hs + 8 * src: hs + 8 * (src + n)]
    lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
    for dtype in ("bf16", "fp32"):
        q = _queries(2, heads * 4, d, dtype, 6)
        a, b = tac.attend_pages(q, cache, table, lengths, 0.088), tac.attend_pages(q, small, t2, lengths, 0.088)
        assert torch.equal(a, b)

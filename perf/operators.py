"""Workloads of the paged-cache operators: what a serving program asks of a record cache
that lives in pages, at every decode step and after every prompt.

`op` names the operator:

  bounds   page_bounds: keys just written -> the box of each touched (page, KV head), 8 bits
  select   select_pages: the pages whose box may hold the largest scores, for each (sequence, KV head)
  attend   attend_pages: one new token's attention over all pages, or (`budget` > 0) over selected ones
  step     the three in turn, as one layer of a decode step on long caches runs them

`own` false: elementary torch operations in 32 bits.  `own` true: the package's calls.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

# (bits, mode) of the K and V norms; modes: 0 linear, 1 log, 2 fp32
NORMS = {"k8v4log": ((8, 0), (4, 1)), "norm8": ((8, 0), (8, 0)), "fp32": ((32, 2), (32, 2))}
FLT_MAX = 3.4028234663852886e38


def _case(name, op, seqs, heads, d, tokens, page, *, tokens_lo=0, group=0, budget=0, dtype="bf16", n_k=64, n_v=64,
          norms="k8v4log", new=0):
    return dict(name=name, op=op, seqs=seqs, heads=heads, d=d, tokens=tokens, tokens_lo=tokens_lo, page=page,
                group=group, budget=budget, dtype=dtype, n_k=n_k, n_v=n_v, norms=norms, new=new)


def listed():
    return [
        # one decode step of a serving batch: a key a head for each of 256 sequences, pages of 256 tokens
        _case("bounds_step_256seq", "bounds", 256, 8, 128, 4096, 256, tokens_lo=1024, new=1),
        # four prompts of odd lengths, the first chunk of some and a later one of others
        _case("bounds_prompts", "bounds", 4, 8, 128, 16384, 64, tokens_lo=8192, new=8191),
        # one prompt of a small model in fp32, small pages
        _case("bounds_prompt_d64_fp32", "bounds", 1, 8, 64, 2047, 16, dtype="fp32", new=2047),
        # one conversation, small pages: the latency of a choice among 257 pages
        _case("select_1seq_4k", "select", 1, 8, 128, 4097, 16, group=4, budget=64),
        # a batch of very different lengths
        _case("select_batch_ragged", "select", 32, 8, 128, 32768, 64, tokens_lo=1024, group=4, budget=64),
        # two documents of 131072 tokens in small pages, fp32 queries in groups of 8
        _case("select_long_p16_fp32", "select", 2, 4, 128, 131071, 16, group=8, budget=512, dtype="fp32"),
        # one layer of one conversation
        _case("attend_1seq_4k", "attend", 1, 8, 128, 4097, 16, group=4),
        # one layer of a batch of very different lengths, 8-bit norms on both sides
        _case("attend_ragged_norm8", "attend", 16, 8, 128, 32768, 256, tokens_lo=1024, group=4, norms="norm8"),
        # a small model (d = 64), fp32 queries
        _case("attend_d64_fp32", "attend", 16, 8, 64, 8192, 64, group=4, dtype="fp32", n_k=128),
        # the largest: 32 caches of 32768 tokens, every record read
        _case("attend_full_32k", "attend", 32, 8, 128, 32768, 64, group=4),
        # the same batch over 64 selected pages a head
        _case("attend_selected", "attend", 32, 8, 128, 32768, 64, tokens_lo=1024, group=4, budget=64),
        # one layer of a decode step on long documents: bounds of the new keys, choice, attention
        _case("step_long_128k", "step", 8, 4, 128, 131072, 64, tokens_lo=65536, group=8, budget=64, n_k=256, new=1),
    ]


def _log(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi], odd as often as not."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["bounds", "select", "attend", "attend", "attend", "step"])
    ns = [16, 32, 48, 56, 64, 64, 128, 256]
    c = dict(op=op, seqs=_log(rng, 1, 256 if op == "bounds" else 64), heads=rng.choice([1, 2, 4, 8]),
             d=rng.choice([64, 128, 128]), tokens=1, tokens_lo=0, page=rng.choice([16, 32, 48, 64, 64, 128, 256]),
             group=0, budget=0, dtype=rng.choice(["bf16", "bf16", "fp32"]), n_k=rng.choice(ns), n_v=rng.choice(ns),
             norms=rng.choice(["k8v4log", "k8v4log", "norm8", "fp32"]), new=0)
    # token-heads are bounded so that no draw is larger than the largest listed case
    cap = (8 << 20) // (2 if c["norms"] == "fp32" else 1)
    c["tokens"] = _log(rng, 1, max(16, min(131072, cap // (2 * c["seqs"] * c["heads"]))))
    c["tokens_lo"] = rng.choice([0, max(1, c["tokens"] // 16)])
    if op == "select":  # with pages enough that there is a choice
        c["tokens"] = max(c["tokens"], _log(rng, 64 * c["page"], 128 * c["page"]))
        c["tokens_lo"] = rng.choice([0, c["tokens"] // 4])
    pages = -(-c["tokens"] // c["page"])
    if op != "bounds":
        c["group"] = rng.choice([1, 2, 3, 4, 4, 5, 8])
    if op == "select":
        c["budget"] = _log(rng, 4, max(4, min(1024, pages // 4)))
    elif op == "step":
        c["budget"] = _log(rng, 2, max(2, min(1024, pages)))
    elif op == "attend" and rng.random() < 0.4:
        c["budget"] = _log(rng, 1, pages)
    if op == "bounds":
        c["new"] = rng.choice([1, _log(rng, 1, min(8192, c["tokens"])), min(8192, c["tokens"])])
    elif op == "step":
        c["new"] = 1
    return c


# ---------------------------------------------------------------------------
# shapes
# ---------------------------------------------------------------------------
def _lengths(c):
    """Tokens of each sequence: all `tokens`, or spread over the logarithm of [tokens_lo, tokens]; of eight
    sequences or more the last is a padded place of the batch, with no token."""
    lo, hi, s = c["tokens_lo"], c["tokens"], c["seqs"]
    if not lo:
        got = [hi] * s
    else:
        got = [max(1, min(hi, int(lo * (hi / lo) ** ((i + 0.5) / s)) | (i & 1))) for i in range(s)]
    if s >= 8 and c["op"] != "bounds":
        got[-1] = 0
    return got


def _news(c):
    """(first new position, new tokens) of each sequence: the last `new` of its tokens, or all of them where that is fewer."""
    return [(max(0, n - c["new"]), min(n, c["new"])) for n in _lengths(c)]


def _pages(c, n):
    return -(-n // c["page"])


def _bits(n):
    return max(1, math.ceil(math.log2(n)))


def _row_bytes(c, n, bits, mode):
    p = c["d"] // 2
    return p * _bits(n) // 8 + p * bits // 8 + (0 if mode == 2 else 8)


def _touched(c):
    """Pages that new rows touch, and those of them that held tokens before."""
    new = [(a, k) for a, k in _news(c) if k]
    return sum(_pages(c, a + k) - a // c["page"] for a, k in new), sum(a % c["page"] > 0 for a, k in new)


def _seen(c):
    """Token-heads that attention reads: all, or those of the selected pages (the last page among them)."""
    total = 0
    for n in _lengths(c):
        if c["budget"] and _pages(c, n) > c["budget"]:
            n = (c["budget"] - 1) * c["page"] + (n - (_pages(c, n) - 1) * c["page"])
        total += n
    return total * c["heads"]


def work(c):
    d, h, esz = c["d"], c["heads"], 2 if c["dtype"] == "bf16" else 4
    total, flops = 0.0, 0.0
    if c["op"] in ("bounds", "step"):
        rows = sum(k for _, k in _news(c)) * h
        touched, before = _touched(c)
        total += rows * d * esz + (touched + before) * h * (2 * d + 4) + 4 * c["seqs"]
        flops += 2 * rows * d
    if c["op"] in ("select", "step"):
        pages = sum(_pages(c, n) for n in _lengths(c))
        total += pages * (h * (2 * d + 4) + 4) + c["seqs"] * h * (c["group"] * d * esz + 4 * c["budget"] + 4)
        flops += 2 * pages * h * c["group"] * d
    if c["op"] in ("attend", "step"):
        (bk, mk), (bv, mv) = NORMS[c["norms"]]
        t = _seen(c)
        total += t * (_row_bytes(c, c["n_k"], bk, mk) + _row_bytes(c, c["n_v"], bv, mv))
        total += 2 * c["seqs"] * h * c["group"] * d * esz
        # two products a query, and about ten operations a pair to decode
        flops += t * (4 * d * c["group"] + 10 * d)
    return {"bytes": total, "flops": flops}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _gen(seed, *key):
    g = torch.Generator(device="cuda")
    v = int(seed) & 0x7FFFFFFF
    for k in key:
        v = (v * 1_000_003 + int(k) + 1) & 0x7FFFFFFFFFFF
    g.manual_seed(v)
    return g


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _hadamard(d, dtype):
    h = torch.ones((1, 1), dtype=dtype, device="cuda")
    while h.shape[0] < d:
        h = torch.cat([torch.cat([h, h], 1), torch.cat([h, -h], 1)], 0)
    return h / math.sqrt(d)


def _order(d):
    """The pair whose code is in position v of a record (d = 64, 128)."""
    m = d // 16
    return [4 * (v % m) + (v // m) % 4 + 4 * m * (v // (4 * m)) for v in range(d // 2)]


def _up16(v):
    return (v + 15) // 16 * 16


def _pack(k, w):
    """Codes [rows, p] below 2^w as w-bit fields, LSB first: [rows, p w / 8] bytes."""
    if w == 8:
        return k.to(torch.uint8)
    b = (k.to(torch.uint8)[..., None] >> torch.arange(w, device="cuda", dtype=torch.uint8)) & 1
    b = b.reshape(k.shape[0], -1, 8) << torch.arange(8, device="cuda", dtype=torch.uint8)
    return b.sum(dim=-1, dtype=torch.uint8)


def _planes(c, slots, n, bits, mode):
    p = c["d"] // 2
    off = _up16(slots * p * bits // 8)
    return {"n": n, "bits": bits, "mode": mode, "off": off, "slots": slots,
            "codes": torch.zeros(_up16(slots * p * _bits(n) // 8), dtype=torch.uint8, device="cuda"),
            "norms": torch.zeros(_up16(off + (0 if mode == 2 else 8 * slots)), dtype=torch.uint8, device="cuda")}


def _encode_into(c, pl, x, at):
    """The records of rows x [rows, d] in slots at..at+rows."""
    d, p, n, bits, mode = c["d"], c["d"] // 2, pl["n"], pl["bits"], pl["mode"]
    rows = x.shape[0]
    y = ((x.float() * pl["signs"]) @ _hadamard(d, torch.float32)).reshape(rows, p, 2)[:, _order(d)]
    k = torch.remainder(torch.floor(torch.atan2(y[..., 1], y[..., 0]) * (n / (2 * math.pi)) + 0.5), n)
    ab = p * _bits(n) // 8
    pl["codes"][at * ab: (at + rows) * ab] = _pack(k, _bits(n)).reshape(-1)
    r = torch.hypot(y[..., 0], y[..., 1])
    nb = p * bits // 8
    if mode == 2:
        pl["norms"][at * nb: (at + rows) * nb] = r.contiguous().view(torch.uint8).reshape(-1)
        return
    hi = r.amax(dim=1, keepdim=True)
    lo = torch.maximum(r.amin(dim=1, keepdim=True), hi * 2.0**-24) if mode == 1 else r.amin(dim=1, keepdim=True)
    top = (1 << bits) - 1
    a, b, v = (torch.log2(lo), torch.log2(hi), torch.log2(torch.maximum(r, lo))) if mode == 1 else (lo, hi, r)
    q = torch.floor((v - a) / (b - a) * top + 0.5).nan_to_num_(0.0).clamp_(0, top)
    pl["norms"][at * nb: (at + rows) * nb] = _pack(q, bits).reshape(-1)
    pl["norms"][pl["off"] + 8 * at: pl["off"] + 8 * (at + rows)] = torch.cat([lo, hi], dim=1).view(torch.uint8).reshape(-1)


def _values(c, pages, g, scales):
    """Rows [pages, heads, page, d]: channel scales of the head, and a direction that a page's tokens share."""
    x = torch.randn((pages, c["heads"], c["page"], c["d"]), generator=g, device="cuda")
    x += torch.randn((pages, c["heads"], 1, c["d"]), generator=g, device="cuda")
    return (x * scales[None, :, None, :]).to(_dtype(c))


def _scales(c, g):
    """Channel scales of each head: lognormal, with one channel in a hundred far larger."""
    s = torch.exp(0.5 * torch.randn((c["heads"], c["d"]), generator=g, device="cuda"))
    return s * torch.where(torch.rand((c["heads"], c["d"]), generator=g, device="cuda") < 0.01, 10.0, 1.0)


def _pow2_scale(a):
    """2^e, e the smallest whole number >= -126 with a <= 127 * 2^e."""
    m, x = torch.frexp(a)
    e = torch.where(a > 0, torch.where(m <= 127.0 / 128.0, x - 7, x - 6), -126).clamp(min=-126)
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def prepare(c, seed):
    """The paged pools as earlier steps left them (in every slot a record: stale ones beyond the sequences' ends),
    page tables and lengths on the device, the new token's queries and keys."""
    d, h, page, lens = c["d"], c["heads"], c["page"], _lengths(c)
    g = _gen(seed, 5)
    per = [_pages(c, n) for n in lens]
    width, pages = max(1, max(per)), sum(per) + 3
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((c["seqs"], width), -1, dtype=torch.int32, device="cuda")
    row = torch.tensor(np.repeat(np.arange(c["seqs"]), per), device="cuda")
    col = torch.tensor(np.concatenate([np.arange(n) for n in per] + [np.zeros(0, np.int64)]).astype(np.int64), device="cuda")
    table[row, col] = order[: row.numel()]
    st = {"case": dict(c), "table": table, "lengths": torch.tensor(lens, dtype=torch.int32, device="cuda"),
          "scale": 1.0 / math.sqrt(d)}
    scales = _scales(c, g)
    chunk = max(1, (1 << 19) // (h * page))
    if c["op"] in ("attend", "step"):
        for kv, (n, (bits, mode)) in enumerate(zip((c["n_k"], c["n_v"]), NORMS[c["norms"]])):
            pl = _planes(c, pages * h * page, n, bits, mode)
            pl["signs"] = torch.where(torch.rand(d, generator=g, device="cuda") < 0.5, -1.0, 1.0)
            neg = (pl["signs"] < 0).cpu().numpy().reshape(-1, 32)
            pl["words"] = (neg.astype(np.uint64) << np.arange(32, dtype=np.uint64)).sum(axis=1).astype(np.uint32)
            st["kv"[kv]] = pl
    if c["op"] in ("select", "step", "bounds"):
        st["lohi"] = torch.zeros((pages, h, 2, d), dtype=torch.int8, device="cuda")
        st["bscale"] = torch.zeros((pages, h), dtype=torch.float32, device="cuda")
    for at in range(0, pages, chunk):
        m = min(chunk, pages - at)
        x = _values(c, m, g, scales)
        if "lohi" in st:
            lo, hi = x.float().amin(dim=2), x.float().amax(dim=2)
            s = _pow2_scale(torch.maximum(-lo, hi).amax(dim=-1))
            st["lohi"][at: at + m, :, 0] = torch.floor(lo / s[..., None]).to(torch.int8)
            st["lohi"][at: at + m, :, 1] = torch.ceil(hi / s[..., None]).to(torch.int8)
            st["bscale"][at: at + m] = s
        if "k" in st:
            _encode_into(c, st["k"], x.reshape(-1, d), at * h * page)
            _encode_into(c, st["v"], _values(c, m, g, scales.flip(0)).reshape(-1, d), at * h * page)
    if c["op"] != "bounds":
        st["q"] = (0.5 * torch.randn((c["seqs"], h * c["group"], d), generator=g, device="cuda")).to(_dtype(c))
    if c["op"] in ("bounds", "step"):
        new = _news(c)
        st["start"] = torch.tensor([a for a, _ in new], dtype=torch.int32, device="cuda")
        st["first"] = torch.tensor(np.concatenate([[0], np.cumsum([k for _, k in new])]), dtype=torch.int32, device="cuda")
        x = torch.randn((sum(k for _, k in new), h, d), generator=g, device="cuda")
        st["keys"] = (x * scales[None]).to(_dtype(c))
    if c["op"] == "attend" and c["budget"]:
        # pages that an earlier choice named: the last one and others at random, in ascending order
        n = (st["lengths"].long() + page - 1) // page
        rank = torch.rand((c["seqs"], h, width), generator=g, device="cuda")
        j = torch.arange(width, device="cuda")
        rank = torch.where(j == n[:, None, None] - 1, -1.0, torch.where(j < n[:, None, None], rank, 2.0))
        keep = min(c["budget"], width)
        sel = rank.argsort(dim=-1)[..., :keep]
        count = torch.minimum(n, torch.tensor(c["budget"], device="cuda"))[:, None].expand(-1, h)
        live = torch.arange(keep, device="cuda") < count[..., None]
        sel = torch.where(live, sel, width).sort(dim=-1).values
        st["selected"] = torch.full((c["seqs"], h, c["budget"]), -1, dtype=torch.int32, device="cuda")
        st["selected"][..., :keep] = torch.where(sel < width, sel, -1).to(torch.int32)
        st["counts"] = count.to(torch.int32).contiguous()
    return st


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------
def _plain_bounds(st):
    """The boxes after the new keys: (codes int8 [pages, heads, 2, d], scales fp32 [pages, heads])."""
    c, x = st["case"], st["keys"].float()
    rows, h, d = x.shape
    at = torch.arange(rows, device="cuda")
    seq = torch.searchsorted(st["first"][1:].contiguous(), at.to(torch.int32), right=True)
    pos = st["start"].long()[seq] + at - st["first"].long()[seq]
    page = st["table"].long()[seq, pos // c["page"]]
    where = page[:, None, None].expand(rows, h, d)
    lo, hi = (torch.full(st["lohi"].shape[:2] + (d,), s * math.inf, device="cuda") for s in (1, -1))
    lo.scatter_reduce_(0, where, x, "amin")
    hi.scatter_reduce_(0, where, x, "amax")
    bad = torch.zeros(st["bscale"].shape, device="cuda").scatter_reduce_(0, where[..., 0], (~torch.isfinite(x)).any(dim=-1).float(), "amax") > 0
    touched = torch.zeros(lo.shape[0], dtype=torch.bool, device="cuda").index_fill_(0, page, True)
    kept = torch.zeros(lo.shape[0], device="cuda").index_add_(0, page, (pos % c["page"] == 0).float())[:, None] == 0
    s_old = torch.where(kept, st["bscale"], 0.0)
    s_new = _pow2_scale(torch.where(touched[:, None], torch.maximum(-lo, hi).amax(dim=-1), 0.0))
    s = torch.where(bad, math.inf, torch.maximum(s_old, s_new))
    s = torch.where(touched[:, None], s, st["bscale"])
    ratio = torch.where(torch.isinf(s), 0.0, s_old / s)[..., None]
    old = st["lohi"].float()
    low = torch.minimum(torch.where(kept[..., None], torch.floor(old[:, :, 0] * ratio), math.inf), torch.floor(lo / s[..., None]))
    high = torch.maximum(torch.where(kept[..., None], torch.ceil(old[:, :, 1] * ratio), -math.inf), torch.ceil(hi / s[..., None]))
    low = torch.where(torch.isinf(s)[..., None], -127.0, low)
    high = torch.where(torch.isinf(s)[..., None], 127.0, high)
    codes = torch.where(touched[:, None, None, None], torch.stack([low, high], dim=2), old)
    return codes.to(torch.int8), s


def _plain_select(st, lohi, bscale):
    """(selected int32 [seqs, heads, budget], counts int32 [seqs, heads])."""
    c = st["case"]
    b, h, grp, d, width = c["seqs"], c["heads"], c["group"], c["d"], st["table"].shape[1]
    q = torch.nan_to_num(st["q"].float(), nan=0.0, posinf=0.0, neginf=0.0).reshape(b, h, grp, d)
    sq = _pow2_scale(q.abs().amax(dim=-1))
    qc = torch.round(q / sq[..., None])
    page = st["table"].long()
    box = lohi[page.clamp(min=0)].float().permute(0, 2, 3, 4, 1)               # [seqs, heads, 2, d, width]
    dot = qc.clamp(min=0) @ box[:, :, 1] + qc.clamp(max=0) @ box[:, :, 0]       # whole numbers below 2^24
    sp = bscale[page.clamp(min=0)].permute(0, 2, 1)
    score = torch.clamp((dot * sq[..., None]) * sp[:, :, None], -FLT_MAX, FLT_MAX).amax(dim=2)
    score = torch.where(torch.isinf(sp), FLT_MAX, score)
    score = torch.where((page < 0)[:, None], -math.inf, score)
    n = ((st["lengths"].long() + c["page"] - 1) // c["page"])[:, None, None]
    j = torch.arange(width, device="cuda")
    score = torch.where((j == 0) | (j == n - 1), math.inf, score)
    score = torch.where(j < n, score, -math.inf)
    best = score.sort(dim=-1, descending=True, stable=True).indices
    keep = min(c["budget"], width)
    count = torch.minimum(n, torch.tensor(c["budget"], device="cuda")).expand(b, h, 1)
    best = torch.where(torch.arange(keep, device="cuda") < count, best[..., :keep], width).sort(dim=-1).values
    out = torch.full((b, h, c["budget"]), -1, dtype=torch.int32, device="cuda")
    out[..., :keep] = torch.where(best < width, best, -1).to(torch.int32)
    return out, count[..., 0].to(torch.int32)


def _fields(rows, w, p):
    """p codes of w bits, LSB first, of byte rows [..., bytes]."""
    bit = torch.arange(p, device="cuda") * w
    low = rows[..., bit >> 3].to(torch.int32)
    high = rows[..., ((bit >> 3) + 1).clamp(max=rows.shape[-1] - 1)].to(torch.int32)
    return ((low | (high << 8)) >> (bit & 7).to(torch.int32)) & ((1 << w) - 1)


def _plain_rows(c, pl, slot):
    """The rows [..., d] that the records in `slot` stand for, in fp32."""
    d, p, w = c["d"], c["d"] // 2, _bits(pl["n"])
    ab, nb = p * w // 8, p * pl["bits"] // 8
    k = _fields(pl["codes"][: pl["slots"] * ab].reshape(-1, ab)[slot], w, p)
    norms = pl["norms"][: pl["slots"] * nb].reshape(-1, nb)[slot]
    if pl["mode"] == 2:
        r = norms.view(torch.float32)
    else:
        v = _fields(norms, pl["bits"], p).float()
        head = pl["norms"][pl["off"]: pl["off"] + 8 * pl["slots"]].view(torch.float32).reshape(-1, 2)[slot]
        lo, hi, top = head[..., :1], head[..., 1:], float((1 << pl["bits"]) - 1)
        if pl["mode"] == 1:
            a, b = torch.log2(lo), torch.log2(hi)
            r = torch.where(hi > lo, torch.exp2(a + v * ((b - a) / top)), lo)
        else:
            r = lo + v * ((hi - lo) / top)
    angle = k.clamp(max=pl["n"] - 1).float() * (2 * math.pi / pl["n"])
    back = torch.tensor(np.argsort(_order(d)), device="cuda")
    y = torch.stack([r * torch.cos(angle), r * torch.sin(angle)], dim=-1)[..., back, :]
    return (y.reshape(*y.shape[:-2], d) @ _hadamard(d, torch.float32)) * pl["signs"]


def _plain_attend(st, selected=None):
    """[seqs, heads * group, d], the queries' type."""
    c, page = st["case"], st["case"]["page"]
    b, h, grp, d = c["seqs"], c["heads"], c["group"], c["d"]
    if selected is None:
        j = torch.arange(st["table"].shape[1], device="cuda").expand(b, h, -1)
    else:
        j = selected.long()
    pos = (j[..., None] * page + torch.arange(page, device="cuda")).reshape(b, h, -1)
    live = (pos >= 0) & (pos < st["lengths"][:, None, None])
    phys = torch.gather(st["table"].long()[:, None].expand(b, h, -1), 2, (pos // page).clamp(0, st["table"].shape[1] - 1))
    live &= phys >= 0
    slot = torch.where(live, (phys * h + torch.arange(h, device="cuda")[:, None]) * page + pos % page, 0)
    q = st["q"].float().reshape(b, h, grp, d)
    s = (q @ _plain_rows(c, st["k"], slot).transpose(-1, -2)) * st["scale"]
    s = torch.where(live[:, :, None], s, -math.inf)
    top = s.amax(dim=-1, keepdim=True)
    e = torch.where(live[:, :, None], torch.exp(s - torch.where(torch.isinf(top), 0.0, top)), 0.0)
    total = e.sum(dim=-1, keepdim=True)
    v = torch.where(live[..., None], _plain_rows(c, st["v"], slot), 0.0)
    out = torch.where(total > 0, (e @ v) / total, 0.0)
    return out.reshape(b, h * grp, d).to(st["q"].dtype)


def _box_values(lohi, bscale):
    """The keys' bounds that the 8-bit codes stand for."""
    return lohi * bscale[..., None, None]


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def _handles(st):
    """The package's handles on the pools, as a program keeps them."""
    import paper_2603_27467_gb300 as tac
    c, got = st["case"], {}
    if "k" in st:
        caches = []
        for pl in (st["k"], st["v"]):
            cfg = tac.LayerCfg(c["d"], pl["n"], pl["bits"], pl["mode"], pl["words"])
            caches.append(tac.Cache(cfg, pl["slots"], pl["codes"], pl["norms"]))
        got["cache"] = tac.PagedCache(caches[0], caches[1], c["heads"], c["page"])
    if "lohi" in st:
        got["bounds"] = tac.PageBounds(st["lohi"], st["bscale"], c["page"])
    return got


def run(st):
    op, c = st["case"]["op"], st["case"]
    if own:
        import paper_2603_27467_gb300 as tac
        h = st.get("handles") or st.setdefault("handles", _handles(st))
        if op == "bounds":
            tac.page_bounds(h["bounds"], st["keys"], st["table"], st["start"], st["first"])
            return _box_values(st["lohi"], st["bscale"])
        if op == "select":
            return tac.select_pages(st["q"], h["bounds"], st["table"], st["lengths"], c["budget"])
        if op == "attend":
            return tac.attend_pages(st["q"], h["cache"], st["table"], st["lengths"], st["scale"],
                                    st.get("selected"), st.get("counts"))
        tac.page_bounds(h["bounds"], st["keys"], st["table"], st["start"], st["first"])
        sel, counts = tac.select_pages(st["q"], h["bounds"], st["table"], st["lengths"], c["budget"])
        out = tac.attend_pages(st["q"], h["cache"], st["table"], st["lengths"], st["scale"], sel, counts)
        return {"selected": sel, "counts": counts, "out": out}
    if op == "bounds":
        return _box_values(*_plain_bounds(st))
    if op == "select":
        return _plain_select(st, st["lohi"], st["bscale"])
    if op == "attend":
        return _plain_attend(st, st.get("selected"))
    sel, counts = _plain_select(st, *_plain_bounds(st))
    return {"selected": sel, "counts": counts, "out": _plain_attend(st, sel)}


# ---------------------------------------------------------------------------
# the same in 64 bits
# ---------------------------------------------------------------------------
def _exact_scale(a):
    """2^e for each element of a float64 array: the smallest e >= -126 with a <= 127 * 2^e."""
    e = np.ceil(np.log2(np.maximum(a, 1e-300) / 127.0))
    e = np.where(a > 127.0 * np.exp2(e), e + 1, np.where(a <= 127.0 * np.exp2(e - 1), e - 1, e))
    return np.exp2(np.maximum(e, -126.0))


def _exact_bounds(c, st):
    """(lo, hi) in whole steps and the step, float64, [pages, heads, d] and [pages, heads]."""
    codes = st["lohi"].cpu().numpy().astype(np.float64)
    lo, hi, s = codes[:, :, 0].copy(), codes[:, :, 1].copy(), st["bscale"].cpu().numpy().astype(np.float64)
    keys, table = st["keys"].double().cpu().numpy(), st["table"].cpu().numpy()
    at = 0
    for i, (start, count) in enumerate(_news(c)):
        while count:
            take = min(count, c["page"] - start % c["page"])
            page, x = table[i, start // c["page"]], keys[at: at + take]
            step = _exact_scale(np.abs(x).max(axis=(0, 2)))
            a, b = np.floor(x.min(axis=0) / step[:, None]), np.ceil(x.max(axis=0) / step[:, None])
            if start % c["page"]:
                both = np.maximum(step, s[page])
                a = np.minimum(np.floor(lo[page] * (s[page] / both)[:, None]), np.floor(x.min(axis=0) / both[:, None]))
                b = np.maximum(np.ceil(hi[page] * (s[page] / both)[:, None]), np.ceil(x.max(axis=0) / both[:, None]))
                step = both
            lo[page], hi[page], s[page] = a, b, step
            start, count, at = start + take, count - take, at + take
    return lo, hi, s


def _exact_select(c, st, lo, hi, s):
    q = st["q"].double().cpu().numpy().reshape(c["seqs"], c["heads"], c["group"], c["d"])
    step = _exact_scale(np.abs(q).max(axis=-1))
    qc, table = np.rint(q / step[..., None]), st["table"].cpu().numpy()
    sel = np.full((c["seqs"], c["heads"], c["budget"]), -1, np.int32)
    counts = np.zeros((c["seqs"], c["heads"]), np.int32)
    for i, n in enumerate(_lengths(c)):
        n = _pages(c, n)
        if not n:
            continue
        at = table[i, :n]
        for h in range(c["heads"]):
            best = np.full(n, -np.inf)
            for a in range(c["group"]):
                v = qc[i, h, a]
                dot = hi[at, h] @ np.maximum(v, 0) + lo[at, h] @ np.minimum(v, 0)
                best = np.maximum(best, dot * step[i, h, a] * s[at, h])
            best[[0, n - 1]] = np.inf
            got = np.sort(np.lexsort((np.arange(n), -best))[: c["budget"]])
            sel[i, h, : len(got)], counts[i, h] = got, len(got)
    return sel, counts


def _exact_pairs(c, pl, slot):
    """Rotated rows y^ [tokens, d/2, 2] of records, float64, in record order."""
    p, w = c["d"] // 2, _bits(pl["n"])

    def codes(plane, width):
        raw = plane[: pl["slots"] * p * width // 8].reshape(pl["slots"], -1)[slot].to(torch.int64)
        bits = (raw[..., None] >> torch.arange(8, device="cuda")) & 1
        return (bits.reshape(len(slot), p, width) << torch.arange(width, device="cuda")).sum(dim=-1)

    if pl["mode"] == 2:
        r = pl["norms"][: pl["slots"] * p * 4].view(torch.float32).reshape(-1, p)[slot].double()
    else:
        v = codes(pl["norms"], pl["bits"]).double()
        head = pl["norms"][pl["off"]: pl["off"] + 8 * pl["slots"]].view(torch.float32).reshape(-1, 2)[slot].double()
        t = v / ((1 << pl["bits"]) - 1)
        if pl["mode"] == 1:
            r = torch.where(head[:, :1] == head[:, 1:], head[:, :1], head[:, :1] ** (1 - t) * head[:, 1:] ** t)
        else:
            r = head[:, :1] * (1 - t) + head[:, 1:] * t
    z = torch.polar(r, codes(pl["codes"], w).double() * (2 * math.pi / pl["n"]))
    return torch.view_as_real(z)


def _exact_attend(c, st, sel=None):
    d, page, hm = c["d"], c["page"], _hadamard(c["d"], torch.float64)
    order = torch.tensor(_order(d), device="cuda")
    q = st["q"].double().reshape(c["seqs"], c["heads"], c["group"], d)
    turned = ((q * st["k"]["signs"].double()) @ hm).reshape(*q.shape[:-1], d // 2, 2)[..., order, :].reshape(q.shape)
    out = torch.zeros_like(q)
    for i, n in enumerate(_lengths(c)):
        for h in range(c["heads"]):
            j = np.arange(_pages(c, n)) if sel is None else sel[i, h][sel[i, h] >= 0]
            pos = (np.asarray(j, np.int64)[:, None] * page + np.arange(page)).reshape(-1)
            pos = torch.from_numpy(pos[pos < n]).cuda()
            if not len(pos):
                continue
            slot = (st["table"][i].long()[pos // page] * c["heads"] + h) * page + pos % page
            k = _exact_pairs(c, st["k"], slot).reshape(-1, d)
            w = torch.softmax(turned[i, h] @ k.T * st["scale"], dim=-1)
            y = (w @ _exact_pairs(c, st["v"], slot).reshape(-1, d)).reshape(-1, d // 2, 2)
            flat = torch.empty_like(y)
            flat[:, order] = y
            out[i, h] = (flat.reshape(-1, d) @ hm) * st["v"]["signs"].double()
    return out.reshape(c["seqs"], -1, d)


def exact(c, seed):
    st = prepare(c, seed)
    if c["op"] == "bounds":
        lo, hi, s = _exact_bounds(c, st)
        return np.stack([lo, hi], axis=2) * s[..., None, None]
    if c["op"] == "select":
        codes = st["lohi"].cpu().numpy().astype(np.float64)
        return _exact_select(c, st, codes[:, :, 0], codes[:, :, 1], st["bscale"].cpu().numpy().astype(np.float64))
    if c["op"] == "attend":
        return _exact_attend(c, st, st["selected"].cpu().numpy() if c["budget"] else None)
    sel, counts = _exact_select(c, st, *_exact_bounds(c, st))
    return {"selected": sel, "counts": counts, "out": _exact_attend(c, st, sel)}

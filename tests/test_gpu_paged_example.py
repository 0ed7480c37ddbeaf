"""The paged decode example end to end, and codebooks of the two norm schemes at every code width (GB300)."""
import math
import os
import sys

import pytest

import pages_ref as ref

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples"))


def test_example_reads_less_and_loses_little(tac_gpu):
    """With every page chosen the two calls read the same tokens; fewer pages read less and leave a
    larger error; a quarter of the themes' pages are enough for most of the attention."""
    import paged_decode
    lengths = [3000, 1111, 64, 1]
    all_, some, few = (paged_decode.run(lengths, b, steps=2, layers=1, seed=5) for b in (64, 16, 2))
    assert all_["share_read"] == 1.0 and all_["relative_error"] < 2.0**-7     # one bf16 rounding each
    assert few["share_read"] < some["share_read"] < 0.6
    assert some["relative_error"] < few["relative_error"] < 2.0
    assert math.isfinite(few["relative_error"])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("nk,nv", [(2, 256), (8, 8), (16, 128), (32, 4), (128, 32), (256, 16), (48, 56), (64, 256)])
@pytest.mark.parametrize("vnorm", [(4, 1), (8, 0)])
def test_norm_schemes_at_every_code_width(tac_gpu, orc, dtype, d, nk, nv, vnorm):
    """8-bit linear keys with 4-bit log or 8-bit linear values, whose kernels are built apart."""
    import test_gpu_pages as pages
    lens = [100, 33, 0, 16]
    cache, table = pages._pools(tac_gpu, d, 2, 32, lens, nk + nv, (nk, 8, 0), (nv, *vnorm))
    for group in (3, 6):
        pages._check_attend(tac_gpu, orc, cache, table, lens, pages._queries(len(lens), 2 * group, d, dtype, group))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_weights_over_many_powers_of_two(tac_gpu, orc, dtype):
    """Keys and values whose sizes differ by 2^20 from token to token: the running exponent of the
    weights moves up and the large values stand far above the others."""
    import numpy as np
    import torch
    import parity
    tac, heads, d, page, n, group = tac_gpu, 2, 128, 16, 300, 4
    import test_gpu_pages as pages
    cache, table = pages._pools(tac, d, heads, page, [n], 8, (64, 8, 0), (64, 4, 1))
    g = pages._gen(77)
    slot = cache.slots(table, torch.arange(n, device="cuda"), torch.zeros(n, dtype=torch.long, device="cuda"))
    v = torch.randn((n, heads, d), generator=g, device="cuda") * torch.exp2(torch.linspace(-10, 10, n, device="cuda"))[:, None, None]
    tac.encode_multi([tac.EncodeJob(cache.v.cfg, v.reshape(-1, d), cache.v, slot)])
    q = pages._queries(1, heads * group, d, dtype, 3) * 0.1
    pages._check_attend(tac, orc, cache, table, [n], q)
    flip = v.flip(0).contiguous()
    tac.encode_multi([tac.EncodeJob(cache.v.cfg, flip.reshape(-1, d), cache.v, slot)])
    got, want = pages._check_attend(tac, orc, cache, table, [n], q)
    # the 2-norm of the error stays that of the queries' type, whatever the order the exponents come in
    rel = np.linalg.norm(parity.to_f64(got) - want) / np.linalg.norm(want)
    assert rel < (2.0**-8 if dtype == "bf16" else 2.0**-18), rel


def test_tables_of_many_sequences(tac_gpu, orc):
    """More sequences (and selections) than a warp plans alone, in a table wider than any needs."""
    import numpy as np
    import torch
    tac = tac_gpu
    import test_gpu_pages as pages
    lens = [int(x) for x in np.random.default_rng(5).integers(0, 40, size=300)]
    cache, table = pages._pools(tac, 64, 1, 16, lens, 3, (64, 8, 0), (64, 4, 1), width=50)
    rows = ref.pool_rows(orc, cache.k), ref.pool_rows(orc, cache.v)
    q = pages._queries(300, 2, 64, "bf16", 1)
    pages._check_attend(tac, orc, cache, table, lens, q, rows=rows)
    sel = torch.tensor([[[0, 2, -1]]] * 300, dtype=torch.int32, device="cuda")
    cnt = torch.tensor([[s % 4] for s in range(300)], dtype=torch.int32, device="cuda")
    pages._check_attend(tac, orc, cache, table, lens, q, sel, cnt, rows=rows)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,rows,start", [(1, 2000, 0), (2, 255, 130), (2, 4096, 77), (16, 9000, 3)])
def test_bounds_of_long_pages(tac_gpu, dtype, d, heads, rows, start):
    """Pages of 256 and 1024 tokens, whose rows several warps share."""
    import torch
    tac = tac_gpu
    import test_gpu_pages as pages
    for page in (256, 1024):
        table, count = pages._table([start + rows], page, 1, 3)
        bounds = tac.PageBounds.empty(count, heads, d, page)
        bounds.codes.fill_(5)
        bounds.scales.fill_(0.5)
        keys = (torch.randn((rows, heads, d), generator=pages._gen(rows), device="cuda") * 7).to(pages._dtype(dtype))
        keys[rows // 2, 0, 3] = math.inf
        pages._check_bounds(tac, keys, bounds, table, [start], [0, rows], page)

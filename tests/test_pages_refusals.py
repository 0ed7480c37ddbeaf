"""What the paged-cache entry points refuse, and with which status (host only: nothing is launched)."""
import ctypes

import pytest

OK = 1 << 12      # an aligned address that is never read


def _paging(tac, **kw):
    v = dict(table=OK, stride=4, width=4, seqs=2, lengths=OK, pages=8, heads=2, page=16) | kw
    return tac._PAGING_FMT.pack(v["table"], v["stride"], v["width"], v["seqs"], v["lengths"], v["pages"], v["heads"], v["page"])


def _boxes(tac, codes=OK, scales=OK, d=64):
    return tac._BOXES_FMT.pack(codes, scales, d)


def _cfg(d=64, n=64, b=8, m=0):
    return bytes((ctypes.c_int32 * 8)(d, n, b, m, 0, 0, 0, 0))


def _attend(tac, **kw):
    v = dict(k=_cfg(), v=_cfg(), planes=[OK] * 4, capacity=256, paging=_paging(tac), sel=0, cnt=0, budget=0, dtype=0, group=4,
             scale=0.125, q=OK, qs=512, qr=64, out=OK, os=512, orow=64) | kw
    return tac._ATT_PAGES_FMT.pack(v["k"], v["v"], *v["planes"], v["capacity"], v["paging"], v["sel"], v["cnt"], v["budget"],
                                   v["dtype"], v["group"], v["scale"], v["q"], v["qs"], v["qr"], v["out"], v["os"], v["orow"])


PAGING = [(dict(seqs=-1), 1), (dict(width=-1), 1), (dict(pages=-1), 1), (dict(heads=0), 1), (dict(page=0), 1), (dict(page=8), 1),
          (dict(page=24), 2), (dict(page=65552), 1), (dict(stride=3), 1), (dict(table=0), 1), (dict(table=OK + 2), 1),
          (dict(width=1 << 27, stride=1 << 27, page=32), 2), (dict(seqs=1 << 24, heads=4), 2)]


@pytest.mark.parametrize("kw,code", PAGING + [(dict(lengths=0), 1), (dict(lengths=OK + 1), 1)])
def test_paging(tac_host, kw, code):
    tac, lib = tac_host, tac_host.load()
    bad = _paging(tac, **kw)
    assert lib.tac_select_pages(_boxes(tac), bad, OK, 0, 4, 512, 64, 4, 1, 1, OK, OK, None) == code
    assert tac.last_error()
    assert lib.tac_attend_pages(_attend(tac, paging=bad), OK, 1 << 40, None) == code
    assert lib.tac_attend_pages_workspace_bytes(_attend(tac, paging=bad)) == -1
    if "lengths" not in kw:
        assert lib.tac_page_bounds(_boxes(tac), bad, OK, 0, 2, 128, 64, None, OK, None) == code


@pytest.mark.parametrize("boxes,code", [(dict(d=32), 2), (dict(d=256), 2), (dict(codes=0), 1), (dict(codes=OK + 8), 1),
                                        (dict(scales=0), 1), (dict(scales=OK + 2), 1)])
def test_boxes(tac_host, boxes, code):
    tac, lib = tac_host, tac_host.load()
    assert lib.tac_select_pages(_boxes(tac, **boxes), _paging(tac), OK, 0, 4, 512, 64, 4, 1, 1, OK, OK, None) == code
    assert lib.tac_page_bounds(_boxes(tac, **boxes), _paging(tac), OK, 0, 2, 128, 64, None, OK, None) == code
    assert lib.tac_select_pages(None, _paging(tac), OK, 0, 4, 512, 64, 4, 1, 1, OK, OK, None) == 1
    assert lib.tac_page_bounds(_boxes(tac), None, OK, 0, 2, 128, 64, None, OK, None) == 1


@pytest.mark.parametrize("k,dtype,rows,rs,hs,first,start", [
    (0, 0, 2, 128, 64, None, OK), (OK + 8, 0, 2, 128, 64, None, OK), (OK, 2, 2, 128, 64, None, OK), (OK, 0, -1, 128, 64, OK, OK),
    (OK, 0, 3, 128, 64, None, OK), (OK, 0, 2, 132, 64, None, OK), (OK, 0, 2, 128, -64, None, OK), (OK, 0, 2, 128, 66, None, OK),
    (OK, 0, 2, 128, 64, None, 0), (OK, 0, 2, 128, 64, None, OK + 1), (OK, 0, 2, 128, 64, OK + 2, OK), (OK, 0, 1 << 31, 128, 64, OK, OK)])
def test_bounds_arguments(tac_host, k, dtype, rows, rs, hs, first, start):
    tac = tac_host
    assert tac.load().tac_page_bounds(_boxes(tac), _paging(tac), k, dtype, rows, rs, hs, first, start, None) == 1


@pytest.mark.parametrize("q,dtype,group,ss,rs,budget,kf,kl,sel,cnt", [
    (0, 0, 4, 512, 64, 4, 1, 1, OK, OK), (OK + 4, 0, 4, 512, 64, 4, 1, 1, OK, OK), (OK, 9, 4, 512, 64, 4, 1, 1, OK, OK),
    (OK, 0, 0, 512, 64, 4, 1, 1, OK, OK), (OK, 0, 9, 512, 64, 4, 1, 1, OK, OK), (OK, 0, 4, 513, 64, 4, 1, 1, OK, OK),
    (OK, 0, 4, 512, 65, 4, 1, 1, OK, OK), (OK, 0, 4, 512, -64, 4, 1, 1, OK, OK), (OK, 0, 4, 512, 64, 0, 0, 0, OK, OK),
    (OK, 0, 4, 512, 64, 4, -1, 0, OK, OK), (OK, 0, 4, 512, 64, 4, 3, 2, OK, OK), (OK, 0, 4, 512, 64, 4, 2**31 - 1, 2**31 - 1, OK, OK),
    (OK, 0, 4, 512, 64, 4, 1, 1, 0, OK), (OK, 0, 4, 512, 64, 4, 1, 1, OK, OK + 2)])
def test_select_arguments(tac_host, q, dtype, group, ss, rs, budget, kf, kl, sel, cnt):
    tac = tac_host
    assert tac.load().tac_select_pages(_boxes(tac), _paging(tac), q, dtype, group, ss, rs, budget, kf, kl, sel, cnt, None) == 1


def test_select_table_too_wide(tac_host):
    tac = tac_host
    wide = _paging(tac, width=262145, stride=262145)
    assert tac.load().tac_select_pages(_boxes(tac), wide, OK, 0, 4, 512, 64, 4, 1, 1, OK, OK, None) == 2


@pytest.mark.parametrize("kw,code", [
    (dict(k=_cfg(d=32), v=_cfg(d=32)), 2), (dict(v=_cfg(d=128)), 1), (dict(k=_cfg(n=3)), 2), (dict(v=_cfg(b=5)), 2),
    (dict(v=_cfg(m=7)), 1), (dict(group=0), 1), (dict(group=9), 1), (dict(dtype=3), 1), (dict(scale=float("nan")), 1),
    (dict(capacity=255), 1), (dict(capacity=-1), 1), (dict(sel=OK), 1), (dict(cnt=OK), 1), (dict(sel=OK, cnt=OK), 1),
    (dict(sel=OK + 1, cnt=OK, budget=4), 1), (dict(sel=OK, cnt=OK, budget=2**31 - 1), 2), (dict(planes=[0, OK, OK, OK]), 1),
    (dict(planes=[OK, OK, OK, OK + 8]), 1), (dict(q=0), 1), (dict(out=0), 1), (dict(q=OK + 8), 1), (dict(qs=516), 1),
    (dict(qr=4), 1), (dict(orow=-64), 1)])
def test_attend_arguments(tac_host, kw, code):
    tac, lib = tac_host, tac_host.load()
    assert lib.tac_attend_pages(_attend(tac, **kw), OK, 1 << 40, None) == code
    assert tac.last_error()
    assert lib.tac_attend_pages_workspace_bytes(_attend(tac, **kw)) == -1


def test_no_sequences_is_no_work(tac_host):
    """Nothing to do returns TAC_OK without a device, whatever the pointers."""
    tac, lib = tac_host, tac_host.load()
    none = _paging(tac, seqs=0, table=0, lengths=0)
    assert lib.tac_page_bounds(_boxes(tac), none, 0, 0, 0, 0, 0, None, 0, None) == 0
    assert lib.tac_select_pages(_boxes(tac), none, 0, 0, 4, 0, 0, 4, 1, 1, 0, 0, None) == 0
    assert lib.tac_attend_pages(_attend(tac, paging=none, q=0, out=0, planes=[0] * 4), None, 0, None) == 0
    assert lib.tac_attend_pages(None, None, 0, None) == 1


def test_binding_checks_tensors(tac_host):
    """Tensors on the CPU, of another type or shape, and halves of a selection raise before any call."""
    import torch
    tac = tac_host
    q = torch.zeros((2, 4, 64))
    table, lens = torch.zeros((2, 4), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    bounds = tac.PageBounds(torch.zeros((8, 2, 2, 64), dtype=torch.int8), torch.zeros((8, 2)), 16)
    cfg = tac.layer_cfg(64, 64, 8, 0)
    cache = tac.PagedCache(tac.Cache(cfg, 256, q, q), tac.Cache(cfg, 256, q, q), 2, 16)
    assert cache.pages == 8
    with pytest.raises(ValueError):
        tac.page_bounds(bounds, q, table, lens)
    with pytest.raises(ValueError):
        tac.select_pages(q, bounds, table, lens, 4)
    with pytest.raises(ValueError):
        tac.attend_pages(q, cache, table, lens, 0.1)
    with pytest.raises(ValueError):
        tac.PagedCache(tac.Cache(cfg, 256, q, q), tac.Cache(cfg, 128, q, q), 2, 16)

"""The 8-bit cache's fillers against ranges, buffers and sizes that a caller got wrong: what the
device's words claim never makes the call read behind the free list."""
import ctypes

import numpy as np
import pytest
import torch

import coded_reference as ref
from paper_2607_27735_amd import binding as B

FAKE = 0x10000


def bounded(n_free=16, **kw):
    p = dict(ctx=FAKE, new=FAKE + 4096, table=FAKE + 8192, free=FAKE + 12288, rng=FAKE + 16384, slots=FAKE + 20480,
             rows=FAKE + 24576, total=FAKE + 28672, out=FAKE + 32768)
    p.update(kw)
    return B.load().ssl_page_map_bounded(2, 64, 8, 32, n_free, *p.values(), None)


def test_refusals_of_the_bounded_call():
    assert bounded(n_free=-1) == B.SSL_ERR_SHAPE
    for name in ("ctx", "new", "table", "free", "rng", "slots", "rows", "total", "out"):
        assert bounded(**{name: None}) == B.SSL_ERR_NULL, name
        assert bounded(**{name: FAKE + 2}) == B.SSL_ERR_ALIGN, name
    assert bounded(n_free=0, free=None, ctx=None) == B.SSL_ERR_NULL      # (an empty list may have no address)
    assert bounded(n_free=0, free=None, total=FAKE) == B.SSL_ERR_SHAPE   # total_len is ctx_len


SIZES = dict(table=16, slots=32, rows=3, total=2, out=2, ctx=2, new=2, rng=2, free=16)   # int32 entries of bounded()'s call
OUTPUTS = ("table", "slots", "rows", "total", "out")


@pytest.mark.parametrize("written", OUTPUTS)
@pytest.mark.parametrize("other", list(SIZES))
def test_overlaps_are_refused(written, other):
    """An output that shares its first or last entry with anything else."""
    if other == written:
        return
    at = FAKE + 0x100000
    for shift in (4 * (SIZES[other] - 1), -4 * (SIZES[written] - 1)):
        assert bounded(**{other: at, written: at + shift}) == B.SSL_ERR_SHAPE
        if other != "free":
            p = dict(ctx=FAKE, new=FAKE + 4096, table=FAKE + 8192, free=FAKE + 12288, rng=FAKE + 16384, slots=FAKE + 20480,
                     rows=FAKE + 24576, total=FAKE + 28672, out=FAKE + 32768)
            p.update({other: at, written: at + shift})
            assert B.load().ssl_page_map(2, 64, 8, 32, *p.values(), None) == B.SSL_ERR_SHAPE


@pytest.mark.parametrize("page,block", [(128, 48), (64, 128), (64, 0), (64, -32), (100, 32)])
def test_an_empty_cache_keeps_to_its_scale_block(page, block):
    """A page of 128 tokens has no blocks of 48: not a cache whose blocks are of 64."""
    with pytest.raises(ValueError):
        B.CodeCache.empty(4, 2, page, block, device="cpu")


@pytest.mark.gpu
def test_neighbours_in_one_buffer():
    """All arrays side by side in one allocation: none overlaps."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    buf = torch.zeros(sum(SIZES.values()), dtype=torch.int32, device="cuda")
    t, at = {}, 0
    for name, n in SIZES.items():
        t[name] = buf[at:at + n]
        at += n
    t["ctx"].copy_(torch.tensor([3, 70]))
    t["new"].copy_(torch.tensor([2, 60]))
    t["rng"].copy_(torch.tensor([0, 16]))
    t["free"].copy_(torch.arange(100, 116))
    t["table"].view(2, 8)[0, 0], t["table"].view(2, 8)[1, 0], t["table"].view(2, 8)[1, 1] = 5, 6, 7
    B.PreparedPageMap(t["ctx"], t["new"], t["table"].view(2, 8), t["free"], t["rng"], 64, t["slots"], t["rows"], t["total"],
                      t["out"]).run()
    torch.cuda.synchronize()
    assert t["total"].tolist() == [5, 70] and t["slots"].tolist() == [5 * 64 + 3, 5 * 64 + 4] + [-1] * 30
    assert t["rows"].tolist() == [0, 2, 62] and t["out"].tolist() == [0, 16] and t["ctx"].tolist() == [3, 70]


@pytest.mark.gpu
@pytest.mark.parametrize("batch", [3, 300])
@pytest.mark.parametrize("first,end", [(0, 5), (2, 40), (2, 2 ** 31 - 1), (7, 9), (12, 14), (0, -1), (2 ** 31 - 1, -2 ** 31),
                                       (-3, 4), (-2 ** 31, 2 ** 31 - 1), (9, 4)])
def test_ranges_past_the_list(first, end, batch):
    """Ten free pages, and ranges that end behind them, start behind them, or are no ranges."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    rng = np.random.default_rng(end % 1000 + batch)
    up = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")
    page, width, n_free = 32, 6, 10
    ctx, new = rng.integers(0, 90, batch), rng.integers(0, 70, batch)
    free = rng.permutation(5000)[:n_free].astype(np.int32)
    table = rng.integers(5000, 9000, (batch, width)).astype(np.int32)
    want = table.copy()
    usable = min(end, n_free) if first >= 0 else first
    tokens = int(new.sum()) + 9
    slots, rows, total, left = ref.page_map(ctx, new, want, free, first, usable, page, tokens)
    got_table = up(table)
    got = B.page_map(up(ctx), up(new), got_table, up(free), up([first, end]), page, tokens)
    torch.cuda.synchronize()
    assert np.array_equal(got_table.cpu().numpy(), want)
    assert np.array_equal(got[0].cpu().numpy(), slots)
    assert np.array_equal(got[1].cpu().numpy(), rows) and np.array_equal(got[2].cpu().numpy(), total)
    assert got[3].tolist() == [left[0], end]


@pytest.mark.gpu
def test_an_empty_list():
    """No free pages: sequences that need none are served, the others are not."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU visible")
    up = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")
    table = up([[3, 9], [4, 8]])
    got = B.page_map(up([30, 32]), up([2, 1]), table, up(np.zeros(0)), up([0, 5]), 32, 4)
    assert got[0].tolist() == [3 * 32 + 30, 3 * 32 + 31, -1, -1] and got[2].tolist() == [32, 32] and got[3].tolist() == [0, 5]
    assert table.tolist() == [[3, 9], [4, 8]]

"""The coded calls at the ends of their tables and register runs: the longest
work items, the largest batches, row blocks of some sequences only, appends of
128-row blocks in long calls, long index sets.  Bars as in test_gpu_coded."""
import numpy as np
import pytest
import torch

import coded_reference as ref
from gpu_common import check_outputs
from paper_2607_27735_amd import binding as B
from test_gpu_coded import CODES, MODES, SM, check_append, index_sets, ints, on_gpu, run_verify

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU visible", allow_module_level=True)


@pytest.mark.parametrize("mode", list(MODES))
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("rows", [1, 4])
def test_longest_items(rows, code, mode):
    """Items of 8192 keys: a wave's 64 tiles fill its run (the stash of four rows ends before)."""
    c = ref.Cache(np.random.default_rng(71), [16384], 1, 64, 32, code)
    try:
        B.set_cu_budget(1 if mode == "two-sweep" else 2 if rows == 1 else 4)
        p = B.make_params(SM, verify_mode=MODES[mode])
        plan = B.verify_coded_plan(B.Shape(1, 1, 1, 128, 16384, rows), p, [16384], [rows])
        assert plan[1:] == ((8192, 2) if mode == "two-sweep" or rows == 1 else (4096, 4))
        run_verify(c, np.random.default_rng(5), 1, [rows], mode=MODES[mode])
        if mode == "two-sweep":   # (three row tiles)
            assert B.verify_coded_plan(B.Shape(1, 8, 1, 128, 16384, 5), p, [16384], [5])[1:] == (8192, 2)
            run_verify(c, np.random.default_rng(5), 8, [5], mode=MODES[mode])
    finally:
        B.set_cu_budget(0)


@pytest.mark.parametrize("mode", list(MODES))
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("batch", [16, 17, 32, 33, 48, 49, 64])
def test_batches(batch, code, mode):
    """Every turn of the sixteen-wide search for an item's sequence, to the table's end."""
    rng = np.random.default_rng(batch)
    ctx = rng.integers(7, 400, batch)
    ctx[-1], ctx[0] = 390, 7
    c = ref.Cache(rng, ctx, 2, 64, 32, code)
    run_verify(c, rng, 4, list(rng.integers(1, 8, batch)), mode=MODES[mode])


@pytest.mark.parametrize("mode", list(MODES))
@pytest.mark.parametrize("batch", [3, 19])
def test_row_blocks_of_some_sequences(batch, mode):
    """More than 64 rows per KV head in some sequences, few in the others: later row
    blocks have fewer sequences than the first."""
    rng = np.random.default_rng(batch)
    ql = rng.integers(1, 5, batch)
    ql[1], ql[-1] = 37, 20
    ctx = rng.integers(40, 500, batch)
    c = ref.Cache(rng, ctx, 2, 64, 64, "int8")
    run_verify(c, rng, 8, list(ql), mode=MODES[mode])
    run_verify(c, rng, 8, list(ql), mode=MODES[mode], per_head=True, window=30)


@pytest.mark.parametrize("mode", list(MODES))
def test_rows_49_to_64_beside_few(mode):
    """The largest item has four row tiles, others one to three."""
    rng = np.random.default_rng(8)
    c = ref.Cache(rng, [700, 300, 1000, 65], 1, 64, 32, "e4m3")
    run_verify(c, rng, 8, [8, 1, 3, 5], mode=MODES[mode])
    run_verify(c, rng, 8, [7, 2, 6, 1], mode=MODES[mode], out_fp32=False)


@pytest.mark.parametrize("code", CODES)
def test_append_long_blocks_of_128(code):
    """Runs of up to 128 rows in windows of 16: led anywhere, found in up to three loads."""
    rng = np.random.default_rng(78)
    check_append(rng, code, 128, 128, 8, [0, 17, 127], [3100, 1003, 2200])
    check_append(rng, code, 128, 256, 16, rng.integers(0, 256, 100), rng.integers(1, 140, 100))


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("ctx,hkv,budget,entries", [([9000], 2, 6001, 12002), ([9000, 4500, 8300, 6000], 8, 4096, 131072),
                                                    ([5000] * 4, 16, 4097, 262208)])
def test_long_index_sets(ctx, hkv, budget, entries, code):
    """More than 2048 entries per set, and calls of 131072 entries and more."""
    rng = np.random.default_rng(budget)
    c = ref.Cache(rng, ctx, hkv, 128, 64, code)
    idx, n = index_sets(rng, ctx, hkv, budget)
    assert sum(n) * hkv == entries
    cache, table = on_gpu(c)
    q, q64 = ref.bf16_normal(rng, len(ctx), hkv, 128, scale=2.0)
    want, oabs = ref.draft(c, q64, lambda b, u: idx[b, u, :n[b]], SM, hkv)
    p = B.make_params(SM, budget=budget, out_fp32=True)
    for o in (B.draft_attn_coded(q.cuda(), cache, table, c.max_ctx, ints(idx), n, p),
              B.draft_step_coded(q.cuda(), cache, table, c.max_ctx, ctx, ctx, p, ints(idx))):
        torch.cuda.synchronize()
        o = o.double().cpu().numpy()
        check_outputs(o, want, oabs, np.ones(want.shape[:2], bool))
        assert np.all(np.abs(o - want) <= 2.0 ** -9 * oabs)

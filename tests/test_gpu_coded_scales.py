"""Coded attention over caches whose scales lie anywhere that the append, or a
caller, may put them: what one call writes the others read.

Bars are those of test_gpu_coded: verify's weights are fp16 relative to their
row's largest, |dO| <= 2^-9 sum P|v| + the weights' absolute step
(coded_reference.weight_floor), scores within 1e-3 of each score."""
import numpy as np
import pytest
import torch

import coded_reference as ref
from gpu_common import check_scores
from paper_2607_27735_amd import binding as B
from test_gpu_coded import CODES, MODES, SM, code_cache, host, ints, on_gpu

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU visible", allow_module_level=True)


def check_verify(c: ref.Cache, q, q_len, mode, cus=0, sm=SM, out_fp32=True):
    """verify over c against the plain form; c is what the GPU's cache holds."""
    cache, table = on_gpu(c)
    p = B.make_params(sm, out_fp32=out_fp32, verify_mode=mode)
    try:
        B.set_cu_budget(cus)
        out, sc = B.verify_attn_coded(q.cuda(), cache, table, c.max_ctx, c.ctx, q_len, p)
    finally:
        B.set_cu_budget(0)
    torch.cuda.synchronize()
    o, s, q64 = out.double().cpu().numpy(), sc.double().cpu().numpy(), q.double().numpy()
    want, oabs, sh = ref.verify(c, q64, q_len, sm, 16)
    batch, hq = q.shape[0], q.shape[2]
    live = np.arange(q.shape[1])[None, :, None] < np.array(q_len)[:, None, None] * np.ones((1, 1, hq), bool)
    assert np.all(np.isfinite(o[live])), f"{int((~np.isfinite(o[live])).sum())} outputs are not finite"
    bound = 2.0 ** -9 * oabs + ref.weight_floor(c, q64, q_len, sm) + (0 if out_fp32 else 2.0 ** -8) * np.abs(want)
    over = (np.abs(o - want) / bound)[live].max()
    assert over <= 1, f"{over:.2f} times the bar"
    check_scores(s, sh.reshape(batch, c.n_kv, hq // c.n_kv, -1).sum(2), c.ctx)
    return o, want


def appended(rng, code, ctx, edit, n_kv=2, page=64, block=32):
    """A cache filled by the append from rows that edit(k, v) has changed, read back."""
    c = ref.Cache(rng, ctx, n_kv, page, block, code)
    cache = code_cache(np.zeros_like(c.k), np.zeros_like(c.v), np.zeros_like(c.ks), np.zeros_like(c.vs), code)
    slots = np.concatenate([c.table[b, np.arange(t) // page] * page + np.arange(t) % page for b, t in enumerate(ctx)])
    k, v = (rng.standard_normal((sum(ctx), n_kv, 128)).astype(np.float32) for _ in range(2))
    edit(k, v)
    up = lambda x: torch.from_numpy(x).to(torch.bfloat16).cuda()
    B.cache_append(cache, up(k), up(v), ints(slots))
    torch.cuda.synchronize()
    c.k, c.v, c.ks, c.vs = host(cache)
    return c


def huge(k, v):
    v[5, 0, 7], v[200, 1, 9], v[303, 0, 100] = np.inf, -np.inf, np.inf   # (bf16's largest)
    v[77, :, 3] = 2.0 ** 119
    v[130, 0] = 2.0 ** 118


@pytest.mark.parametrize("mode", list(MODES))
@pytest.mark.parametrize("code", CODES)
def test_verify_reads_what_the_append_writes(code, mode):
    """Infinities and values near fp32's largest in V: they count by their share of
    their own column, and every other element is as if they were not there."""
    c = appended(np.random.default_rng(1), code, [400, 70], huge)
    assert c.vs.max() == 2.0 ** (120 if code == "e4m3" else 122)
    # (flat rows: no key has more than a hundredth, so that no column passes fp32's range)
    q, _ = ref.bf16_normal(np.random.default_rng(2), 2, 5, 8, 128, scale=0.5)
    check_verify(c, q, [5, 2], MODES[mode])
    check_verify(c, q, [5, 2], MODES[mode], cus=1)


@pytest.mark.parametrize("mode", list(MODES))
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("low,high", [(-70, 90), (-126, 100), (60, 116), (-126, -100)])
def test_verify_scales_of_any_size(low, high, code, mode):
    """V's scales from block to block anywhere between 2^low and 2^high: a key's
    share of its row's sum and scores does not depend on V."""
    rng = np.random.default_rng(high + 200)
    c = ref.Cache(rng, [700, 333], 2, 64, 32, code)
    c.vs[...] = np.where(np.isnan(c.vs), c.vs, 2.0 ** rng.integers(low, high + 1, c.vs.shape))
    q, _ = ref.bf16_normal(rng, 2, 6, 8, 128, scale=1.5)
    check_verify(c, q, [6, 3], MODES[mode])


@pytest.mark.parametrize("mode", list(MODES))
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("low,high", [(-20, 120), (-80, 100), (-126, 110)])
def test_verify_far_scales_against_steep_logits(low, high, code, mode):
    """Keys that grow less likely by 2^-5 each while their block's V grows: their
    weights are alike though their probabilities are 2^150 apart.  (Scores below
    fp32's least normal number are not looked at.)"""
    c = ref.Cache(np.random.default_rng(3), [96], 1, 32, 32, code)
    one = 0x38 if code == "e4m3" else 0x01
    for j in range(3):      # three blocks; the keys of one have one logit
        pg = c.table[0, j]
        c.k[pg, 0], c.ks[pg, 0] = 0, 1.0
        c.k[pg, 0, :, 0] = one
        c.ks[pg, 0, 0] = [3.0, 2.0, 1.0][j]
        c.vs[pg, 0, 0] = 2.0 ** [low, (low + high) // 2, high][j]
    q = torch.zeros(1, 1, 4, 128, dtype=torch.bfloat16)
    step = (high - low) / 2 * np.log(2) / SM            # (a block's step in log2 units: (high - low) / 2)
    q[..., 0] = torch.tensor([step, step * 0.98, step * 1.02, 1.0])
    cache, table = on_gpu(c)
    out, _ = B.verify_attn_coded(q.cuda(), cache, table, 96, [96], [1], B.make_params(SM, out_fp32=True, verify_mode=MODES[mode]))
    torch.cuda.synchronize()
    q64 = q.double().numpy()
    want, oabs, _ = ref.verify(c, q64, [1], SM, 16)
    bound = 2.0 ** -9 * oabs + ref.weight_floor(c, q64, [1], SM)
    over = np.abs(out.double().cpu().numpy() - want) / bound
    assert over.max() <= 1, f"{over.max():.2f} times the bar"


@pytest.mark.parametrize("mode", list(MODES))
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("sm", [SM, 1e-9, 1e-37])
def test_verify_masks_keys_whose_logits_scale_to_nothing(sm, code, mode):
    """The last block, which some rows do not see all of, is of zero keys (the append
    gives them the scale 2^-126, a caller may give 0): masked is masked, however
    small the logits' factor."""
    rng = np.random.default_rng(6)
    c = ref.Cache(rng, [300, 31], 2, 64, 32, code)
    c.ks[c.table[0, 4], 0], c.ks[c.table[0, 4], 1] = 2.0 ** -126, 0.0
    c.ks[c.table[1, 0], 0, 0], c.ks[c.table[1, 0], 1, 0] = 0.0, 2.0 ** -126
    q, _ = ref.bf16_normal(rng, 2, 6, 8, 128, scale=1.5)
    check_verify(c, q, [6, 6], MODES[mode], sm=sm)


@pytest.mark.parametrize("mode", list(MODES))
@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("top", [1e3, 1e5, 9.9e6])
def test_verify_large_logits(top, code, mode):
    """One key takes each row, whichever tile it is in, and V's scales around it differ
    by 2^60.  A normalizer M + log2(L) is two roundings of 2^-24 |logit| log2(e) off, in
    log2 units: 2^-23 |logit| of itself."""
    rng = np.random.default_rng(9)
    c = ref.Cache(rng, [700], 1, 64, 32, code)
    c.k[c.table[0], 0] = 0
    c.ks[c.table[0]] = 1.0
    for t, x in ((3, 2), (130, -3), (333, 3), (600, 1)):          # whole multiples of the logit's unit
        mag = {1: (0x38, 1), 2: (0x40, 2), 3: (0x44, 3)}[abs(x)][code == "int8"]
        sign = 0 if x > 0 else (128 if code == "e4m3" else None)
        c.k[c.table[0, t // 64], 0, t % 64, 0] = np.uint8(256 - mag) if sign is None else mag + sign
    c.vs[c.table[0]] = 2.0 ** rng.integers(-30, 31, c.vs[c.table[0]].shape)
    q = torch.zeros(1, 3, 4, 128, dtype=torch.bfloat16)
    q[..., 0] = torch.tensor([1.0, -1.0, 0.5, -0.25]) * (top / 3 / SM)
    cache, table = on_gpu(c)
    out, sc = B.verify_attn_coded(q.cuda(), cache, table, 700, [700], [3], B.make_params(SM, out_fp32=True, verify_mode=MODES[mode]))
    torch.cuda.synchronize()
    want, oabs, sh = ref.verify(c, q.double().numpy(), [3], SM, 16)
    bar, least = 2.0 ** -9 + 2.0 ** -23 * top, 2.0 ** -31 * oabs.max(-1, keepdims=True)
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= bar * oabs + least)
    s, sh = sc.double().cpu().numpy(), sh.reshape(1, 1, 4, -1).sum(2)
    assert np.array_equal(sh > 1e-3, s > 1e-3) and np.allclose(s[sh > 1e-3], sh[sh > 1e-3], rtol=bar)


@pytest.mark.parametrize("mode", list(MODES))
@pytest.mark.parametrize("positions", [3, 10, 12, 16, 23])
def test_verify_scales_of_any_size_in_every_row_tile(positions, mode):
    """12 to 92 rows per KV head: one to four row tiles, and row blocks."""
    rng = np.random.default_rng(positions)
    c = ref.Cache(rng, [500, 260], 2, 64, 32, "e4m3")
    c.vs[...] = np.where(np.isnan(c.vs), c.vs, 2.0 ** rng.integers(-100, 101, c.vs.shape))
    q, _ = ref.bf16_normal(rng, 2, positions, 8, 128, scale=1.5)
    check_verify(c, q, [positions, 2], MODES[mode])
    check_verify(c, q, [positions, positions], MODES[mode], out_fp32=False)

"""Precision and range of the draft over a coded cache.

A weight (probability times V's scale) is two bf16 numbers, the second of what
the first leaves: off by at most 2^-8 2^-8 = 2^-16 of itself.  The logits of
these flat rows have sum |q k| sm_scale < 5, so a probability is off by at most
2 * 5 * 128 * 2^-24 = 7.7e-5, and sums of at most a few hundred fp32 terms by
2^-16: in all 7.7e-5 + 2 * 2^-16 = 1.1e-4 < 2^-12 of sum P|v|."""
import numpy as np
import pytest
import torch

import coded_reference as ref
from paper_2607_27735_amd import binding as B
from test_gpu_coded import CODES, SM, index_sets, ints, on_gpu
from test_gpu_coded_scales import appended

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU visible", allow_module_level=True)


def run(c, idx, n, q, units, budget, out_fp32=True, cus=0, per_head=False, step=False):
    cache, table = on_gpu(c)
    p = B.make_params(SM, budget=budget, out_fp32=out_fp32, per_head=per_head)
    try:
        B.set_cu_budget(cus)
        if step:
            o = B.draft_step_coded(q.cuda(), cache, table, c.max_ctx, c.ctx, c.ctx, p, ints(idx))
        else:
            o = B.draft_attn_coded(q.cuda(), cache, table, c.max_ctx, ints(idx), n, p)
    finally:
        B.set_cu_budget(0)
    torch.cuda.synchronize()
    want, oabs = ref.draft(c, q.double().numpy(), lambda b, u: idx[b, u, :n[b]], SM, units)
    return o.double().cpu().numpy(), want, oabs


@pytest.mark.parametrize("code", CODES)
@pytest.mark.parametrize("budget", [36, 60, 200, 500])
@pytest.mark.parametrize("pow2", [False, True])
def test_flat_rows(budget, code, pow2):
    """Rows whose keys count alike: every weight is between two 8-bit numbers."""
    rng = np.random.default_rng(budget)
    c = ref.Cache(rng, [600, 35], 2, 64, 32, code, pow2=pow2)
    idx, n = index_sets(rng, c.ctx, 2, budget)
    q, _ = ref.bf16_normal(rng, 2, 8, 128, scale=0.25)
    for cus in (0, 1):
        for step in (False, True):
            o, want, oabs = run(c, idx, n, q, 2, budget, cus=cus, step=step)
            over = (np.abs(o - want) / (2.0 ** -12 * oabs)).max()
            assert over <= 1, f"{over:.2f} times the bar"
    o, want, oabs = run(c, idx, n, q, 2, budget, out_fp32=False)
    assert np.all(np.abs(o - want) <= 2.0 ** -12 * oabs + 2.0 ** -8 * np.abs(want) * (1 + 2.0 ** -8))


def huge(k, v):
    v[5, 0, 7], v[200, 1, 9], v[303, 0, 100] = np.inf, -np.inf, np.inf   # (bf16's largest)
    v[77, :, 3] = 2.0 ** 119


@pytest.mark.parametrize("code", CODES)
def test_reads_what_the_append_writes(code):
    """Infinities and values near fp32's largest in V, in keys that are their row's
    likeliest and in others: finite where the plain form is."""
    c = appended(np.random.default_rng(1), code, [400, 70], huge)
    rng = np.random.default_rng(2)
    idx, n = index_sets(rng, c.ctx, 2, 400)
    q, q64 = ref.bf16_normal(rng, 2, 8, 128, scale=0.25)
    for head, key in ((0, 5), (1, 303), (5, 200), (6, 77)):   # rows that give one of them the most, about a third
        k = c.values("k", 0, head // 4, np.array([key]))[0]
        q[0, head] = torch.from_numpy(k * (5.3 / SM / (k @ k))).to(torch.bfloat16)
    o, want, oabs = run(c, idx, n, q, 2, 400)
    fits = np.abs(want) < 2.0 ** 127.9
    assert fits.all() and np.all(np.isfinite(o)), f"{int((~np.isfinite(o)).sum())} outputs are not finite"
    assert np.all(np.abs(o - want) <= 2.0 ** -9 * oabs)

"""Cross and shared-prefix attention on values outside the ordinary: NaN and infinite logits of real keys, the type's lowest
value behind a causal limit, logits far beyond a trained layer's.

What the definition gives: a row with a NaN or +inf logit among its visible keys has no finite result (it must not look
like a row without keys); a logit of -inf has weight 0, and a row of nothing but such logits has no key to weigh (zeros,
log-sum-exp -inf); a key that a row does not see has no part in it."""
import math

import pytest
import torch

import test_gpu_segment_attn as base
from paper_2609_38984_b200 import swam

U16, U32 = base.U16, base.U32
pytestmark = pytest.mark.gpu
DT = base.DT
NAN, INF = math.nan, math.inf

# (type, variant, queries, heads, kv heads, head dim, keys): every kernel and row tile, direct and in pieces
PLANS = [
    ("bf16", swam.ATTN_AUTO, 300, 2, 2, 64, 300),         # tcgen05, 256-row tiles
    ("bf16", swam.ATTN_AUTO, 300, 2, 2, 128, 300),
    ("bf16", swam.ATTN_AUTO, 100, 2, 2, 64, 300),         # tcgen05, 128-row tiles, two key streams
    ("bf16", swam.ATTN_AUTO, 100, 2, 2, 128, 300),
    ("bf16", swam.ATTN_AUTO, 300, 2, 2, 64, 5000),        # in pieces
    ("bf16", swam.ATTN_AUTO, 100, 2, 2, 128, 5000),
    ("bf16", swam.ATTN_AUTO, 1, 2, 2, 64, 300),           # warp-level
    ("bf16", swam.ATTN_AUTO, 1, 2, 2, 128, 5000),
    ("bf16", swam.ATTN_AUTO, 70, 2, 2, 32, 300),
    ("bf16", swam.ATTN_WARP_MMA, 100, 2, 2, 64, 300),
    ("f32", swam.ATTN_AUTO, 1, 2, 2, 64, 300),
    ("f32", swam.ATTN_AUTO, 70, 2, 2, 128, 300),
    ("f32", swam.ATTN_AUTO, 30, 2, 2, 32, 5000),
]
IDS = ["-".join(map(str, (p[0], "warp" if p[1] else "auto") + p[2:])) for p in PLANS]
plans = pytest.mark.parametrize("plan", PLANS, ids=IDS)


def context(plan, B):
    dtype, variant, n_q, H, kv, D, n_kv = plan
    ctx = base.make_ctx(B, H, D, kv, swam.F32 if dtype == "f32" else swam.BF16)
    ctx.set_option(swam.OPT_ATTN_VARIANT, variant)
    return ctx


@plans
def test_a_nan_query_is_its_own_rows_loss_only(plan):
    dtype, variant, n_q, H, kv, D, n_kv = plan
    dt, B = DT[dtype], 2
    gen = torch.Generator(device="cuda").manual_seed(n_q + D)
    ctx = context(plan, B)
    q = base.rand(gen, B, n_q, H, D, dtype=dt)
    k, v = base.rand(gen, B, n_kv, kv, D, dtype=dt), base.rand(gen, B, n_kv, kv, D, dtype=dt)
    lost = torch.zeros(n_q, dtype=torch.bool, device="cuda")
    lost[[t for t in (0, 7, 31, 64, 99, 200) if t < n_q]] = True
    q[1, lost, 1, 5] = NAN
    out, lse = ctx.cross_attn(q, k, v, want_lse=True)
    ctx.check()
    assert torch.isnan(out[1, lost, 1]).all() and torch.isnan(lse[1, 1, lost]).all()
    clean = q.clone()
    clean[1, lost, 1] = 0.0
    want, want_lse = ctx.cross_attn(clean, k, v, want_lse=True)
    ctx.check()
    # the other rows by the definition (a warp that holds a lost row takes its sums in another order, so not to the bit)
    out[1, lost, 1], lse[1, 1, lost] = want[1, lost, 1], want_lse[1, 1, lost]
    mask = torch.ones(n_q, n_kv, dtype=torch.bool, device="cuda")
    base.compare(out, lse, clean, lambda b, h: (k[b, :, h].double(), v[b, :, h].double(), mask), D, dt)

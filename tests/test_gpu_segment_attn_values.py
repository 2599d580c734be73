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


def positions(n_kv):
    return sorted({0, 1, 2, 3, 15, 16, 17, 31, 32, 33, 64, 65, 100, 127, 128, 129, 160, n_kv - 2, n_kv - 1})


def one_component(plan, raw):
    """q and k with a single component each, whose product (exact in 24 bits) is raw[b][c] for every query of sample b."""
    dtype, variant, n_q, H, kv, D, n_kv = plan
    B = len(raw)
    q = torch.zeros(B, n_q, H, D, dtype=DT[dtype], device="cuda")
    k = torch.zeros(B, n_kv, kv, D, dtype=DT[dtype], device="cuda")
    q[..., 3] = 2.0 ** 20
    k[..., 3] = (torch.tensor(raw, dtype=torch.float64, device="cuda") * 2.0 ** -20).to(DT[dtype])[:, :, None]
    return q, k


@plans
@pytest.mark.parametrize("what", [NAN, INF])
def test_a_row_with_a_nan_or_infinite_logit_is_no_row_without_keys(plan, what):
    """Sample b has one bad key, at the b-th position, in its first head only: every row of that head is lost, and none of
    the other head's."""
    dtype, variant, n_q, H, kv, D, n_kv = plan
    dt, at = DT[dtype], positions(n_kv)
    B = len(at)
    gen = torch.Generator(device="cuda").manual_seed(n_q + D)
    ctx = context(plan, B)
    q = base.rand(gen, B, n_q, H, D, dtype=dt)
    q[..., 0] = q[..., 0].abs() + 0.5
    k, v = base.rand(gen, B, n_kv, kv, D, dtype=dt), base.rand(gen, B, n_kv, kv, D, dtype=dt)
    for b, c in enumerate(at):
        if what != what:
            k[b, c, 0] = what
        else:
            k[b, c, 0, 0] = what
    out, lse = ctx.cross_attn(q, k, v, want_lse=True)
    ctx.check()
    for b, c in enumerate(at):
        lost, e = out[b, :, 0], lse[b, 0]
        assert not torch.isfinite(lost).any(), (c, lost[torch.isfinite(lost)][:4])
        assert (torch.isnan(e) | (e == INF)).all(), (c, e[:4])
    mask = torch.ones(n_q, n_kv, dtype=torch.bool, device="cuda")
    base.compare(out[:, :, 1:], lse[:, 1:], q[:, :, 1:], lambda b, h: (k[b, :, 1].double(), v[b, :, 1].double(), mask), D, dt)


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


def test_joint_attention_passes_a_nan_key_on():
    """The joint attention of the same block, at every position of a key tile."""
    for D in (64, 128):
        B, L = 132, 8 + 2 * 64 + 8
        gen = torch.Generator(device="cuda").manual_seed(D)
        ctx = swam.Swam(B, 8, 2, 64, 8, 1, D, 14, 18, dtype=swam.BF16)
        q, k, v = (base.rand(gen, B, L, 1, D, dtype=torch.bfloat16) for _ in range(3))
        for b in range(B):
            k[b, b] = NAN
        out, lse = ctx.sparse_attn(q, k, v, want_lse=True)
        ctx.check()
        assert torch.isnan(out).all() and torch.isnan(lse).all()


@pytest.mark.parametrize("dtype,variant", base.VARIANTS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n_q", [100, 200])
@pytest.mark.parametrize("lowest", [-1, 1])
def test_the_types_lowest_value_behind_a_causal_limit(dtype, variant, D, n_q, lowest):
    """Values of the type's lowest (largest) number at keys that the first rows do not see: those rows know nothing of them."""
    dt, H, n_prefix, n_own, first = DT[dtype], 2, 50, n_q + 20, 64
    gen = torch.Generator(device="cuda").manual_seed(n_q + D)
    ctx = base.make_ctx(1, H, D, H, swam.F32 if dtype == "f32" else swam.BF16)
    ctx.set_option(swam.OPT_ATTN_VARIANT, variant)
    q = base.rand(gen, 1, n_q, H, D, dtype=dt)
    kp, vp = (base.rand(gen, 1, n_prefix, H, D, dtype=dt) for _ in range(2))
    k, v = (base.rand(gen, 1, n_own, H, D, dtype=dt) for _ in range(2))
    v[:, first:] = lowest * torch.finfo(dt).max
    out, lse = ctx.prefix_attn(q, kp, vp, k, v, causal=True, want_lse=True)
    ctx.check()
    rows = first - (n_own - n_q)                       # row t sees the own keys up to n_own - n_q + t
    t = torch.arange(rows, device="cuda")[:, None]
    mask = torch.ones(rows, n_prefix + first, dtype=torch.bool, device="cuda")
    mask[:, n_prefix:] = torch.arange(first, device="cuda")[None, :] <= n_own - n_q + t

    def segments(b, h):
        return (torch.cat([kp[0, :, h], k[0, :first, h]]).double(), torch.cat([vp[0, :, h], v[0, :first, h]]).double(), mask)
    base.compare(out[:, :rows], lse[:, :, :rows], q[:, :rows], segments, D, dt)


@pytest.mark.parametrize("dtype,variant", base.VARIANTS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n_q", [100, 200])
def test_the_types_lowest_value_at_keys_of_vanishing_weight(dtype, variant, D, n_q):
    """Keys whose weights are below 2^-140 in fact, with values of the type's lowest number: 2^-140 * 2^128 is nothing beside
    the tolerance, so the result is the mean over the other keys."""
    dt, H, n_kv = DT[dtype], 1, 256
    plan = (dtype, variant, n_q, H, H, D, n_kv)
    gen = torch.Generator(device="cuda").manual_seed(D)
    ctx = context(plan, 1)
    far = -256.0 * math.sqrt(D)                       # logits of 0 and -256: 2^-369
    q, k = one_component(plan, [[0.0 if c % 2 else far for c in range(n_kv)]])
    v = base.rand(gen, 1, n_kv, H, D, dtype=dt)
    v[:, ::2] = torch.finfo(dt).min
    out, lse = ctx.cross_attn(q, k, v, want_lse=True)
    ctx.check()
    keys, mask = k[0, 1::2, 0].double(), torch.ones(n_q, n_kv // 2, dtype=torch.bool, device="cuda")
    base.compare(out, lse, q, lambda b, h: (keys, v[0, 1::2, 0].double(), mask), D, dt)


@plans
@pytest.mark.parametrize("low,high", [(-1.5 * 2.0 ** 35, 3.0), (-1.25 * 2.0 ** 36, -1.125 * 2.0 ** 33), (2.0 ** 20, 1.625 * 2.0 ** 35),
                                      (-1.0 * 2.0 ** 35, -1.0 * 2.0 ** 20), (-INF, 2.0), (-INF, -1.75 * 2.0 ** 37),
                                      (-1.0 * 2.0 ** 146, 1.375 * 2.0 ** 60)])
def test_one_key_far_above_all_others(plan, low, high):
    """The weights are 1 and 0 (the logits lie at least 2^16 apart), wherever the one key stands: the result is its value, off by
    the rounding of a weight that need not be 1 (its reference may be any number near the logit), of the result and of the
    exponentials."""
    dtype, variant, n_q, H, kv, D, n_kv = plan
    dt, at = DT[dtype], positions(n_kv)
    B = len(at)
    gen = torch.Generator(device="cuda").manual_seed(n_q + D)
    ctx = context(plan, B)
    if low == -INF:
        low = -1.0 * 2.0 ** 146               # 2^20 * -2^126 overflows to -inf
    q, k = one_component(plan, [[high if c == x else low for c in range(n_kv)] for x in at])
    v = base.rand(gen, B, n_kv, kv, D, dtype=dt)
    out, lse = ctx.cross_attn(q, k, v, want_lse=True)
    ctx.check()
    want = torch.stack([v[b, c] for b, c in enumerate(at)])[:, None].double()
    tol = ((2.0 ** -17 + 8 * U32) + (U16 * (2 + U16) if dtype == "bf16" else 0.0)) * want.abs()
    assert ((out.double() - want).abs() <= tol).all(), [(c, out[b, 0, 0, :2].tolist(), want[b, 0, 0, :2].tolist())
                                                        for b, c in enumerate(at) if not torch.allclose(out[b].double(), want[b].expand_as(out[b]), atol=0.05)]
    logit = high / math.sqrt(D)
    assert ((lse.double() - logit).abs() <= 8 * U32 * abs(logit) + 2.0 ** -17).all()


@plans
@pytest.mark.parametrize("raw", [1.625 * 2.0 ** 35, -1.625 * 2.0 ** 35, 1.171875 * 2.0 ** 40, -1.0 * 2.0 ** 60, 1.328125 * 2.0 ** 100])
def test_equal_logits_of_any_size_weigh_the_same(plan, raw):
    """All logits alike, however large: the mean of the values.  Tolerance: N sums in fp32, the rounding of the weights and of
    the result."""
    dtype, variant, n_q, H, kv, D, n_kv = plan
    dt, B = DT[dtype], 2
    gen = torch.Generator(device="cuda").manual_seed(n_q + D)
    ctx = context(plan, B)
    q, k = one_component(plan, [[raw] * n_kv] * B)
    v = base.rand(gen, B, n_kv, kv, D, dtype=dt)
    lens = [n_kv, n_kv - 37]
    out, lse = ctx.cross_attn(q, k, v, kv_len=torch.tensor(lens, dtype=torch.int32, device="cuda"), want_lse=True)
    ctx.check()
    for b, n in enumerate(lens):
        want, A = v[b, :n].double().mean(0), v[b, :n].double().abs().mean(0)
        tol = (2.0 ** -17 + 2 * (n + 8) * U32) * A + (U16 * (A * (1 + U16) + want.abs() * (1 + 2 * U16)) if dtype == "bf16" else 0.0)
        assert ((out[b].double() - want).abs() <= tol).all(), (b, out[b, 0, 0, :3], want[0, :3])
        ref = raw / math.sqrt(D) + math.log(n)
        assert ((lse[b].double() - ref).abs() <= 8 * U32 * abs(ref) + 2.0 ** -17 + (n + 8) * U32).all()


@plans
def test_rows_of_nothing_but_minus_infinity(plan):
    """Logits that overflow to -inf throughout: no weight is above 0, zeros and -inf as for a row without keys."""
    dtype, variant, n_q, H, kv, D, n_kv = plan
    ctx = context(plan, 1)
    q, k = one_component(plan, [[-1.0 * 2.0 ** 146] * n_kv])
    v = base.rand(torch.Generator(device="cuda").manual_seed(1), 1, n_kv, kv, D, dtype=DT[dtype])
    out, lse = ctx.cross_attn(q, k, v, want_lse=True)
    ctx.check()
    assert (out == 0).all() and (lse == -INF).all()

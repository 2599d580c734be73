"""Cross attention and shared-prefix attention against their definition in 64 bits.

Tolerances follow from the arithmetic (u16 = 2^-8 and u32 = 2^-24 are half steps of bf16 and fp32 relative to the value).
With p the exact weights (sum 1), A = sum_c p_c |v_c| and S the largest sum of |scale q_d k_d| of a row:
 - a score is off by at most e = (D + 4) u32 S (D products and their sum, the scale in the log2 domain), a weight therefore by
   2 e relative (numerator and sum), plus 2^-17 for the approximate exponentials (2^-18 each in numerator and sum);
 - the sums over N keys add N u32 relative to A in fp32, and N u32 again in the sum of the weights;
 - bf16: each weight is rounded once (u16 of A) and the result once (u16 of |out|).
An output may be off by the sum of these, a log-sum-exp by e + 2^-17 + N u32 + 4 u32 |lse|."""
import ctypes
import math

import pytest
import torch

from paper_2609_38984_b200 import swam

U16, U32 = 2.0 ** -8, 2.0 ** -24
pytestmark = pytest.mark.gpu


def make_ctx(B, H, D, kv, dtype):
    return swam.Swam(B, 16, 2, 64, 8, H, D, 14, 18, n_kv_heads=kv, dtype=dtype)


def rand(gen, *shape, dtype, scale=1.0):
    return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(dtype)


def reference(q, keys, values, limits, scale):
    """One (sample, head): q [T, D], keys/values [C, D] in 64 bits, limits [T] lists of visible key indices as a mask.
    Returns out, lse, A, S."""
    x = (q @ keys.T) * scale
    x = x.masked_fill(~limits, -math.inf)
    lse = torch.logsumexp(x, dim=1) if keys.shape[0] else torch.full((q.shape[0],), -math.inf, dtype=torch.float64, device=q.device)
    p = torch.exp(x - torch.where(torch.isinf(lse), torch.zeros_like(lse), lse)[:, None])
    S = ((q.abs() @ keys.abs().T) * scale).masked_fill(~limits, 0.0)
    S = S.amax(dim=1) if keys.shape[0] else torch.zeros_like(lse)
    return p @ values, lse, p @ values.abs(), S


def compare(out, lse, q, segments, D, dtype):
    """segments(b, h) -> keys, values (64-bit, real ones only), mask [T, C]"""
    B, T, H, _ = q.shape
    scale = 1.0 / math.sqrt(D)
    f32 = dtype == torch.float32
    for b in range(B):
        for h in range(H):
            keys, values, mask = segments(b, h)
            ref, ref_lse, A, S = reference(q[b, :, h].double(), keys, values, mask, scale)
            N = keys.shape[0]
            e = (D + 4) * U32 * S + 2.0 ** -18
            tol = (2 * e + 2 * (N + 8) * U32)[:, None] * A + U32 * ref.abs()
            if not f32:
                tol = tol + U16 * (A * (1 + U16) + ref.abs() * (1 + 2 * U16))
            got = out[b, :, h].double()
            empty = ~mask.any(dim=1) if N else torch.ones(T, dtype=torch.bool, device=q.device)
            assert torch.isfinite(got).all(), (b, h)
            assert (got[empty] == 0).all(), (b, h)
            err = (got - ref).abs()
            assert (err <= tol + 1e-30).all(), (b, h, float((err - tol).max()), float((err / (tol + 1e-30)).max()))
            if lse is not None:
                gl = lse[b, h].double()
                assert (gl[empty] == -math.inf).all()
                ok = ~empty
                tl = e + (N + 8) * U32 + 4 * U32 * ref_lse.abs()
                assert ((gl - ref_lse).abs()[ok] <= tl[ok]).all(), (b, h, float(((gl - ref_lse).abs() - tl)[ok].max()))


def cross_case(dtype, B, n_q, H, kv, D, n_kv, lens, *, seed=0, scale=1.0, pad=float("nan"), interleaved=False, variant=None):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    ctx = make_ctx(B, H, D, kv, swam.F32 if dtype == torch.float32 else swam.BF16)
    if variant is not None:
        ctx.set_option(swam.OPT_ATTN_VARIANT, variant)
    q = rand(gen, B, n_q, H, D, dtype=dtype, scale=scale)
    if interleaved:
        kvt = rand(gen, B, n_kv, 2, kv, D, dtype=dtype)
        k, v = kvt[:, :, 0], kvt[:, :, 1]
    else:
        k, v = rand(gen, B, n_kv, kv, D, dtype=dtype), rand(gen, B, n_kv, kv, D, dtype=dtype)
    for b, n in enumerate(lens):
        k[b, n:] = pad
        v[b, n:] = pad
    kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
    out, lse = ctx.cross_attn(q, k, v, kv_len=kv_len, want_lse=True)
    ctx.check()
    g = H // kv

    def segments(b, h):
        n = lens[b]
        return k[b, :n, h // g].double(), v[b, :n, h // g].double(), torch.ones(n_q, n, dtype=torch.bool, device="cuda")
    compare(out, lse, q, segments, D, dtype)
    return ctx, q, k, v, kv_len, out, lse


def prefix_case(dtype, B, groups, n_q, H, kv, D, n_prefix, n_own, plens, olens, causal, *, seed=0, scale=1.0, pad=float("nan"),
                variant=None):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    ctx = make_ctx(B, H, D, kv, swam.F32 if dtype == torch.float32 else swam.BF16)
    if variant is not None:
        ctx.set_option(swam.OPT_ATTN_VARIANT, variant)
    q = rand(gen, B, n_q, H, D, dtype=dtype, scale=scale)
    kp, vp = (rand(gen, groups, n_prefix, kv, D, dtype=dtype) for _ in range(2))
    k, v = (rand(gen, B, n_own, kv, D, dtype=dtype) for _ in range(2))
    for i, n in enumerate(plens):
        kp[i, n:], vp[i, n:] = pad, pad
    for i, n in enumerate(olens):
        k[i, n:], v[i, n:] = pad, pad
    pl = torch.tensor(plens, dtype=torch.int32, device="cuda")
    ol = torch.tensor(olens, dtype=torch.int32, device="cuda")
    out, lse = ctx.prefix_attn(q, kp, vp, k, v, prefix_len=pl, own_len=ol, causal=causal, want_lse=True)
    ctx.check()
    g, per = H // kv, B // groups

    def segments(b, h):
        np_, no = plens[b // per], olens[b]
        keys = torch.cat([kp[b // per, :np_, h // g], k[b, :no, h // g]]).double()
        vals = torch.cat([vp[b // per, :np_, h // g], v[b, :no, h // g]]).double()
        mask = torch.ones(n_q, np_ + no, dtype=torch.bool, device="cuda")
        if causal:
            t = torch.arange(n_q, device="cuda")[:, None]
            mask[:, np_:] = torch.arange(no, device="cuda")[None, :] < no - n_q + t + 1
        return keys, vals, mask
    compare(out, lse, q, segments, D, dtype)
    return ctx, (q, kp, vp, k, v, pl, ol), out, lse


DT = {"bf16": torch.bfloat16, "f32": torch.float32}
VARIANTS = [("bf16", swam.ATTN_AUTO), ("bf16", swam.ATTN_WARP_MMA), ("f32", swam.ATTN_AUTO)]


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("dtype,variant", VARIANTS)
@pytest.mark.parametrize("n_q,H,kv", [(1, 4, 4), (1, 8, 2), (5, 6, 2), (33, 3, 3), (130, 4, 2), (300, 2, 1), (70, 20, 1)])
def test_cross_lengths(dtype, variant, D, n_q, H, kv):
    """Ragged lengths around the tile sizes, one key, no key (an empty row), NaN in every padded place."""
    n_kv = 300
    lens = [300, 0, 1, 63, 64, 65, 127, 128, 129, 255, 257]
    cross_case(DT[dtype], len(lens), n_q, H, kv, D, n_kv, lens, seed=n_q + D, variant=variant)


@pytest.mark.parametrize("dtype,variant", VARIANTS)
def test_cross_one_state_and_one_query(dtype, variant):
    cross_case(DT[dtype], 2, 1, 2, 1, 64, 1, [1, 0], variant=variant)
    cross_case(DT[dtype], 1, 1, 1, 1, 128, 1, [1], variant=variant)


@pytest.mark.parametrize("dtype,variant", VARIANTS)
@pytest.mark.parametrize("D", [64, 128])
def test_cross_long_keys_are_split_and_merged(dtype, variant, D):
    """Few rows and many keys: pieces over the keys, some of them without real keys."""
    cross_case(DT[dtype], 3, 2, 8, 4, D, 9000, [9000, 130, 4097], seed=3, variant=variant, interleaved=True)


@pytest.mark.parametrize("dtype,variant", VARIANTS)
@pytest.mark.parametrize("D", [64, 128])
def test_cross_growing_and_extreme_logits(dtype, variant, D):
    """Row maxima that grow from tile to tile (the running reference is raised again and again), and logits of several
    hundred, where all but a few weights vanish."""
    B, n_q, H, n_kv = 1, 150, 2, 1000
    gen = torch.Generator(device="cuda").manual_seed(9)
    dt = DT[dtype]
    ctx = make_ctx(B, H, D, H, swam.F32 if dt == torch.float32 else swam.BF16)
    ctx.set_option(swam.OPT_ATTN_VARIANT, variant)
    q = rand(gen, B, n_q, H, D, dtype=dt).abs() + 0.25
    k = rand(gen, B, n_kv, H, D, dtype=dt)
    k = (k + torch.arange(n_kv, device="cuda")[None, :, None, None] * (8.0 / n_kv)).to(dt)
    v = rand(gen, B, n_kv, H, D, dtype=dt)
    for sign in (1, -1):
        kk = k if sign == 1 else -k
        out, lse = ctx.cross_attn(q, kk, v, want_lse=True)
        ctx.check()
        compare(out, lse, q, lambda b, h: (kk[b, :, h].double(), v[b, :, h].double(),
                                           torch.ones(n_q, n_kv, dtype=torch.bool, device="cuda")), D, dt)


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("dtype,variant", VARIANTS)
@pytest.mark.parametrize("n_kv", [20, 77, 100, 128, 215])
def test_cross_logits_that_grow_inside_a_tile(dtype, variant, D, n_kv):
    """Every key outweighs the one before it by about a factor of two, so that weights of a tile are rescaled by later ones of
    the same tile, at every place where a tile may end."""
    B, n_q, H = 1, 150, 2
    gen = torch.Generator(device="cuda").manual_seed(10 + n_kv)
    dt = DT[dtype]
    ctx = make_ctx(B, H, D, H, swam.F32 if dt == torch.float32 else swam.BF16)
    ctx.set_option(swam.OPT_ATTN_VARIANT, variant)
    q = rand(gen, B, n_q, H, D, dtype=dt).abs() + 0.25
    k = (rand(gen, B, n_kv, H, D, dtype=dt) / 8 + torch.arange(n_kv, device="cuda")[None, :, None, None] / D ** 0.5).to(dt)
    v = rand(gen, B, n_kv, H, D, dtype=dt)
    lens = torch.tensor([n_kv - 3], dtype=torch.int32, device="cuda")
    for n, kv_len in ((n_kv, None), (n_kv - 3, lens)):
        out, lse = ctx.cross_attn(q, k, v, kv_len=kv_len, want_lse=True)
        ctx.check()
        compare(out, lse, q, lambda b, h: (k[b, :n, h].double(), v[b, :n, h].double(),
                                           torch.ones(n_q, n, dtype=torch.bool, device="cuda")), D, dt)


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("dtype,variant", VARIANTS)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("n_q,H,kv", [(1, 8, 2), (1, 4, 4), (7, 6, 2), (40, 4, 2), (140, 2, 2), (9, 20, 1)])
def test_prefix_lengths(dtype, variant, D, causal, n_q, H, kv):
    """Groups with ragged prefixes (one of them empty) and ragged own keys: none, fewer than queries, tile borders."""
    B, groups = 8, 2
    prefix_case(DT[dtype], B, groups, n_q, H, kv, D, 200, 150, [197, 0], [150, 0, 1, 64, 128, 129, 3, 0], causal, seed=D + n_q,
                variant=variant)


@pytest.mark.parametrize("dtype,variant", VARIANTS)
@pytest.mark.parametrize("groups", [1, 3])
def test_prefix_long_shared_history(dtype, variant, groups):
    prefix_case(DT[dtype], 3 * 7, groups, 1, 8, 2, 128, 5000, 700, [5000, 4100, 257][:groups],
                [(37 * i) % 701 for i in range(21)], False, seed=4, variant=variant)


@pytest.mark.parametrize("dtype,variant", VARIANTS)
def test_prefix_without_prefix_or_without_own_keys(dtype, variant):
    dt = DT[dtype]
    prefix_case(dt, 4, 1, 3, 4, 2, 64, 0, 50, [0], [50, 0, 2, 13], True, variant=variant)
    prefix_case(dt, 4, 2, 3, 4, 2, 64, 90, 0, [90, 33], [0, 0, 0, 0], False, variant=variant)
    prefix_case(dt, 2, 1, 3, 4, 2, 64, 0, 0, [0], [0, 0], False, variant=variant)
    prefix_case(dt, 3, 3, 200, 2, 2, 64, 0, 300, [0, 0, 0], [300, 200, 17], True, variant=variant)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n_q", [100, 128, 300])
@pytest.mark.parametrize("longest", [100, 300, 700])
def test_many_short_samples(D, n_q, longest):
    """Several work items per SM with one, two, three, ... key tiles and none, in every order."""
    B = 100
    gen = torch.Generator().manual_seed(longest)
    lens = [int(x) for x in torch.randint(0, longest + 1, (B,), generator=gen)]
    cross_case(torch.bfloat16, B, n_q, 8, 8, D, longest, lens, seed=longest)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n_q", [100, 300])
def test_many_samples_without_keys_between_others(D, n_q):
    """Long rows of work items without keys before, between and behind items with them (more items than SMs, so that one
    CTA meets them in every order)."""
    B = 120
    lens = [130 if b % 29 == 7 else 0 for b in range(B)]
    lens[-1] = 300
    cross_case(torch.bfloat16, B, n_q, 8, 8, D, 300, lens, seed=11)
    lens = [300 if b < 40 else 0 for b in range(B)]
    cross_case(torch.bfloat16, B, n_q, 4, 4, D, 300, lens, seed=12)
    cross_case(torch.bfloat16, B, n_q, 4, 4, D, 300, [0] * B, seed=13)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_q", [3, 300])
def test_strided_views_and_untouched_rows(dtype, n_q):
    """Sequence-first layouts and slices of wider tensors, read and written in place; everything around them stays."""
    dt = DT[dtype]
    B, H, kv, D, n_kv = 3, 4, 2, 64, 150
    gen = torch.Generator(device="cuda").manual_seed(1)
    ctx = make_ctx(B, H, D, kv, swam.F32 if dt == torch.float32 else swam.BF16)
    qkv = rand(gen, n_q, B, H + 2, D, dtype=dt)                 # token-major, a wider projection
    q = qkv[:, :, 1:1 + H].transpose(0, 1)
    k, v = (rand(gen, B, n_kv + 9, kv, D, dtype=dt)[:, 4:4 + n_kv] for _ in range(2))
    big = torch.full((B + 1, n_q + 5, H + 1, D), 7.0, dtype=dt, device="cuda")
    out = big[1:, 2:2 + n_q, :H]
    lens = torch.tensor([150, 77, 0], dtype=torch.int32, device="cuda")
    want, lse = ctx.cross_attn(q.contiguous(), k.contiguous(), v.contiguous(), kv_len=lens, want_lse=True)
    got, lse2 = ctx.cross_attn(q, k, v, kv_len=lens, out=out, want_lse=True)
    ctx.check()
    assert torch.equal(got, want) and torch.equal(lse, lse2)
    mask = torch.ones_like(big, dtype=torch.bool)
    mask[1:, 2:2 + n_q, :H] = False
    assert (big[mask] == 7.0).all()
    # the last two samples' prefix: the same views as own keys
    p1 = ctx.prefix_attn(q, k[:1], v[:1], k, v, own_len=lens, out=out, causal=True).clone()
    p2 = ctx.prefix_attn(q.contiguous(), k[:1].contiguous(), v[:1].contiguous(), k.contiguous(), v.contiguous(), own_len=lens, causal=True)
    ctx.check()
    assert torch.equal(p1, p2) and (big[mask] == 7.0).all()


def test_offsets_beyond_32_bits():
    """Keys of the second sample start more than 2^32 elements behind the first one's, and rows of one sample pass 2^31."""
    B, H, D, n_kv = 2, 2, 64, 600
    ctx = make_ctx(B, H, D, H, swam.BF16)
    gen = torch.Generator(device="cuda").manual_seed(2)
    tok = 1 << 23                                               # elements between two tokens: 600 tokens span 5e9 elements
    buf = torch.empty(n_kv * tok + 4096, dtype=torch.bfloat16, device="cuda")
    k = buf.as_strided((B, n_kv, H, D), (H * D, tok, D, 1))
    v = buf.as_strided((B, n_kv, H, D), (H * D, tok, D, 1), 1024)
    k.copy_(rand(gen, B, n_kv, H, D, dtype=torch.bfloat16))
    v.copy_(rand(gen, B, n_kv, H, D, dtype=torch.bfloat16))
    for n_q in (1, 200):
        q = rand(gen, B, n_q, H, D, dtype=torch.bfloat16)
        want, l1 = ctx.cross_attn(q, k.contiguous(), v.contiguous(), want_lse=True)
        got, l2 = ctx.cross_attn(q, k, v, want_lse=True)
        ctx.check()
        assert torch.equal(want, got) and torch.equal(l1, l2)
    far = torch.empty((1 << 32) + 2 * n_kv * H * D, dtype=torch.bfloat16, device="cuda")
    k2 = far.as_strided((B, n_kv, H, D), (1 << 32, H * D, D, 1))
    k2.copy_(k)
    for n_q in (1, 200):
        q = rand(gen, B, n_q, H, D, dtype=torch.bfloat16)
        assert torch.equal(ctx.cross_attn(q, k2, v), ctx.cross_attn(q, k.contiguous(), v.contiguous()))
    ctx.check()


def test_bad_lengths_are_clamped_and_reported():
    gen = torch.Generator(device="cuda").manual_seed(5)
    for dt, n_q in ((torch.bfloat16, 3), (torch.bfloat16, 200), (torch.float32, 3)):
        ctx = make_ctx(2, 2, 64, 2, swam.F32 if dt == torch.float32 else swam.BF16)
        q, k, v = rand(gen, 2, n_q, 2, 64, dtype=dt), rand(gen, 2, 40, 2, 64, dtype=dt), rand(gen, 2, 40, 2, 64, dtype=dt)
        out, lse = ctx.cross_attn(q, k, v, kv_len=torch.tensor([41, -3], dtype=torch.int32, device="cuda"), want_lse=True)
        with pytest.raises(swam.SwamError) as e:
            ctx.check()
        assert e.value.code == swam.ERR_DEVICE_CHECK and "length" in str(e.value)
        want, lse_w = ctx.cross_attn(q, k, v, kv_len=torch.tensor([40, 0], dtype=torch.int32, device="cuda"), want_lse=True)
        ctx.check()
        assert torch.equal(out, want) and torch.equal(lse, lse_w)


def test_refusals():
    ctx = make_ctx(4, 4, 64, 2, swam.BF16)
    q = torch.zeros(4, 3, 4, 64, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(4, 10, 2, 64, dtype=torch.bfloat16, device="cuda")
    ok_len = torch.full((4,), 10, dtype=torch.int32, device="cuda")
    before = ctx.launch_count()
    for bad in (dict(q=q[:3]), dict(q=q.float()), dict(k=k[:, :5]), dict(k=k[:, :, :, ::2]), dict(q=q.cpu()),
                dict(kv_len=ok_len[:3]), dict(kv_len=ok_len.long()), dict(kv_len=ok_len.cpu()), dict(q=q[0]),
                dict(k=k[:1].expand(4, 10, 2, 64), v=k[:1].expand(4, 10, 2, 64)), dict(out=q[:, :2]), dict(v=k[:, :, :1])):
        args = dict(q=q, k=k, v=k, kv_len=ok_len)
        args.update(bad)
        with pytest.raises(ValueError):
            ctx.cross_attn(**args)
    three = torch.zeros(4, 10, 3, 64, dtype=torch.bfloat16, device="cuda")      # 3 heads do not divide 4
    with pytest.raises(swam.SwamError) as e:
        ctx.cross_attn(q, three, three)
    assert e.value.code == swam.ERR_INVALID_ARG
    kp = torch.zeros(3, 10, 2, 64, dtype=torch.bfloat16, device="cuda")         # 3 groups do not divide 4 samples
    with pytest.raises(swam.SwamError) as e:
        ctx.prefix_attn(q, kp, kp, k, k)
    assert e.value.code == swam.ERR_INVALID_ARG

    a = swam.SwamCrossArgs()
    st = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)

    def fill(**kw):
        nonlocal a
        a = swam.SwamCrossArgs(q=q.data_ptr(), k=k.data_ptr(), v=k.data_ptr(), out=q.data_ptr() + (1 << 20), n_q=3, n_kv=10)
        for n, x in kw.items():
            setattr(a, n, x)
        return ctx.lib.swam_cross_attn(ctx.ctx, ctypes.byref(a), st)
    inv, uns = swam.ERR_INVALID_ARG, swam.ERR_UNSUPPORTED
    for rc, kw in ((inv, dict(q=None)), (inv, dict(out=None)), (inv, dict(k=None)), (inv, dict(v=None)), (inv, dict(q=q.data_ptr() + 2)),
                   (inv, dict(k=k.data_ptr() + 8)), (inv, dict(lse=q.data_ptr() + 2)), (inv, dict(kv_len=ok_len.data_ptr() + 1)), (inv, dict(n_q=-1)), (inv, dict(n_kv=-1)), (inv, dict(n_kv_heads=3)),
                   (inv, dict(n_kv_heads=-2)), (inv, dict(reserved=1)), (inv, dict(q_token=-256)), (inv, dict(q_token=100)),
                   (inv, dict(q_token=260)), (inv, dict(k_token=64)), (inv, dict(k_token=1 << 41)), (inv, dict(out_sample=256)),
                   (uns, dict(n_kv=(1 << 30) + 1)), (uns, dict(n_q=1 << 29))):
        assert fill(**kw) == rc, kw
    assert ctx.lib.swam_cross_attn(ctx.ctx, None, st) == inv
    assert ctx.lib.swam_prefix_attn(ctx.ctx, None, st) == inv
    n = ctypes.c_size_t()
    assert ctx.lib.swam_cross_attn_scratch_bytes(ctx.ctx, ctypes.byref(a), None) == inv
    # scratch that is missing or too small
    long = torch.zeros(4, 9000, 2, 64, dtype=torch.bfloat16, device="cuda")
    assert fill(k=long.data_ptr(), v=long.data_ptr(), n_kv=9000) == swam.ERR_WORKSPACE
    assert ctx.lib.swam_cross_attn_scratch_bytes(ctx.ctx, ctypes.byref(a), ctypes.byref(n)) == swam.OK and n.value > 0
    small = torch.empty(n.value + 512, dtype=torch.uint8, device="cuda")
    base = (small.data_ptr() + 255) // 256 * 256
    assert fill(k=long.data_ptr(), v=long.data_ptr(), n_kv=9000, scratch=base, scratch_bytes=n.value - 1) == swam.ERR_WORKSPACE
    assert fill(k=long.data_ptr(), v=long.data_ptr(), n_kv=9000, scratch=base + 16, scratch_bytes=n.value) == swam.ERR_WORKSPACE
    assert ctx.launch_count() == before
    ctx.check()
    unbound = swam.Swam(4, 16, 2, 64, 8, 4, 64, 14, 18, n_kv_heads=2, bind=False)
    with pytest.raises(swam.SwamError) as e:
        unbound.cross_attn(q, k, k)
    assert e.value.code == swam.ERR_WORKSPACE


def test_zero_queries_and_zero_states():
    ctx = make_ctx(2, 4, 64, 2, swam.BF16)
    k = torch.zeros(2, 10, 2, 64, dtype=torch.bfloat16, device="cuda")
    q0 = torch.zeros(2, 0, 4, 64, dtype=torch.bfloat16, device="cuda")
    out, lse = ctx.cross_attn(q0, k, k, want_lse=True)
    assert out.shape == (2, 0, 4, 64) and lse.shape == (2, 4, 0)
    for n_q in (1, 200):
        q = torch.ones(2, n_q, 4, 64, dtype=torch.bfloat16, device="cuda")
        out, lse = ctx.cross_attn(q, k[:, :0], k[:, :0], want_lse=True)
        ctx.check()
        assert (out == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("n_q", [1, 150])
def test_repeats_graphs_and_streams_give_the_same_bits(n_q):
    """Repeated calls, two captured graphs replayed on two streams at once, and a call on a side stream."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    B, H, kv, D = 6, 8, 2, 128
    ctx = make_ctx(B, H, D, kv, swam.BF16)
    bf = torch.bfloat16
    q, kp, vp = rand(gen, B, n_q, H, D, dtype=bf), rand(gen, 2, 3000, kv, D, dtype=bf), rand(gen, 2, 3000, kv, D, dtype=bf)
    k, v = rand(gen, B, 400, kv, D, dtype=bf), rand(gen, B, 400, kv, D, dtype=bf)
    own = torch.tensor([400, 0, 17, 399, 128, 256], dtype=torch.int32, device="cuda")
    pre = lambda x: ctx.prefix_attn(x, kp, vp, k, v, own_len=own, want_lse=True)
    cro = lambda x: ctx.cross_attn(x, k, v, kv_len=own, want_lse=True)
    want_p, want_c = pre(q), cro(q)
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(pre(q), want_p)) and all(torch.equal(a, b) for a, b in zip(cro(q), want_c))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = pre(q)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want_p))
    torch.cuda.synchronize()
    qs = torch.zeros_like(q)
    g1, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g1):
        o1 = pre(qs)
    with torch.cuda.graph(g2):
        o2 = cro(qs)
    qs.copy_(q)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(10):
        with torch.cuda.stream(s1):
            g1.replay()
        with torch.cuda.stream(s2):
            g2.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(o1, want_p)) and all(torch.equal(a, b) for a, b in zip(o2, want_c))
    ctx.check()


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("bf16", 128), ("f32", 32)])
def test_block_of_candidates_shares_its_observation(dtype, D):
    """The operators as they are used together: B candidates of one observation.  With observed rows that see the observed
    tokens only, the observed keys are the same for every candidate, and joint attention of a candidate's future and
    action rows is prefix attention; the block's cross attention to a padded text follows on its result."""
    dt = DT[dtype]
    B, n_obs, F, N_s, A, H, kv = 3, 150, 2, 40, 8, 4, 2
    n_own = F * N_s + A
    L = n_obs + n_own
    gen = torch.Generator(device="cuda").manual_seed(8)
    ctx = swam.Swam(B, n_obs, F, N_s, A, H, D, 10, 10, n_kv_heads=kv, dtype=swam.F32 if dt == torch.float32 else swam.BF16)
    ctx.set_visibility(swam.SEES_OBSERVED, swam.SEES_ALL, swam.SEES_ALL)
    q = rand(gen, B, L, H, D, dtype=dt)
    k, v = rand(gen, B, L, kv, D, dtype=dt), rand(gen, B, L, kv, D, dtype=dt)
    for x in (q, k, v):
        x[:, :n_obs] = x[:1, :n_obs]
    joint, joint_lse = ctx.sparse_attn(q, k, v, want_lse=True)
    own, own_lse = ctx.prefix_attn(q[:, n_obs:], k[:1, :n_obs], v[:1, :n_obs], k[:, n_obs:], v[:, n_obs:], want_lse=True)
    ctx.check()
    g = H // kv
    seen = torch.ones(n_own, L, dtype=torch.bool, device="cuda")
    full = lambda b, h: (k[b, :, h // g].double(), v[b, :, h // g].double(), seen)
    compare(own, own_lse, q[:, n_obs:], full, D, dt)
    compare(joint[:, n_obs:], joint_lse[:, :, n_obs:], q[:, n_obs:], full, D, dt)
    # cross attention of all rows of the block: the observed rows from the joint call, the rest from the prefix call
    rows = torch.cat([joint[:, :n_obs], own], dim=1)
    tk, tv = rand(gen, B, 77, H, D, dtype=dt), rand(gen, B, 77, H, D, dtype=dt)
    lens = [77, 0, 20]
    out, lse = ctx.cross_attn(rows, tk, tv, kv_len=torch.tensor(lens, dtype=torch.int32, device="cuda"), want_lse=True)
    ctx.check()
    compare(out, lse, rows, lambda b, h: (tk[b, :lens[b], h].double(), tv[b, :lens[b], h].double(),
                                          torch.ones(L, lens[b], dtype=torch.bool, device="cuda")), D, dt)

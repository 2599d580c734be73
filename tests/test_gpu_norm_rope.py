"""Head norms with rotary positions, and appending to a paged cache, against their definition in 64 bits.

Tolerances (u = 2^-24, half a step of fp32 relative to the value; h the half step of the storage type, 2^-8 or 2^-24):
 - the sum of D <= 128 squares (at most 8 + 5 additions deep, a rounding each, and the fused products), its mean with eps and the
   reciprocal root (2 steps = 4 u): below 16 u / 2 + 4 u = 12 u relative; times the weight and the element 2 u: 14 u;
 - a cosine or sine: the angle, at most pi / 4 = 0.79, is off by 2 u of itself (its conversion and the constant), 1.6 u absolute;
   the polynomial's last additions 2 u, the magnitude u: below 5 u of the magnitude;
 - the product and the fused sum 2 u.
A rotated element is off by (14 + 5 + 2) u magnitude (|a| + |b|) at most, an unrotated one by 14 u |a|, and then rounded: h of the value.
The tests allow 24 u magnitude (|a| + |b|) + 1.01 h |value|."""
import ctypes
import math

import pytest
import torch

import test_gpu_segment_attn as base
from paper_2609_38984_b200 import swam

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32
TYPES = [BF16, F32]


def definition(x, weight, eps, freq, axis, interleaved, magnitude, positions):
    """x [..., heads, D]; positions [..., axes] (None: no rotation) -> result and |a| + |b| of each element, in 64 bits."""
    y = x.double()
    if weight is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * weight.double()
    size = y.abs().clone()
    if positions is None:
        return y, size
    half = len(freq)
    angle = (positions.double()[..., axis] * torch.tensor(freq, dtype=torch.float64, device=x.device))[..., None, :]
    i = torch.arange(half, device=x.device)
    ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    a, b = y[..., ia], y[..., ib]
    out = y.clone()
    out[..., ia] = magnitude * (a * angle.cos() - b * angle.sin())
    out[..., ib] = magnitude * (b * angle.cos() + a * angle.sin())
    size[..., ia] = size[..., ib] = (a.abs() + b.abs()) * max(1.0, magnitude)
    return out, size


def close(got, want, size, dtype):
    h = 2.0 ** -8 if dtype == BF16 else U
    tol = 24 * U * size + 1.01 * h * want.abs() + 1e-37
    err = (got.double() - want).abs()
    assert (err <= tol).all(), (float((err / tol).max()), int((err > tol).sum()))


def ladder(rot, base_=10000.0):
    return [base_ ** (-2 * i / rot) for i in range(rot // 2)]


def ctx_for(B, H, kv, D, dtype):
    return base.make_ctx(B, H, D, kv, swam.F32 if dtype == F32 else swam.BF16)


def weights(gen, D):
    return [1 + 0.3 * torch.randn(D, generator=gen, device="cuda") for _ in range(2)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D,rot", [(32, 32), (32, 8), (32, 24), (32, 2), (64, 64), (64, 32), (64, 56), (128, 128), (128, 64), (128, 32),
                                   (128, 120), (128, 6)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_layouts(dtype, D, rot, interleaved, norm):
    B, n, H, kv = 2, 5, 6, 2
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k = (base.rand(gen, B, n, h, D, dtype=dtype, scale=3.0) for h in (H, kv))
    qw, kw = weights(gen, D) if norm else (None, None)
    rope = swam.Rope(ladder(rot), interleaved=interleaved, magnitude=1.25)
    pos = torch.randint(-1000, 100000, (B, n), generator=gen, device="cuda", dtype=torch.int32)
    ctx = ctx_for(B, H, kv, D, dtype)
    q2, k2 = ctx.norm_rope(q, k, rope, positions=pos, q_weight=qw, k_weight=kw, eps=1e-5)
    ctx.check()
    for got, x, w in ((q2, q, qw), (k2, k, kw)):
        close(got, *definition(x, w, 1e-5, ladder(rot), [0] * (rot // 2), interleaved, 1.25, pos[..., None]), dtype)
        if not norm:
            assert torch.equal(got[..., rot:], x[..., rot:])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,kv", [(1, 1), (24, 24), (32, 8), (15, 5), (33, 3)])
@pytest.mark.parametrize("n", [1, 3, 200])
def test_heads_and_lengths(dtype, H, kv, n):
    """One warp for a token's rows, and several; the default positions."""
    B, D = 3, 64
    gen = torch.Generator(device="cuda").manual_seed(2)
    q, k = (base.rand(gen, B, n, h, D, dtype=dtype) for h in (H, kv))
    qw, kw = weights(gen, D)
    ctx = ctx_for(B, H, kv, D, dtype)
    pos = torch.arange(n, device="cuda").expand(B, n)[..., None]
    q2, k2 = ctx.norm_rope(q, k, swam.Rope(ladder(D)), q_weight=qw, k_weight=kw)
    for got, x, w in ((q2, q, qw), (k2, k, kw)):
        close(got, *definition(x, w, 1e-6, ladder(D), [0] * (D // 2), False, 1.0, pos), dtype)
    # each alone, only normalised, only rotated, and nothing at all
    only_q, none = ctx.norm_rope(q, rope=swam.Rope(ladder(D)), q_weight=qw)
    assert none is None and torch.equal(only_q, q2)
    none, only_k = ctx.norm_rope(k=k, rope=swam.Rope(ladder(D)), k_weight=kw)
    assert none is None and torch.equal(only_k, k2)
    normed, plain = ctx.norm_rope(q, k, q_weight=qw)
    close(normed, *definition(q, qw, 1e-6, [], [], False, 1.0, None), dtype)
    assert torch.equal(plain, k)
    ctx.check()


@pytest.mark.parametrize("dtype", TYPES)
def test_many_tokens(dtype):
    B, n, H, kv, D = 2, 6001, 4, 4, 128
    gen = torch.Generator(device="cuda").manual_seed(3)
    q, k = (base.rand(gen, B, n, h, D, dtype=dtype) for h in (H, kv))
    qw, kw = weights(gen, D)
    ctx = ctx_for(B, H, kv, D, dtype)
    pos = torch.arange(n, device="cuda").expand(B, n)[..., None]
    q2, k2 = ctx.norm_rope(q, k, swam.Rope(ladder(D), interleaved=True), q_weight=qw, k_weight=kw)
    for got, x, w in ((q2, q, qw), (k2, k, kw)):
        close(got, *definition(x, w, 1e-6, ladder(D), [0] * (D // 2), True, 1.0, pos), dtype)


@pytest.mark.parametrize("interleaved", [False, True])
def test_angles_of_any_position(interleaved):
    """Positions up to the ends of int32 and frequencies far above a turn: the reduced angle is exact, the definition's own (64 bits, up
    to 2^31 radians times a step of 2^-52) is what limits the comparison for frequencies up to 1."""
    D = 64
    freq = [1.0, 0.999, -0.7, 0.5, 2.0 ** -10, 3e-7, 1e-30, 0.0] * 4
    pos = torch.tensor([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 10 ** 9, 131072, 65537], dtype=torch.int32, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(4)
    q = base.rand(gen, 1, 8, 2, D, dtype=F32)
    ctx = ctx_for(1, 2, 2, D, F32)
    got, _ = ctx.norm_rope(q, rope=swam.Rope(freq, interleaved=interleaved), positions=pos)
    want, size = definition(q, None, 0, freq, [0] * 32, interleaved, 1.0, pos[None, :, None])
    # a frequency is half a step of 64 bits off in either form, the definition's product once more: 2^31 * 2^-52 radians
    err, tol = (got.double() - want).abs(), (24 * U + 2.0 ** -21) * size + 1.01 * U * want.abs()
    assert (err <= tol).all(), float((err / tol).max())
    # whole numbers of eighths of a turn: a position times 2 pi / 8, to the step of that double
    eighth = [2 * math.pi / 8] * 32
    got, _ = ctx.norm_rope(q, rope=swam.Rope(eighth, interleaved=interleaved), positions=torch.arange(8, dtype=torch.int32, device="cuda"))
    close(got, *definition(q, None, 0, eighth, [0] * 32, interleaved, 1.0, torch.arange(8, device="cuda")[None, :, None]), F32)
    # a frequency and the same one plus a turn differ by what the sum's double can hold
    a, _ = ctx.norm_rope(q, rope=swam.Rope([1e6] * 32, interleaved=interleaved), positions=torch.ones(8, dtype=torch.int32, device="cuda"))
    want, size = definition(q, None, 0, [math.fmod(1e6, 2 * math.pi)] * 32, [0] * 32, interleaved, 1.0, torch.ones(1, 8, 1, device="cuda"))
    # (fmod takes off 159154 times the double nearest 2 pi, each 2.5e-16 from a turn: 4e-11 in all)
    assert ((a.double() - want).abs() <= (24 * U + 1e-10) * size + 1.01 * U * want.abs()).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_three_axes_and_shared_positions(dtype):
    B, n, H, kv, D = 2, 40, 4, 2, 128
    gen = torch.Generator(device="cuda").manual_seed(5)
    q, k = (base.rand(gen, B, n, h, D, dtype=dtype) for h in (H, kv))
    axis = [0] * 16 + [1] * 24 + [2] * 24
    freq = ladder(32) + ladder(48) + ladder(48)
    rope = swam.Rope(freq, axes=axis)
    shared = torch.randint(0, 300, (n, 3), generator=gen, device="cuda", dtype=torch.int32)
    ctx = ctx_for(B, H, kv, D, dtype)
    one = ctx.norm_rope(q, k, rope, positions=shared)
    each = ctx.norm_rope(q, k, rope, positions=shared.expand(B, n, 3).contiguous())
    for a, b, x in zip(one, each, (q, k)):
        assert torch.equal(a, b)
        close(a, *definition(x, None, 0, freq, axis, False, 1.0, shared.expand(B, n, 3)), dtype)
    # the default position is the token's number on every axis
    t = torch.arange(n, device="cuda", dtype=torch.int32)[:, None].expand(n, 3).contiguous()
    for a, b in zip(ctx.norm_rope(q, k, rope), ctx.norm_rope(q, k, rope, positions=t)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rot,interleaved", [(64, False), (56, False), (56, True)])
def test_views_and_in_place(dtype, rot, interleaved):
    """q and k inside a fused projection, rotated where they lie: same bits as out of place, the rest of the buffer untouched."""
    B, n, H, kv, D = 2, 70, 4, 2, 64
    gen = torch.Generator(device="cuda").manual_seed(6)
    qkv = base.rand(gen, B, n, H + 2 * kv, D, dtype=dtype)
    before = qkv.clone()
    q, k = qkv[:, :, :H], qkv[:, :, H:H + kv]
    qw, kw = weights(gen, D)
    ctx = ctx_for(B, H, kv, D, dtype)
    rope = swam.Rope(ladder(rot), interleaved=interleaved)
    q2, k2 = ctx.norm_rope(q, k, rope, q_weight=qw, k_weight=kw)
    assert torch.equal(qkv, before)
    close(q2, *definition(q, qw, 1e-6, ladder(rot), [0] * (rot // 2), interleaved, 1.0, torch.arange(n, device="cuda").expand(B, n)[..., None]), dtype)
    r = ctx.norm_rope(q, k, rope, q_weight=qw, k_weight=kw, q_out=q, k_out=k)
    assert r[0] is q and torch.equal(q, q2) and torch.equal(k, k2)
    assert torch.equal(qkv[:, :, H + kv:], before[:, :, H + kv:])


def test_special_values():
    """A row of zeros stays zero under a norm; NaN and infinities stay in their row; the smallest and largest numbers."""
    D = 64
    ctx = ctx_for(1, 4, 4, D, F32)
    q = torch.randn(1, 2, 4, D, device="cuda")
    q[0, 0, 0] = 0
    q[0, 0, 1, 5] = float("nan")
    q[0, 0, 2, 40] = float("inf")
    w = torch.ones(D, device="cuda")
    for weight in (None, w):
        got, _ = ctx.norm_rope(q, rope=swam.Rope(ladder(32)), q_weight=weight)
        assert (got[0, 0, 0] == 0).all()
        assert torch.isfinite(got[0, 0, 3]).all() and torch.isfinite(got[0, 1]).all()
        # the NaN's pair is lost, the rest of the row only with a norm; behind the rotated part an infinity is itself
        assert torch.isnan(got[0, 0, 1, [5, 21]]).all() and bool(torch.isnan(got[0, 0, 1]).all()) == (weight is not None)
        if weight is None:
            assert got[0, 0, 2, 40] == float("inf") and torch.isfinite(got[0, 0, 2, :40]).all()
    tiny, _ = ctx.norm_rope(torch.full((1, 1, 4, D), 1e-30, device="cuda"), q_weight=w, eps=0.0)
    assert not torch.isnan(tiny).any()            # the squares vanish: 1 / 0 times 1e-30
    ctx.check()


# ---------------------------------------------------------------------------------------------------------------------- the cache
class Cache:
    def __init__(self, dtype, samples, capacity, kv, D, page, seed=0, interleaved=False):
        host = torch.Generator().manual_seed(seed)
        per = (capacity + page - 1) // page
        n = samples * per + 3
        if interleaved:
            both = torch.full((n, page, 2, kv, D), 9.0, device="cuda").to(dtype)
            self.k, self.v = both[:, :, 0], both[:, :, 1]
        else:
            self.k, self.v = (torch.full((n, page, kv, D), 9.0, device="cuda").to(dtype) for _ in range(2))
        self.table = torch.randperm(n, generator=host, dtype=torch.int32)[:samples * per].reshape(samples, per).cuda()
        self.page = page

    def rows(self, pages, b, first, n):
        at = torch.arange(first, first + n, device="cuda")
        return pages[self.table[b].long()[at // self.page], at % self.page]


def append_case(dtype, new, past, H, kv, D, page, rot, interleaved, norm, with_q=True, front=0, behind=0, explicit=False, views=False):
    gen = torch.Generator(device="cuda").manual_seed(7)
    total = front + sum(new) + behind
    cache = Cache(dtype, len(new), max(a + b for a, b in zip(new, past)) or 1, kv, D, page, interleaved=views)
    if views:
        qkv = base.rand(gen, total, H + 2 * kv, D, dtype=dtype)
        q, k, v = qkv[:, :H], qkv[:, H:H + kv], qkv[:, H + kv:]
    else:
        q, k, v = (base.rand(gen, total, h, D, dtype=dtype) for h in (H, kv, kv))
    qw, kw = weights(gen, D) if norm else (None, None)
    starts = [front]
    for n in new:
        starts.append(starts[-1] + n)
    q_start = torch.tensor(starts, dtype=torch.int32, device="cuda")
    kv_len = torch.tensor([a + b for a, b in zip(new, past)], dtype=torch.int32, device="cuda")
    rope = swam.Rope(ladder(rot), interleaved=interleaved) if rot else None
    positions = torch.randint(0, 50000, (total,), generator=gen, device="cuda", dtype=torch.int32) if explicit else None
    q_out = torch.full((total, H, D), 9.0, device="cuda").to(dtype) if with_q else None
    ctx = ctx_for(1, H, kv, D, dtype)
    equal = front == behind == 0 and len(set(new)) == 1
    got = ctx.append_kv(k, v, cache.k, cache.v, cache.table, kv_len, q_start=None if equal else q_start, q=q if with_q else None, rope=rope,
                        positions=positions, q_weight=qw if with_q else None, k_weight=kw, q_out=q_out)
    ctx.check()
    assert got is q_out
    seen = torch.zeros(cache.k.shape[:2], dtype=torch.bool, device="cuda")
    for b, n in enumerate(new):
        if n == 0:
            continue
        s = slice(starts[b], starts[b] + n)
        pos = (positions[s] if explicit else torch.arange(past[b], past[b] + n, device="cuda"))[:, None] if rot else None
        close(cache.rows(cache.k, b, past[b], n), *definition(k[s], kw, 1e-6, ladder(rot) if rot else [], [0] * (rot // 2), interleaved, 1.0, pos), dtype)
        assert torch.equal(cache.rows(cache.v, b, past[b], n), v[s])
        if with_q:
            close(got[s], *definition(q[s], qw, 1e-6, ladder(rot) if rot else [], [0] * (rot // 2), interleaved, 1.0, pos), dtype)
        at = torch.arange(past[b], past[b] + n, device="cuda")
        seen[cache.table[b].long()[at // page], at % page] = True
    # nothing else was written
    assert (cache.k[~seen] == 9).all() and (cache.v[~seen] == 9).all()
    if with_q:
        assert (got[:front] == 9).all() and (got[front + sum(new):] == 9).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("new,past", [([1], [0]), ([1] * 40, [b * 13 for b in range(40)]), ([5, 0, 33, 1], [0, 7, 15, 200]),
                                      ([700, 300], [31, 0]), ([2, 2, 2], [15, 16, 17])])
@pytest.mark.parametrize("H,kv,D,page", [(8, 2, 64, 16), (5, 5, 32, 64), (4, 1, 128, 256)])
def test_append(dtype, new, past, H, kv, D, page):
    append_case(dtype, new, past, H, kv, D, page, D, False, True)
    append_case(dtype, new, past, H, kv, D, page, D - 8, True, False, with_q=False)


@pytest.mark.parametrize("dtype", TYPES)
def test_append_forms(dtype):
    append_case(dtype, [3, 4, 50], [1, 100, 40], 4, 2, 64, 32, 0, False, True)                    # no rotation
    append_case(dtype, [3, 4, 50], [1, 100, 40], 4, 2, 64, 32, 0, False, False)                   # nothing but copies
    append_case(dtype, [3, 4, 50], [1, 100, 40], 4, 2, 64, 32, 24, False, True)                   # halves that end inside 16 bytes
    append_case(dtype, [3, 4, 50], [1, 100, 40], 4, 2, 64, 32, 64, False, True, explicit=True)
    append_case(dtype, [3, 4, 50], [1, 100, 40], 4, 2, 64, 32, 64, False, True, front=2, behind=3)
    append_case(dtype, [3, 4, 50], [1, 100, 40], 4, 2, 64, 32, 64, False, True, views=True)
    many = [b % 3 for b in range(1100)]
    append_case(dtype, many, [b % 29 for b in range(1100)], 2, 1, 32, 16, 32, True, True)         # more samples than 32 * 32


@pytest.mark.parametrize("dtype", TYPES)
def test_bad_places_are_not_written_and_reported(dtype):
    H, kv, D, page = 4, 2, 64, 16
    for what, value in (("page", -1), ("page", 1 << 30), ("len", 2 ** 31 - 1), ("len", 1), ("len", 100), ("start", 10 ** 9), ("start", -5)):
        cache = Cache(dtype, 3, 48, kv, D, page)
        k = torch.randn(9, kv, D, device="cuda").to(dtype)
        v = torch.randn(9, kv, D, device="cuda").to(dtype)
        kv_len = torch.tensor([20, 20, 20], dtype=torch.int32, device="cuda")
        q_start = torch.tensor([0, 3, 6, 9], dtype=torch.int32, device="cuda")
        table = cache.table.clone()
        if what == "page":
            table[1, 1] = value
        elif what == "len":
            kv_len[1] = value
        else:
            q_start[1] = value
        ctx = ctx_for(1, H, kv, D, dtype)
        ctx.append_kv(k, v, cache.k, cache.v, table, kv_len, q_start=q_start)
        with pytest.raises(swam.SwamError) as e:
            ctx.check()
        assert e.value.code == swam.ERR_DEVICE_CHECK
        if what != "start":
            assert torch.equal(cache.rows(cache.v, 0, 17, 3), v[:3])
        else:
            assert (cache.rows(cache.v, 0, 0, 48) == 9).all() and (cache.rows(cache.v, 1, 0, 48) == 9).all()
        assert torch.equal(cache.rows(cache.v, 2, 17, 3), v[6:])
        if what == "len" and value == 1:
            assert torch.equal(cache.rows(cache.v, 1, 0, 1), v[5:6])          # its last token has a place
        ctx.check()


def test_appended_in_a_graph_and_on_another_stream():
    dtype, H, kv, D, page = BF16, 4, 2, 64, 16
    cache = Cache(dtype, 2, 64, kv, D, page)
    q, k, v = (torch.randn(2, h, D, device="cuda").to(dtype) for h in (H, kv, kv))
    kv_len = torch.tensor([1, 10], dtype=torch.int32, device="cuda")
    ctx = ctx_for(1, H, kv, D, dtype)
    rope = swam.Rope(ladder(D))
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        got = ctx.append_kv(k, v, cache.k, cache.v, cache.table, kv_len, q=q, rope=rope)
    del rope                                                    # (what the call read of it is in the graph)
    for step in range(20):
        q.copy_(torch.randn_like(q))
        k.copy_(torch.randn_like(k))
        v.copy_(torch.randn_like(v))
        graph.replay()
        for b, past in enumerate((step, 9 + step)):
            pos = torch.tensor([[past]], device="cuda")
            close(cache.rows(cache.k, b, past, 1), *definition(k[b:b + 1], None, 0, ladder(D), [0] * 32, False, 1.0, pos), dtype)
            assert torch.equal(cache.rows(cache.v, b, past, 1), v[b:b + 1])
            close(got[b:b + 1], *definition(q[b:b + 1], None, 0, ladder(D), [0] * 32, False, 1.0, pos), dtype)
        kv_len += 1
    ctx.check()


def test_refusals():
    B, n, H, kv, D = 2, 6, 4, 2, 64
    ctx = ctx_for(B, H, kv, D, BF16)
    q, k = (torch.zeros(B, n, h, D, dtype=BF16, device="cuda") for h in (H, kv))
    rope, w = swam.Rope(ladder(D)), torch.ones(D, device="cuda")

    def refused(call, error=ValueError, code=None):
        before = ctx.launch_count()
        with pytest.raises(error) as e:
            call()
        if code is not None:
            assert e.value.code == code
        assert ctx.launch_count() == before

    refused(lambda: ctx.norm_rope())
    refused(lambda: ctx.norm_rope(q.float()))
    refused(lambda: ctx.norm_rope(q.cpu()))
    refused(lambda: ctx.norm_rope(q[:1]))
    refused(lambda: ctx.norm_rope(q[:, :, :2]))
    refused(lambda: ctx.norm_rope(q, k[:, :3]))
    refused(lambda: ctx.norm_rope(q[0]))
    refused(lambda: ctx.norm_rope(q.transpose(1, 2).contiguous().transpose(1, 2)))
    refused(lambda: ctx.norm_rope(q, rope=rope, positions=torch.zeros(n, dtype=torch.int64, device="cuda")))
    refused(lambda: ctx.norm_rope(q, rope=rope, positions=torch.zeros(n + 1, dtype=torch.int32, device="cuda")))
    refused(lambda: ctx.norm_rope(q, rope=rope, positions=torch.zeros(n, dtype=torch.int32)))
    refused(lambda: ctx.norm_rope(q, q_weight=w.bfloat16()))
    refused(lambda: ctx.norm_rope(q, q_weight=w[:32]))
    refused(lambda: ctx.norm_rope(q, q_out=q[:, :3]))
    refused(lambda: ctx.norm_rope(q, k_out=k))
    refused(lambda: ctx.norm_rope(k=torch.zeros(B, n, 3, D, dtype=BF16, device="cuda")), swam.SwamError, swam.ERR_INVALID_ARG)
    both = torch.zeros(B * n * H * D + 1024, dtype=BF16, device="cuda")
    x, y = both[:-1024].view(B, n, H, D), both[1024:].view(B, n, H, D)
    refused(lambda: ctx.norm_rope(x, q_out=y), swam.SwamError, swam.ERR_INVALID_ARG)               # overlapping, not in place
    refused(lambda: ctx.norm_rope(q, k, q_out=torch.empty_like(q), k_out=q[:, :, :kv]), swam.SwamError, swam.ERR_INVALID_ARG)
    refused(lambda: ctx.norm_rope(q, eps=-1.0), swam.SwamError, swam.ERR_INVALID_ARG)
    refused(lambda: ctx.norm_rope(q, eps=float("nan")), swam.SwamError, swam.ERR_INVALID_ARG)
    refused(lambda: ctx.norm_rope(q, rope=swam.Rope(ladder(128))), swam.SwamError, swam.ERR_INVALID_ARG)
    refused(lambda: ctx.norm_rope(q, rope=swam.Rope([float("inf")])), swam.SwamError, swam.ERR_INVALID_ARG)
    refused(lambda: ctx.norm_rope(q, rope=swam.Rope([2.0 ** 21])), swam.SwamError, swam.ERR_INVALID_ARG)
    refused(lambda: ctx.norm_rope(q, rope=swam.Rope([1.0], axes=[8])), swam.SwamError, swam.ERR_INVALID_ARG)
    empty, _ = ctx.norm_rope(q[:, :0], rope=rope)
    assert empty.shape == (B, 0, H, D)

    cache = Cache(BF16, 2, 40, kv, D, 16)
    kv_len = torch.tensor([3, 3], dtype=torch.int32, device="cuda")
    kn, vn, qn = (torch.zeros(2, h, D, dtype=BF16, device="cuda") for h in (kv, kv, H))

    def append(**kw):
        a = dict(k=kn, v=vn, k_pages=cache.k, v_pages=cache.v, page_table=cache.table, kv_len=kv_len)
        return lambda: ctx.append_kv(**{**a, **kw})

    refused(append(v=vn[:1]))
    refused(append(k=kn[:, :1]))
    refused(append(q=qn[:1]))
    refused(append(q_out=qn))
    refused(append(k=kn.float()))
    refused(append(kv_len=kv_len.long()))
    refused(append(page_table=cache.table[:1]))
    refused(append(q_start=kv_len))
    refused(append(rope=rope, positions=torch.zeros(3, dtype=torch.int32, device="cuda")))
    refused(append(k_weight=w.double()))
    refused(append(k_pages=cache.k[:, :8], v_pages=cache.v[:, :8]), swam.SwamError, swam.ERR_INVALID_ARG)
    refused(append(v_pages=cache.k), swam.SwamError, swam.ERR_INVALID_ARG)
    refused(append(v=kn, k=cache.k[0, :2]), swam.SwamError, swam.ERR_INVALID_ARG)
    refused(append(q=qn, q_out=cache.k[:1].view(-1, H, D)[:2]), swam.SwamError, swam.ERR_INVALID_ARG)
    refused(append(k=kn[:1], v=vn[:1]), swam.SwamError, swam.ERR_INVALID_ARG)                       # one token, two samples, no q_start
    before = ctx.launch_count()
    append(k=kn[:0], v=vn[:0])()
    assert ctx.launch_count() == before
    # the C entry
    a = swam.SwamAppendArgs()
    c = ctx._cache(cache.k, cache.v, cache.table, kv_len, None)
    a.cache, a.k, a.v, a.n_tokens = ctypes.addressof(c), kn.data_ptr(), vn.data_ptr(), 2
    for name, value in (("cache", None), ("k", None), ("v", None), ("k", kn.data_ptr() + 2), ("q", qn.data_ptr()), ("n_tokens", -1),
                        ("k_token", 64), ("v_token", -8), ("positions", kv_len.data_ptr() + 2), ("k_weight", w.data_ptr() + 4)):
        keep = getattr(a, name)
        setattr(a, name, value)
        assert ctx.lib.swam_append_kv(ctx.ctx, ctypes.byref(a), None) == swam.ERR_INVALID_ARG, name
        setattr(a, name, keep)
    assert ctx.launch_count() == before


# ---------------------------------------------------------------------------------------------------------------------- together
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D,page", [(64, 16), (128, 64)])
def test_a_rollout_over_a_paged_history(dtype, D, page):
    """Observation chunks and single tokens of three robots go into the cache and attend it, step after step; each step equals
    shared-prefix attention's kind of sum over everything the sample has seen so far, from keys made by norm_rope."""
    H, kv, B = 4, 2, 3
    gen = torch.Generator(device="cuda").manual_seed(11)
    ctx = ctx_for(B, H, kv, D, dtype)
    cache = Cache(dtype, B, 400, kv, D, page)
    qw, kw = weights(gen, D)
    rope = swam.Rope(swam.rope_frequencies(D, factor=4.0, trained=128), magnitude=swam.rope_magnitude(4.0))
    lens = [0] * B
    history = [([], []) for _ in range(B)]
    for new in ([40, 1, 17], [1, 1, 1], [130, 0, 2], [1, 1, 1], [5, 70, 1]):
        total = sum(new)
        qkv = base.rand(gen, total, H + 2 * kv, D, dtype=dtype)
        q, k, v = qkv[:, :H], qkv[:, H:H + kv], qkv[:, H + kv:]
        lens = [a + b for a, b in zip(lens, new)]
        starts = [0]
        for n in new:
            starts.append(starts[-1] + n)
        kv_len, q_start = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (lens, starts))
        q2 = ctx.append_kv(k, v, cache.k, cache.v, cache.table, kv_len, q_start=q_start, q=q, rope=rope, q_weight=qw, k_weight=kw)
        out, lse = ctx.paged_attn(q2, cache.k, cache.v, cache.table, kv_len, q_start=q_start, max_q=max(new), causal=True, want_lse=True)
        ctx.check()
        for b, n in enumerate(new):
            if n == 0:
                continue
            s = slice(starts[b], starts[b + 1])
            # the same token through norm_rope: same bits
            pos = torch.arange(lens[b] - n, lens[b], device="cuda", dtype=torch.int32)
            one = ctx_for(1, H, kv, D, dtype)
            qr, kr = one.norm_rope(q[s][None], k[s][None], rope, positions=pos, q_weight=qw, k_weight=kw)
            assert torch.equal(qr[0], q2[s])
            history[b][0].append(kr[0])
            history[b][1].append(v[s])
            keys, values = (torch.cat(x) for x in history[b])
            assert keys.shape[0] == lens[b]
            mask = torch.arange(lens[b], device="cuda")[None] <= pos[:, None]
            base.compare(out[None, s], lse[None, :, s], q2[None, s], lambda _, h: (keys[:, h // 2].double(), values[:, h // 2].double(), mask), D, dtype)
            # and through the contiguous cache of the existing call
            if n > 1:
                o, l = one.prefix_attn(q2[s][None], keys[None, :0], values[None, :0], keys[None], values[None], causal=True, want_lse=True)
                base.compare(o, l, q2[None, s], lambda _, h: (keys[:, h // 2].double(), values[:, h // 2].double(), mask), D, dtype)

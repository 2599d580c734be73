"""The ways in which the segment-attention calls cut their work, each against the definition in 64 bits, with the number
of launches that tells which way was taken; and what the calls say about lengths and sizes at their limits."""
import ctypes

import pytest
import torch

import test_gpu_segment_attn as base
from paper_2609_38984_b200 import swam

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def launches(ctx, call):
    n = ctx.launch_count()
    call()
    ctx.check()
    return ctx.launch_count() - n


def scratch_bytes(ctx, **kw):
    n = ctypes.c_size_t()
    rc = ctx.lib.swam_cross_attn_scratch_bytes(ctx.ctx, ctypes.byref(swam.SwamCrossArgs(**kw)), ctypes.byref(n))
    return rc, n.value


def test_the_longest_key_ranges_are_cut_into_pieces_that_a_bounded_wait_outlasts():
    """A wait in the tensor-core kernel may last as long as a work item: some 3110 clocks a tile of 128 keys, against a limit of 4e9
    clocks.  So an item has at most 2^26 keys, whatever the number of items (here more than there are SMs)."""
    B, H, D, n_q = 40, 8, 128, 300
    ctx = base.make_ctx(B, H, D, 1, swam.BF16)
    piece = B * n_q * H * (D * 4 + 8)
    for n_kv, pieces in ((1 << 20, 0), (1 << 26, 0), ((1 << 26) + 1, 2), (1 << 27, 2), (1 << 29, 8)):
        assert scratch_bytes(ctx, n_q=n_q, n_kv=n_kv) == (swam.OK, pieces * piece), n_kv


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_lengths_of_tensors_without_rows_are_checked(dtype):
    """A length other than 0 for a tensor without rows is out of range like any other."""
    dt, B = base.DT[dtype], 4
    gen = torch.Generator(device="cuda").manual_seed(1)
    ctx = base.make_ctx(B, 4, 64, 2, swam.F32 if dtype == "f32" else swam.BF16)
    some = base.rand(gen, B, 30, 2, 64, dtype=dt)
    none = some[:, :0]
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    for n_q in (1, 3, 200):
        q = base.rand(gen, B, n_q, 4, 64, dtype=dt)
        for bad in (lambda: ctx.cross_attn(q, none, none, kv_len=ints(0, 0, 0, 5)),
                    lambda: ctx.cross_attn(q, none, none, kv_len=ints(-1, 0, 0, 0)),
                    lambda: ctx.prefix_attn(q, some[:2], some[:2], none, none, own_len=ints(0, 0, 3, 0)),
                    lambda: ctx.prefix_attn(q, some[:2], some[:2], none, none, own_len=ints(0, -1, 0, 0), causal=True),
                    lambda: ctx.prefix_attn(q, none[:1], none[:1], some, some, prefix_len=ints(1))):
            out = bad()
            with pytest.raises(swam.SwamError) as e:
                ctx.check()
            assert e.value.code == swam.ERR_DEVICE_CHECK and "length" in str(e.value)
            assert torch.isfinite(out).all()
        want = ctx.prefix_attn(q, some[:2], some[:2], none, none)
        got = ctx.prefix_attn(q, some[:2], some[:2], none, none, own_len=ints(0, 0, 0, 0))
        ctx.check()
        assert torch.equal(got, want)
        assert (ctx.cross_attn(q, none, none, kv_len=ints(0, 0, 0, 0)) == 0).all()
        ctx.check()


def test_an_output_over_an_input_is_refused():
    """Results over an input that other rows still read: the same tensor, or two contiguous ones that share a part.  Different
    heads or samples of one wider tensor are fine."""
    ctx = base.make_ctx(2, 4, 64, 4, swam.BF16)
    gen = torch.Generator(device="cuda").manual_seed(1)
    q = base.rand(gen, 2, 30, 4, 64, dtype=BF)
    kv = base.rand(gen, 2, 30, 2, 4, 64, dtype=BF)
    k, v = kv[:, :, 0], kv[:, :, 1]
    flat = base.rand(gen, 2 * 30 * 4 * 64 * 2, dtype=BF)
    a, b = flat[:15360].view(2, 30, 4, 64), flat[7680:23040].view(2, 30, 4, 64)
    before = ctx.launch_count()
    for args, out in (((q, k, v), q), ((q, k, v), k), ((q, k, v), v), ((a, k, v), b), ((b, k, v), a), ((q, a, k), b), ((q, k, b), a)):
        with pytest.raises(swam.SwamError) as e:
            ctx.cross_attn(*args, out=out)
        assert e.value.code == swam.ERR_INVALID_ARG and "overlap" in str(e.value)
    for pre, own, out in (((k[:1], v[:1]), (a, a), a), ((a[:1], k[:1]), (k, v), a)):
        with pytest.raises(swam.SwamError) as e:
            ctx.prefix_attn(q, *pre, *own, out=out)
        assert e.value.code == swam.ERR_INVALID_ARG and "overlap" in str(e.value)
    assert ctx.launch_count() == before
    want = ctx.cross_attn(q, k, v)
    wide = base.rand(gen, 2, 30, 16, 64, dtype=BF)
    wide[:, :, :4], wide[:, :, 4:8], wide[:, :, 12:] = q, k, v
    got = ctx.cross_attn(wide[:, :, :4], wide[:, :, 4:8], wide[:, :, 12:], out=wide[:, :, 8:12])
    ctx.check()
    assert torch.equal(got, want) and torch.equal(wide[:, :, :4], q) and torch.equal(wide[:, :, 12:], v)
    # samples of one buffer side by side
    two = base.rand(gen, 4, 30, 4, 64, dtype=BF)
    two[:2] = q
    assert torch.equal(ctx.cross_attn(two[:2], k, v, out=two[2:]), want)
    two[::2] = q
    assert torch.equal(ctx.cross_attn(two[::2], k, v, out=two[1::2]), want)
    ctx.check()


def test_what_the_binding_keeps_of_past_sizes_is_bounded():
    """A decoding loop calls with another length every time; the sizes that the binding remembers stay few."""
    ctx = base.make_ctx(1, 2, 64, 2, swam.BF16)
    q = torch.zeros(1, 1, 2, 64, dtype=BF, device="cuda")
    k = torch.zeros(1, 400, 2, 64, dtype=BF, device="cuda")
    for n in range(1, 400):
        ctx.cross_attn(q, k[:, :n], k[:, :n])
    ctx.check()
    kept = [x for x in vars(ctx).values() if isinstance(x, dict)]
    assert kept and all(len(x) <= 64 for x in kept)


def test_keys_without_heads_are_refused():
    ctx = base.make_ctx(2, 4, 64, 2, swam.BF16)
    q = torch.zeros(2, 3, 4, 64, dtype=BF, device="cuda")
    k = torch.zeros(2, 0, 0, 64, dtype=BF, device="cuda")
    with pytest.raises(ValueError):
        ctx.cross_attn(q, k, k)
    with pytest.raises(ValueError):
        ctx.prefix_attn(q, k, k, k, k)

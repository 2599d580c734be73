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


def prefix_again(ctx, t, causal):
    q, kp, vp, k, v, pl, ol = t
    ol = ol if k.shape[1] else None            # (lengths of a tensor without rows take a launch to check)
    return launches(ctx, lambda: ctx.prefix_attn(q, kp, vp, k, v, prefix_len=pl, own_len=ol, causal=causal, want_lse=True))


def ragged(n, most):
    """Lengths from none to all, tile borders among them."""
    steps = [most, 0, 1, 128, 129, most - 1, 16, 640, 255, 513]
    return [min(most, steps[i % len(steps)]) for i in range(n)]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("n_q,H,kv", [(64, 3, 3), (32, 4, 2), (40, 3, 3), (20, 4, 2), (9, 10, 2)])
def test_both_passes_in_one_tensor_core_launch(D, causal, n_q, H, kv):
    """33 to 64 rows a sample, two samples to a tile, and more than 512 own keys: shared tiles and samples' own tiles in one
    launch (queries as boxes of 64-row samples, or row by row), then the merge."""
    B, groups, n_own = 6, 3, 700
    ctx, t, _, _ = base.prefix_case(BF, B, groups, n_q, H, kv, D, 400, n_own, [400, 0, 131], ragged(B, n_own), causal, seed=D + n_q)
    assert prefix_again(ctx, t, causal) == 2
    ctx, t, _, _ = base.prefix_case(BF, B, groups, n_q, H, kv, D, 3000, n_own, [3000, 2049, 130], ragged(B, n_own)[::-1], causal,
                                    seed=D + n_q + 1)
    assert prefix_again(ctx, t, causal) == 2


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("n_q,H,kv", [(64, 3, 3), (32, 4, 2), (40, 3, 3), (20, 4, 2)])
def test_shared_256_row_tiles_and_a_second_tensor_core_pass(D, causal, n_q, H, kv):
    """Groups of five such samples: 256-row tiles over several samples (the last one of a group ends inside the next group's
    samples), the own keys as a second launch on the tensor cores, and the merge."""
    B, groups, n_own = 10, 2, 700
    ctx, t, _, _ = base.prefix_case(BF, B, groups, n_q, H, kv, D, 3000, n_own, [3000, 1111], ragged(B, n_own), causal, seed=D + n_q)
    assert prefix_again(ctx, t, causal) == 3


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("per_group,n_q,H,kv", [(4, 40, 3, 3), (4, 64, 3, 3), (2, 40, 3, 3), (2, 32, 4, 2), (9, 7, 10, 2)])
def test_shared_tiles_without_own_keys(D, per_group, n_q, H, kv):
    """Several samples to a tensor-core tile with a final result: one launch, no merge."""
    B = 2 * per_group
    ctx, t, _, _ = base.prefix_case(BF, B, 2, n_q, H, kv, D, 300, 0, [300, 129], [0] * B, False, seed=D + n_q)
    assert prefix_again(ctx, t, False) == 1
    ctx, t, _, _ = base.prefix_case(BF, B, 2, n_q, H, kv, D, 300, 0, [0, 17], [0] * B, True, seed=D + n_q)
    assert prefix_again(ctx, t, True) == 1


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n_q,H,kv", [(300, 2, 2), (256, 4, 2), (100, 6, 2)])
def test_256_row_tiles_in_pieces(D, n_q, H, kv):
    """More than 128 rows and many keys for few heads: pieces of 256-row tiles, some of them without real keys."""
    lens = [5000, 4097, 700, 0]
    ctx, q, k, v, kv_len, _, _ = base.cross_case(BF, len(lens), n_q, H, kv, D, 5000, lens, seed=D + n_q, interleaved=True)
    assert launches(ctx, lambda: ctx.cross_attn(q, k, v, kv_len=kv_len, want_lse=True)) == 2
    # the same through a prefix of each sample's own
    ctx, t, _, _ = base.prefix_case(BF, 2, 2, n_q, H, kv, D, 3000, 1500, [3000, 1025], [1500, 70], True, seed=D + n_q)
    assert prefix_again(ctx, t, True) == 2


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

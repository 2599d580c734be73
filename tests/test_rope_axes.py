"""Positions with more components than the rotation uses."""
import pytest

from paper_2609_38984_b200 import swam


def test_the_number_of_axes_can_be_given():
    assert swam.Rope([1.0, 0.5]).n_axes == 1
    assert swam.Rope([1.0, 0.5], axes=[0, 2]).n_axes == 3
    assert swam.Rope([1.0, 0.5], axes=[0, 1], n_axes=3).n_axes == 3
    assert swam.Rope([1.0, 0.5], n_axes=3).n_axes == 3
    assert swam.Rope([1.0], axes=[0], n_axes=2)._c.n_axes == 2
    for bad in (0, -1, 2, 9):
        with pytest.raises(ValueError):
            swam.Rope([1.0, 0.5], axes=[0, 2], n_axes=bad)
    with pytest.raises(ValueError):
        swam.Rope([1.0], n_axes=9)


@pytest.mark.gpu
def test_positions_with_an_axis_that_nothing_turns_by():
    """A three-axis model whose rotated part has pairs for the first two: its positions are taken as they are, with the same result as those two."""
    import torch

    import test_gpu_norm_rope as rope_tests
    D, n = 64, 9
    gen = torch.Generator(device="cuda").manual_seed(3)
    ctx = rope_tests.ctx_for(1, 4, 2, D, torch.float32)
    q = torch.randn(1, n, 4, D, generator=gen, device="cuda")
    three = torch.randint(0, 500, (n, 3), generator=gen, device="cuda", dtype=torch.int32)
    freq, axis = rope_tests.ladder(16) + rope_tests.ladder(16), [0] * 8 + [1] * 8
    want, _ = ctx.norm_rope(q, rope=swam.Rope(freq, axes=axis), positions=three[:, :2].contiguous())
    rope = swam.Rope(freq, axes=axis, n_axes=3)
    got, _ = ctx.norm_rope(q, rope=rope, positions=three)
    assert torch.equal(got, want)
    with pytest.raises(ValueError):
        ctx.norm_rope(q, rope=rope, positions=three[:, :2].contiguous())
    # and on the way into a cache
    cache = rope_tests.Cache(torch.float32, 1, 16, 2, D, 16)
    k = torch.randn(n, 2, D, generator=gen, device="cuda")
    out = ctx.append_kv(k, k.clone(), cache.k, cache.v, cache.table, torch.tensor([n], dtype=torch.int32, device="cuda"), q=q[0], rope=rope, positions=three)
    ctx.check()
    assert torch.equal(out, want[0])

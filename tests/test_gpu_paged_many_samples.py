"""Ragged batches whose call does not say how many new tokens a sample has at most: the fp32 kernel's blocks find their rows by the samples'
own lengths."""
import math

import pytest
import torch

import test_gpu_paged_attn as paged
import test_gpu_segment_attn as base
from paper_2609_38984_b200 import swam

pytestmark = pytest.mark.gpu
F32, U32 = paged.KINDS[2], base.U32


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("new,lens", [([1, 0, 300, 2, 0, 64, 65], [40, 5, 400, 33, 0, 64, 70]), ([1, 0, 300, 2, 0, 64, 65], [5000, 50, 400, 33, 0, 9000, 70]),
                                      ([0, 0, 7], [3, 9, 2000]), ([1] * 20 + [150], [10 + 100 * b for b in range(21)])])
@pytest.mark.parametrize("causal", [False, True])
def test_without_a_bound_on_the_new_tokens(D, new, lens, causal):
    lens = [max(a, b) for a, b in zip(new, lens)]
    c, want, want_lse = paged.check(F32, causal, new, lens, 4, 2, D, 32, front=1, behind=2, run=dict(max_q=0))
    for _ in range(2):
        out, lse = c.run(causal, max_q=0)
        assert torch.equal(out[1:-2], want[1:-2]) and torch.equal(lse[:, 1:-2], want_lse[:, 1:-2])


@pytest.mark.parametrize("n", [300, 1000])
def test_hundreds_of_samples(n):
    """More samples than a block has threads."""
    new = [(1, 0, 2, 90, 3)[b % 5] for b in range(n)]
    lens = [max(new[b], 1 + (b * 37) % 150) for b in range(n)]
    paged.check(F32, True, new, lens, 4, 2, 32, 16, run=dict(max_q=0))


def test_as_many_samples_as_a_call_takes():
    """65535 samples of two new tokens and 32 heads, each with a page of its own sample's number modulo 64."""
    n, H, D, page = 65535, 32, 32, 16
    gen = torch.Generator(device="cuda").manual_seed(1)
    ctx = base.make_ctx(1, H, D, H, swam.F32)
    k, v = (base.rand(gen, 64, page, H, D, dtype=torch.float32) for _ in range(2))
    table = (torch.arange(n, device="cuda", dtype=torch.int32) % 64)[:, None].contiguous()
    kv_len = (2 + torch.arange(n, device="cuda", dtype=torch.int32) % 13).contiguous()
    q_start = torch.arange(0, 2 * n + 1, 2, device="cuda", dtype=torch.int32)
    q = base.rand(gen, 2 * n, H, D, dtype=torch.float32)
    out, lse = ctx.paged_attn(q, k, v, table, kv_len, q_start=q_start, causal=True, want_lse=True)
    ctx.check()
    # the definition in 64 bits, the samples of one page at a time; tolerances as in test_gpu_segment_attn.py
    scale = 1.0 / math.sqrt(D)
    for r in range(64):
        b = torch.arange(r, n, 64, device="cuda")
        rows = (2 * b[:, None] + torch.arange(2, device="cuda")).flatten()
        limit = (kv_len[b].long()[:, None] - 1 + torch.arange(2, device="cuda")).flatten()          # keys that a row sees
        x, keys, values = q[rows].double(), k[r].double(), v[r].double()
        hidden = torch.arange(page, device="cuda")[None, None] >= limit[:, None, None]
        logits = (torch.einsum("thd,chd->thc", x, keys) * scale).masked_fill(hidden, -math.inf)
        S = (torch.einsum("thd,chd->thc", x.abs(), keys.abs()) * scale).masked_fill(hidden, 0.0).amax(-1)
        p, want = torch.softmax(logits, -1), torch.logsumexp(logits, -1)
        e = (D + 4) * U32 * S + 2.0 ** -18
        ref, A = torch.einsum("thc,chd->thd", p, values), torch.einsum("thc,chd->thd", p, values.abs())
        assert ((out[rows].double() - ref).abs() <= (2 * e + 2 * (page + 8) * U32)[..., None] * A + U32 * ref.abs()).all(), r
        assert ((lse[:, rows].T.double() - want).abs() <= e + (page + 8) * U32 + 4 * U32 * want.abs()).all(), r

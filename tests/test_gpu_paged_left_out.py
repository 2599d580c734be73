"""Rows of samples that a paged attention call leaves out: an output and a log-sum-exp that are there stay as they are, whichever kernel and
however many pieces the keys are cut into."""
import ctypes

import pytest
import torch

import test_gpu_paged_attn as paged
from paper_2609_38984_b200 import swam

pytestmark = pytest.mark.gpu


def through_the_c_entry(c, out, lse, max_q, causal=True):
    """The call with scratch full of threes: a piece that nobody wrote would count as one with keys."""
    cache = c.ctx._cache(c.k_pages, c.v_pages, c.table, c.kv_len, c.q_start)
    a = swam.SwamPagedArgs(ctypes.addressof(cache), c.q.data_ptr(), out.data_ptr(), lse.data_ptr(), None, 0, c.total, max_q, 0, int(causal), 0, 0)
    need = ctypes.c_size_t()
    assert c.ctx.lib.swam_paged_attn_scratch_bytes(c.ctx.ctx, ctypes.byref(a), ctypes.byref(need)) == swam.OK
    scratch = torch.full((need.value // 4 + 64,), 3.0, device="cuda")
    a.scratch, a.scratch_bytes = (scratch.data_ptr() + 255) & ~255, need.value
    assert c.ctx.lib.swam_paged_attn(c.ctx.ctx, ctypes.byref(a), torch.cuda.current_stream().cuda_stream) == swam.OK
    torch.cuda.synchronize()


@pytest.mark.parametrize("kind", paged.KINDS)
@pytest.mark.parametrize("new", [[2, 4, 1, 3], [20, 33, 9, 30], [70, 95, 3, 90]])
@pytest.mark.parametrize("lens", [[900, 1400, 300, 2000], [100, 130, 99, 110], [20000, 17000, 700, 30000]])
@pytest.mark.parametrize("spoilt", ["max_q", "order", "order, no bound"])
def test_rows_of_a_sample_that_is_left_out_stay_as_they_are(kind, new, lens, spoilt):
    H, kv, D = 8, 2, 64
    c = paged.case(kind, list(new), lens, H, kv, D, 64, front=2, behind=3)
    out = torch.full((c.total, H, D), 7.0, device="cuda").to(c.dtype)
    lse = torch.full((H, c.total), 7.0, device="cuda")
    if spoilt == "max_q":          # the second sample has more new tokens than the call says
        left, max_q = [1], new[3]
    else:                          # the end of the first sample's stretch, and with it the start of the second's, is nowhere
        left, max_q = [0, 1], 0 if "no bound" in spoilt else max(new)
        c.q_start[1] = 10 ** 9
    through_the_c_entry(c, out, lse, max_q)
    with pytest.raises(swam.SwamError) as e:
        c.ctx.check()
    assert e.value.code == swam.ERR_DEVICE_CHECK
    for b in left:
        s = slice(c.starts[b], c.starts[b + 1])
        assert (out[s] == 7).all() and (lse[:, s] == 7).all(), b
        c.new[b] = 0
    assert (out[:2] == 7).all() and (out[-3:] == 7).all() and (lse[:, :2] == 7).all() and (lse[:, -3:] == 7).all()
    c.compare(out, lse, True)

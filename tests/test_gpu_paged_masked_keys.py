"""Keys that the causal limit hides from a row may hold anything: huge numbers, infinities and NaN of the last new tokens reach only the rows that
see them."""
import pytest
import torch

import test_gpu_paged_attn as paged

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", paged.KINDS)
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("n,length", [(2, 600), (12, 700), (14, 4000), (30, 900), (60, 900), (64, 140), (140, 900), (140, 140), (300, 5000)])
@pytest.mark.parametrize("value", [3e38, -3e38, float("inf"), float("-inf"), float("nan"), "both"])
def test_hidden_keys_hold_anything(kind, D, n, length, value):
    """Rows in front of the last three tokens equal the definition without these, tokens without any key among them."""
    H, kv, page = 4, 2, 16
    hidden = min(3, n - 1)
    c = paged.case(kind, [n, 5], [length, 333], H, kv, D, page)
    for i in range(length - hidden, length):
        at = int(c.table_host[0, i // page]), i % page
        if value == "both":
            c.k_pages[at] = float("inf")
            c.k_pages[at][:, ::2] = -float("inf")
        else:
            c.k_pages[at] = value
    out, lse = c.run(True)
    c.ctx.check()
    seen = n - hidden
    # what sees no hidden key, against the definition
    c.new[0], c.lens[0] = seen, length - hidden
    c.keys[0], c.values[0] = c.keys[0][:length - hidden], c.values[0][:length - hidden]
    c.compare(out, lse, True)
    if value != value or value == "both":
        assert not torch.isfinite(out[n - hidden:n].float()).any()

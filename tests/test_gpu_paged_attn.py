"""Attention over a paged cache against its definition in 64 bits.

Tolerances are those of test_gpu_segment_attn.py, whose derivation covers any order of the sums: the pages only say where a key
is.  Whatever a page holds behind its sample's last token is NaN here, and so are the pages that belong to nobody."""
import ctypes
import math

import pytest
import torch

import test_gpu_segment_attn as base
from paper_2609_38984_b200 import swam

U16, U32 = base.U16, base.U32
pytestmark = pytest.mark.gpu
NAN = float("nan")
BF16, F32 = torch.bfloat16, torch.float32
# storage type and attention variant: tcgen05 or warp-level by size, warp-level always, fp32
KINDS = [(BF16, swam.ATTN_AUTO), (BF16, swam.ATTN_WARP_MMA), (F32, swam.ATTN_AUTO)]


class Case:
    """A ragged batch: `new` tokens and `lens` tokens in all per sample, the cache in shuffled pages."""

    def __init__(self, dtype, new, lens, H, kv, D, page, seed=0, scale=1.0, pad=NAN, front=0, behind=0, interleaved=False):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        host = torch.Generator().manual_seed(seed)
        self.dtype, self.new, self.lens, self.H, self.kv, self.D, self.page = dtype, new, lens, H, kv, D, page
        self.total = front + sum(new) + behind
        counts = [(n + page - 1) // page for n in lens]
        n_pages = sum(counts) + 2
        order = torch.randperm(n_pages, generator=host, dtype=torch.int32)
        table = torch.full((len(new), max(counts + [1])), -7, dtype=torch.int32)
        at = 0
        for b, c in enumerate(counts):
            table[b, :c] = order[at:at + c]
            at += c
        self.table_host = table
        if interleaved:        # keys and values of a page side by side, as views
            both = torch.full((n_pages, page, 2, kv, D), pad, device="cuda").to(dtype)
            self.k_pages, self.v_pages = both[:, :, 0], both[:, :, 1]
        else:
            self.k_pages = torch.full((n_pages, page, kv, D), pad, device="cuda").to(dtype)
            self.v_pages = self.k_pages.clone()
        self.keys, self.values = [], []
        for b, n in enumerate(lens):
            k, v = (base.rand(gen, n, kv, D, dtype=dtype) for _ in range(2))
            self.keys.append(k)
            self.values.append(v)
            for c in range(counts[b]):
                m = min(page, n - c * page)
                self.k_pages[table[b, c], :m] = k[c * page:c * page + m]
                self.v_pages[table[b, c], :m] = v[c * page:c * page + m]
        starts = [front]
        for n in new:
            starts.append(starts[-1] + n)
        self.starts = starts
        self.table = table.cuda()
        self.kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.q_start = torch.tensor(starts, dtype=torch.int32, device="cuda")
        self.q = base.rand(gen, self.total, H, D, dtype=dtype, scale=scale)
        self.ctx = base.make_ctx(1, H, D, kv, swam.F32 if dtype == F32 else swam.BF16)

    def run(self, causal, **kw):
        kw.setdefault("q_start", self.q_start)
        kw.setdefault("max_q", max(self.new))
        return self.ctx.paged_attn(self.q, self.k_pages, self.v_pages, self.table, self.kv_len, causal=causal, want_lse=True, **kw)

    def compare(self, out, lse, causal):
        self.ctx.check()
        g = self.H // self.kv
        for b, n in enumerate(self.new):
            if n == 0:
                continue
            length, at = self.lens[b], self.starts[b]
            c = torch.arange(length, device="cuda")
            mask = torch.ones(n, length, dtype=torch.bool, device="cuda")
            if causal:
                mask = c[None] <= (length - n + torch.arange(n, device="cuda"))[:, None]
            base.compare(out[None, at:at + n], lse[None, :, at:at + n], self.q[None, at:at + n],
                         lambda _, h: (self.keys[b][:, h // g].double(), self.values[b][:, h // g].double(), mask), self.D, self.dtype)


def case(kind, *a, **kw):
    c = Case(kind[0], *a, **kw)
    c.ctx.set_option(swam.OPT_ATTN_VARIANT, kind[1])
    return c


def check(kind, causal, *a, run=None, **kw):
    c = case(kind, *a, **kw)
    out, lse = c.run(causal, **(run or {}))
    c.compare(out, lse, causal)
    return c, out, lse


# one token, tokens of a ragged batch around the tiles' sizes, and chunks of several tiles; samples without new tokens, without keys, with
# fewer keys than tokens
RAGGED = [([1] * 7, [1, 15, 16, 17, 64, 129, 700]),
          ([1, 5, 0, 2, 4], [40, 5, 33, 1300, 4]),
          ([33, 1, 17, 64], [33, 257, 130, 2]),
          ([130, 300, 7, 1], [400, 300, 1000, 64])]


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("H,kv,page", [(4, 4, 16), (8, 2, 64), (6, 2, 32), (5, 1, 128)])
@pytest.mark.parametrize("new,lens", RAGGED)
def test_ragged_batches(kind, D, causal, H, kv, page, new, lens):
    check(kind, causal, new, lens, H, kv, D, page)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256, 1024])
@pytest.mark.parametrize("new", [[1, 1, 1], [70, 3, 140]])
def test_page_sizes(kind, page, new):
    check(kind, True, new, [513, 1030, 257], 8, 2, 64, page)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("H,kv", [(8, 2), (3, 3)])
def test_single_tokens_behind_long_histories(kind, D, H, kv):
    """Keys shared out over many CTAs: one sample alone, and samples of very different lengths."""
    check(kind, True, [1], [20001], H, kv, D, 16)
    check(kind, True, [1] * 5, [1, 20000, 3, 700, 9000], H, kv, D, 64)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("new,lens", [([40], [5000]), ([64, 64], [3000, 6100]), ([300], [7000])])
def test_chunks_cut_along_the_keys(D, new, lens):
    for causal in (False, True):
        check(KINDS[0], causal, new, lens, 4, 2, D, 32)
        check(KINDS[2], causal, new, lens, 4, 2, D, 32)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("D", [64, 128])
def test_chunks_of_many_tiles(kind, D):
    check(kind, True, [1000, 37, 520], [1500, 2037, 520], 4, 2, D, 64)


@pytest.mark.parametrize("kind", KINDS)
def test_very_many_samples(kind):
    """More samples than a block has threads; some without new tokens, some without keys."""
    n = 300
    new = [(1, 0, 2, 1, 3)[b % 5] for b in range(n)]
    lens = [0 if b % 11 == 3 else 1 + (b * 37) % 150 for b in range(n)]
    check(kind, True, new, lens, 4, 2, 32, 16)
    new = [(1, 0, 40)[b % 3] for b in range(n)]
    check(kind, False, new, lens, 4, 2, 64, 16)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("D,kv,new,lens", [(64, 2, 20, 300), (128, 2, 20, 300), (64, 2, 40, 300), (128, 8, 300, 1000)])
def test_more_row_tiles_than_sms(D, kv, new, lens, causal):
    """Blocks that running ones take over: samples in no order of lengths, some of them empty; at most 64, at most 128 and more rows."""
    n = 150 if kv == 2 else 14
    counts = [0 if b % 9 == 4 else 1 + (b * 7919) % new for b in range(n)]
    lengths = [0 if b % 13 == 5 else 1 + (b * 104729) % lens for b in range(n)]
    counts[3], lengths[7] = new, lens
    c, want, want_lse = check(KINDS[0], causal, counts, lengths, 2 * kv, kv, D, 32)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        out, lse = c.run(causal)
    for _ in range(3):
        out.zero_()
        graph.replay()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("new", [[1, 1], [40, 3], [300, 20]])
def test_tables_with_room_for_much_more(kind, new):
    """Lengths far below what the table could hold, with and without bounds."""
    c = case(kind, new, [2500, 700], 8, 2, 64, 16)
    wide = torch.full((2, 8000), -1, dtype=torch.int32, device="cuda")
    wide[:, :c.table.shape[1]] = c.table
    c.table = wide
    for kw in (dict(), dict(max_kv=2500), dict(max_kv=100000), dict(max_q=0)):
        out, lse = c.run(True, **kw)
        c.compare(out, lse, True)


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("new,lens", [([70, 33, 1], [6000, 40, 1]), ([40, 0, 100, 12], [512, 900, 5200, 12]), ([100, 100, 100], [100, 2000, 3900])])
@pytest.mark.parametrize("causal", [False, True])
def test_few_chunks_of_unequal_histories(D, new, lens, causal):
    """Pieces of one size for all samples: one history has many, another a single one.  A call before leaves other pieces in the workspace."""
    first = case(KINDS[0], [90, 90], [8000, 7000], 4, 2, D, 32, seed=1)
    c = case(KINDS[0], new, lens, 4, 2, D, 32, seed=2)
    first.run(causal)
    c.ctx = first.ctx
    for kw in (dict(), dict(max_kv=20000)):
        out, lse = c.run(causal, **kw)
        c.compare(out, lse, causal)


@pytest.mark.parametrize("D,H,kv,new,lens", [(64, 8, 2, [245, 130, 77], [5000, 21000, 17500]), (128, 4, 2, [300, 1, 64], [18000, 700, 40]),
                                             (64, 4, 4, [100, 33, 0, 90, 120], [33, 30000, 17000, 19000, 2]), (32, 4, 1, [60, 80], [20000, 16500])])
@pytest.mark.parametrize("causal", [False, True])
def test_long_ragged_histories_of_few_row_tiles(D, H, kv, new, lens, causal):
    """Pieces for several blocks an SM, of one size; a repeat, with other blocks taken over, gives the same bits."""
    c, out, lse = check(KINDS[0], causal, new, lens, H, kv, D, 128)
    for _ in range(3):
        again, lse2 = c.run(causal)
        assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("D,H,kv", [(128, 6, 2), (64, 12, 4)])
def test_many_short_chunks_behind_long_histories(kind, D, H, kv):
    """17 to 32 rows of a sample and key/value head, some samples with fewer or none, histories of 1 to 2600 keys."""
    new = [6 + i % 5 - 6 * (i % 7 == 3) for i in range(76)]
    lens = [max(new[i], (i * 353) % 2600 + 1) for i in range(76)]
    for causal in (False, True):
        check(kind, causal, new, lens, H, kv, D, 64)


def test_two_threads_with_one_context():
    """Calls from two threads, each on a stream of its own: the binding keeps nothing of a call in the context."""
    import threading
    cases = [case(KINDS[0], [n] * 3, [700, 30 + n, 1500], 8, 2, 64, 16, seed=n) for n in (1, 70)]
    ctx = cases[0].ctx
    want = [c.run(True) for c in cases]
    for c in cases:
        c.ctx = ctx
    wrong = []

    def work(c, w):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(200):
                out, lse = c.run(True)
                torch.cuda.current_stream().synchronize()
                if not (torch.equal(out, w[0]) and torch.equal(lse, w[1])):
                    wrong.append(c.new)
    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=x) for x in zip(cases, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("new", [[2, 3], [80, 200]])
def test_rows_of_nobody_stay_as_they_are(kind, new):
    for lens in ([900, 33], [0, 0], [5, 0]):
        c = case(kind, new, lens, 4, 2, 64, 16, front=3, behind=5)
        out = torch.full((c.total, 4, 64), 7.0, device="cuda").to(c.dtype)
        got, lse = c.run(True, out=out)
        assert got is out
        c.compare(out, lse, True)
        assert (out[:3] == 7).all() and (out[-5:] == 7).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n", [1, 90])
def test_strided_views_and_equal_samples(kind, n):
    """Queries inside a fused projection, keys and values interleaved, a wider table, an output with gaps; no q_start."""
    H, kv, D = 4, 2, 64
    c = case(kind, [n] * 3, [n + 400, n, n + 17], H, kv, D, 16, interleaved=True)
    qkv = torch.full((c.total, H + 2 * kv, D), NAN, device="cuda").to(c.dtype)
    qkv[:, :H] = c.q
    wide = torch.full((3, c.table.shape[1] + 5), -1, dtype=torch.int32, device="cuda")
    wide[:, :c.table.shape[1]] = c.table
    gaps = torch.full((c.total, 2, H, D), 7.0, device="cuda").to(c.dtype)
    out, lse = c.ctx.paged_attn(qkv[:, :H], c.k_pages, c.v_pages, wide[:, :c.table.shape[1]], c.kv_len, causal=True, out=gaps[:, 0], want_lse=True)
    c.compare(out, lse, True)
    assert (gaps[:, 1] == 7).all()
    plain, _ = c.run(True)
    assert torch.equal(plain, out)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n", [1, 150])
def test_samples_that_share_pages(kind, n):
    c = case(kind, [n, n], [700, 700], 4, 2, 64, 64)
    c.table[1, :8] = c.table[0, :8]
    for x in (c.keys, c.values):
        x[1][:512] = x[0][:512]
    out, lse = c.run(True)
    c.compare(out, lse, True)


@pytest.mark.parametrize("n,D", [(1, 128), (140, 128), (140, 64), (1, 32)])
def test_logits_of_any_size_and_masked_infinities(n, D):
    """Growing logits move the running maximum in every tile; keys that the causal limit hides may be huge."""
    for kind in KINDS:
        c = case(kind, [n], [900], 4, 2, D, 16, scale=6.0)
        ramp = torch.linspace(0.05, 4.0, 900, device="cuda")[:, None, None]
        c.keys[0] = (c.keys[0].float() * ramp).to(c.dtype)
        for i in range(57):
            m = min(16, 900 - 16 * i)
            c.k_pages[c.table_host[0, i], :m] = c.keys[0][16 * i:16 * i + m]
        out, lse = c.run(True)
        c.compare(out, lse, True)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n", [1, 100])
def test_a_nan_key_reaches_the_rows_that_see_it_only(kind, n):
    c = case(kind, [n, n], [500, 500], 4, 2, 64, 16)
    c.k_pages[c.table_host[0, 2], 3] = NAN
    out, lse = c.run(False)
    c.ctx.check()
    assert not torch.isfinite(out[:n].float()).any() and not torch.isfinite(lse[:, :n]).any()
    assert torch.isfinite(out[n:].float()).all() and torch.isfinite(lse[:, n:]).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n", [1, 90])
def test_pages_and_lengths_out_of_range_are_reported(kind, n):
    """Nothing is read through them: the call ends, other samples are right, check() reports once."""
    good = case(kind, [n, n, n], [300, 310, 320], 4, 2, 64, 16)
    want, want_lse = good.run(True)
    good.compare(want, want_lse, True)

    def reported(change, spoilt, **kw):
        c = case(kind, [n, n, n], [300, 310, 320], 4, 2, 64, 16)
        change(c)
        out, lse = c.run(True, **kw)
        with pytest.raises(swam.SwamError) as e:
            c.ctx.check()
        assert e.value.code == swam.ERR_DEVICE_CHECK
        for b in range(3):
            if b not in spoilt:
                assert torch.equal(out[b * n:(b + 1) * n], want[b * n:(b + 1) * n])
        c.ctx.check()

    def set_(tensor, index, value):
        def change(c):
            getattr(c, tensor)[index] = value
        return change

    for value in (-1, 1 << 30, -(1 << 31), 10 ** 6):
        reported(set_("table", (1, 4), value), {1})
    reported(set_("kv_len", 1, -5), {1})
    reported(set_("kv_len", 2, 2 ** 31 - 1), {2})
    reported(set_("q_start", 3, 10 ** 9), {2})
    reported(set_("q_start", 0, -4), {0})
    reported(set_("q_start", 1, 2 ** 31 - 1), {0, 1})
    reported(lambda c: None, {2}, max_kv=315)
    if n > 1:
        reported(lambda c: None, {0, 1, 2}, max_q=n - 1)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n", [1, 100])
def test_graphs_streams_and_repeats_give_the_same_bits(kind, n):
    c = case(kind, [n] * 4, [900, 30 + n, 2000, n], 8, 2, 64, 16)
    want, want_lse = c.run(True)
    c.compare(want, want_lse, True)
    for _ in range(5):
        out, lse = c.run(True)
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        out, lse = c.run(True)
    # the same graph with other lengths, then with these again: the plan knows sizes only
    keep = c.kv_len.clone()
    c.kv_len.copy_(torch.tensor([n, 30 + n, 5, n], dtype=torch.int32))
    graph.replay()
    short = c.lens
    c.lens, keys, values = [n, 30 + n, 5, n], c.keys, c.values
    c.keys, c.values = [k[:m] for k, m in zip(keys, c.lens)], [v[:m] for v, m in zip(values, c.lens)]
    c.compare(out, lse, True)
    c.lens, c.keys, c.values = short, keys, values
    c.kv_len.copy_(keep)
    graph.replay()
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    # two calls at once on two streams, scratch of their own
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        o2, l2 = c.run(True)
    o1, l1 = c.run(True)
    torch.cuda.synchronize()
    assert torch.equal(o1, want) and torch.equal(o2, want) and torch.equal(l1, want_lse) and torch.equal(l2, want_lse)


@pytest.mark.parametrize("n", [1, 40])
def test_offsets_beyond_32_bits(n):
    """Pages so far apart that their elements' offsets pass 2^32 bytes and 2^31 elements."""
    kv, D, page = 8, 128, 64
    stride = 1 << 28                                             # elements between pages: 9 of them span 2^31
    store = torch.empty(9 * stride + page * kv * D, dtype=BF16, device="cuda")
    pages = store.as_strided((10, page, kv, D), (stride, kv * D, D, 1))
    gen = torch.Generator(device="cuda").manual_seed(3)
    for i in range(10):
        pages[i] = base.rand(gen, page, kv, D, dtype=BF16)
    small = pages.contiguous()
    table = torch.tensor([[9, 0, 8], [3, 9, 5]], dtype=torch.int32, device="cuda")
    kv_len = torch.tensor([150, 192], dtype=torch.int32, device="cuda")
    ctx = base.make_ctx(1, 16, D, kv, swam.BF16)
    q = base.rand(gen, 2 * n, 16, D, dtype=BF16)
    far = ctx.paged_attn(q, pages, pages, table, kv_len)
    near = ctx.paged_attn(q, small, small.clone(), table, kv_len)
    ctx.check()
    assert torch.equal(far, near)


def test_no_tokens():
    c = case(KINDS[0], [1, 1], [20, 30], 4, 2, 64, 16)
    before = c.ctx.launch_count()
    out, lse = c.ctx.paged_attn(c.q[:0], c.k_pages, c.v_pages, c.table, c.kv_len, want_lse=True)
    assert out.shape == (0, 4, 64) and lse.shape == (4, 0) and c.ctx.launch_count() == before


def test_refusals():
    c = case(KINDS[0], [1, 1], [20, 30], 4, 2, 64, 16)
    args = dict(q=c.q, k_pages=c.k_pages, v_pages=c.v_pages, page_table=c.table, kv_len=c.kv_len)

    def refused(error=ValueError, code=None, **kw):
        before = c.ctx.launch_count()
        with pytest.raises(error) as e:
            c.ctx.paged_attn(**{**args, **kw})
        if code is not None:
            assert e.value.code == code
        assert c.ctx.launch_count() == before

    refused(q=c.q.float())
    refused(q=c.q.cpu())
    refused(q=c.q[:, :2])
    refused(q=c.q[:, :1].expand(2, 4, 64))
    refused(q=c.q[None])
    refused(q=c.q[:1].expand(2, 4, 64))
    refused(v_pages=c.v_pages[:, :8])
    refused(k_pages=c.k_pages[..., :32], v_pages=c.v_pages[..., :32])
    refused(k_pages=c.k_pages[:, :, :0], v_pages=c.v_pages[:, :, :0])
    refused(page_table=c.table.long())
    refused(page_table=c.table[:1])
    refused(page_table=c.table.t().contiguous().t())
    refused(kv_len=c.kv_len.long())
    refused(kv_len=c.kv_len.cpu())
    refused(q_start=c.q_start[:2])
    refused(out=c.q[:1])
    refused(swam.SwamError, swam.ERR_INVALID_ARG, out=c.q)
    three = torch.zeros(5, 48, 2, 64, dtype=BF16, device="cuda")
    refused(swam.SwamError, swam.ERR_INVALID_ARG, k_pages=three, v_pages=three.clone())                  # 48 tokens a page
    refused(swam.SwamError, swam.ERR_INVALID_ARG, k_pages=three[:, :8], v_pages=three[:, :8])            # 8
    refused(swam.SwamError, swam.ERR_INVALID_ARG, k_pages=c.k_pages[:0], v_pages=c.v_pages[:0])          # no pages
    odd = torch.zeros(5, 16, 3, 64, dtype=BF16, device="cuda")
    refused(swam.SwamError, swam.ERR_INVALID_ARG, k_pages=odd, v_pages=odd.clone())                      # 3 heads for 4
    refused(swam.SwamError, swam.ERR_INVALID_ARG, q=torch.zeros(3, 4, 64, dtype=BF16, device="cuda"))    # 3 tokens, 2 samples, no q_start
    refused(swam.SwamError, swam.ERR_INVALID_ARG, max_q=-1)
    refused(swam.SwamError, swam.ERR_INVALID_ARG, max_kv=-1)

    # the C entry: pointers, strides, scratch
    lib, ctx = c.ctx.lib, c.ctx.ctx
    out = torch.empty_like(c.q)
    cache = c.ctx._cache(c.k_pages, c.v_pages, c.table, c.kv_len, None)

    def call(scratch=True, cache_fields=None, **fields):
        x = swam.SwamPagedCache.from_buffer_copy(cache)
        for name, value in (cache_fields or {}).items():
            setattr(x, name, value)
        a = swam.SwamPagedArgs(ctypes.addressof(x), c.q.data_ptr(), out.data_ptr(), None, None, 0, 2, 0, 0, 1, 0, 0)
        for name, value in fields.items():
            setattr(a, name, value)
        return lib.swam_paged_attn(ctx, ctypes.byref(a), None)

    assert call() == swam.OK
    torch.cuda.synchronize()
    before = c.ctx.launch_count()
    bad = swam.ERR_INVALID_ARG
    for fields in (dict(cache=None), dict(q=None), dict(out=None), dict(q=c.q.data_ptr() + 2), dict(out=out.data_ptr() + 8), dict(lse=out.data_ptr() + 2),
                   dict(n_tokens=-2), dict(q_token=-256), dict(q_token=128), dict(q_token=257), dict(out_token=1 << 39), dict(n_tokens=3),
                   dict(cache_fields=dict(kv_len=None)), dict(cache_fields=dict(page_table=None)), dict(cache_fields=dict(k=None)),
                   dict(cache_fields=dict(v=c.v_pages.data_ptr() + 4)), dict(cache_fields=dict(kv_len=c.kv_len.data_ptr() + 1)),
                   dict(cache_fields=dict(page_size=24)), dict(cache_fields=dict(page_size=0)), dict(cache_fields=dict(page_size=8)),
                   dict(cache_fields=dict(page_size=1 << 21)), dict(cache_fields=dict(n_samples=-1)), dict(cache_fields=dict(n_samples=0)),
                   dict(cache_fields=dict(n_pages=0)), dict(cache_fields=dict(max_pages=0)), dict(cache_fields=dict(reserved=1)),
                   dict(cache_fields=dict(n_kv_heads=3)), dict(cache_fields=dict(n_kv_heads=-2)), dict(cache_fields=dict(table_sample=1)),
                   dict(cache_fields=dict(k_token=64)), dict(cache_fields=dict(v_token=129)), dict(cache_fields=dict(k_page=1 << 39)),
                   dict(out=c.k_pages.data_ptr())):
        assert call(**fields) == bad, fields
    assert call(cache_fields=dict(max_pages=1 << 26)) == swam.ERR_UNSUPPORTED
    assert call(cache_fields=dict(n_samples=1 << 16)) == swam.ERR_UNSUPPORTED
    assert call(n_tokens=1 << 29) == swam.ERR_UNSUPPORTED
    # keys beyond 512 may be cut, which needs scratch
    x = swam.SwamPagedCache.from_buffer_copy(cache)
    x.max_pages, x.table_sample = 64, 64
    a = swam.SwamPagedArgs(ctypes.addressof(x), c.q.data_ptr(), out.data_ptr(), None, None, 0, 2, 0, 0, 1, 0, 0)
    need = ctypes.c_size_t()
    assert lib.swam_paged_attn_scratch_bytes(ctx, ctypes.byref(a), ctypes.byref(need)) == swam.OK and need.value > 0
    assert lib.swam_paged_attn(ctx, ctypes.byref(a), None) == swam.ERR_WORKSPACE
    buf = torch.empty(need.value + 512, dtype=torch.uint8, device="cuda")
    a.scratch, a.scratch_bytes = (buf.data_ptr() + 255) & ~255, need.value - 1
    assert lib.swam_paged_attn(ctx, ctypes.byref(a), None) == swam.ERR_WORKSPACE
    a.scratch, a.scratch_bytes = ((buf.data_ptr() + 255) & ~255) + 16, need.value
    assert lib.swam_paged_attn(ctx, ctypes.byref(a), None) == swam.ERR_WORKSPACE
    assert c.ctx.launch_count() == before
    unbound = swam.Swam(1, 16, 2, 64, 8, 4, 64, 14, 18, n_kv_heads=2, bind=False)
    with pytest.raises(swam.SwamError) as e:
        unbound.paged_attn(**args)
    assert e.value.code == swam.ERR_WORKSPACE

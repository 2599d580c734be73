"""What the operators around a paged key/value cache are measured on.

norm_rope: the step in front of the joint attention.  Every head of q and k is divided by the root of its mean square and
multiplied by a weight (optional), then the first `rot` of its elements are rotated, pair by pair, by angles that grow with
the token's position.  A pair is (i, i + rot/2), or (2i, 2i+1) when interleaved; pair i turns by freq[i] radians per position along
axis[i] of a position with one or three axes (frame, row, column).
    x' = x / sqrt(mean(x^2) + eps) * w;   (a, b) -> magnitude * (a cos - b sin, b cos + a sin)
append: the new tokens of a ragged batch go into a paged cache: k normalised and rotated on the way, v as it is, and q is
normalised and rotated for the attention that follows.  Token i of the n new ones of sample b is number kv_len[b] - n + i of the
sample, which is its position too; it lives in page page_table[b, number / page], row number % page.
paged: those queries attend the cache: query i of n sees the keys [0, kv_len[b]), with `causal` [0, kv_len[b] - n + i + 1).
    out = sum_c softmax_c(q . k_c / sqrt(dim)) v_c,   lse = ln sum_c exp(q . k_c / sqrt(dim))
A query that sees no key gives zeros and -inf.  Query head h reads key/value head h / (heads / kv_heads).
"""
import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_EPS = 1e-6


def _norm_rope(name, dtype, batch, n, heads, kv_heads, dim, rot, axes, interleaved, norm, factor, far):
    """`far`: the first position of the last sample (one axis); `factor`: how far beyond 4096 positions the angles are stretched."""
    c = dict(op="norm_rope", dtype=dtype, batch=batch, n=n, heads=heads, kv_heads=kv_heads, dim=dim, rot=rot, axes=axes,
             interleaved=interleaved, norm=norm, factor=factor, far=far)
    return c if name is None else dict(name=name, **c)


def _append(name, dtype, samples, n_lo, n_hi, heads, kv_heads, dim, page, past_lo, past_hi, rot, interleaved, norm):
    """New tokens spread evenly over n_lo .. n_hi and tokens before them over past_lo .. past_hi, one number per sample."""
    c = dict(op="append", dtype=dtype, samples=samples, n_lo=n_lo, n_hi=n_hi, heads=heads, kv_heads=kv_heads, dim=dim, page=page,
             past_lo=past_lo, past_hi=past_hi, rot=rot, interleaved=interleaved, norm=norm)
    return c if name is None else dict(name=name, **c)


def _paged(name, dtype, samples, n_lo, n_hi, heads, kv_heads, dim, page, past_lo, past_hi, causal):
    c = dict(op="paged", dtype=dtype, samples=samples, n_lo=n_lo, n_hi=n_hi, heads=heads, kv_heads=kv_heads, dim=dim, page=page,
             past_lo=past_lo, past_hi=past_hi, causal=causal)
    return c if name is None else dict(name=name, **c)


def listed():
    return [
        # the action tokens of one sample, replanned while the rest of the sequence stays: the smallest call
        _norm_rope("norm_rope_actions", "bf16", 1, 32, 24, 24, 64, 64, 1, False, True, 1.0, 2880),
        # the whole larger-imagination sequence, positions by frame, row and column
        _norm_rope("norm_rope_larger_imagination", "bf16", 1, 9280, 32, 32, 128, 128, 3, False, True, 1.0, 0),
        # the multi-view batch, grouped keys, half of each head rotated in neighbouring pairs: the largest
        _norm_rope("norm_rope_multi_view", "bf16", 8, 8672, 24, 8, 64, 32, 1, True, True, 1.0, 8672),
        # fp32 tensors, no norm, far positions of a stretched context, an odd number of tokens
        _norm_rope("norm_rope_f32_far", "f32", 3, 1001, 8, 2, 32, 24, 1, False, False, 32.0, 120000),
        # one new token for each of 64 robots: serving
        _append("append_single_tokens", "bf16", 64, 1, 1, 32, 8, 128, 16, 16, 2000, 128, False, True),
        # ragged chunks of observed tokens of 16 samples: prefilling histories
        _append("append_observations", "bf16", 16, 100, 1728, 24, 24, 64, 64, 0, 1728, 64, False, True),
        # fp32 tensors, interleaved pairs, small pages
        _append("append_f32", "f32", 5, 1, 77, 15, 5, 32, 32, 3, 500, 32, True, False),
        # one new token for each of 64 robots behind histories of very different lengths
        _paged("paged_single_tokens", "bf16", 64, 1, 1, 32, 8, 128, 16, 15, 8191, True),
        # one new token for two samples behind very long histories
        _paged("paged_long_history", "bf16", 2, 1, 1, 32, 8, 128, 64, 100000, 131071, True),
        # 16 action chunks of 64 tokens, which see one another, behind the observed and imagined tokens
        _paged("paged_action_chunks", "bf16", 16, 64, 64, 24, 24, 64, 32, 576, 8640, False),
        # ragged observation chunks, causal, behind histories: the largest
        _paged("paged_observations", "bf16", 8, 300, 2520, 32, 8, 128, 64, 0, 9216, True),
        # fp32 tensors, odd sizes
        _paged("paged_f32", "f32", 6, 1, 50, 15, 5, 64, 16, 10, 1500, True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    while True:
        heads, kv = rng.choice([(24, 24), (32, 32), (32, 8), (16, 16), (16, 2), (12, 4), (15, 5), (24, 8)])
        dim = rng.choice([32, 64, 64, 128, 128])
        rot = rng.choice([dim, dim, dim // 2, dim // 4, dim - 8])
        page = rng.choice([16, 32, 64, 128, 256])
        kind = rng.choice(["norm_rope", "append", "paged", "paged"])
        flags = [rng.random() < 0.5 for _ in range(2)]
        if kind == "norm_rope":
            axes = rng.choice([1, 1, 3])
            case = _norm_rope(None, dtype, _log_int(rng, 1, 8), _log_int(rng, 1, 9280), heads, kv, dim, rot, axes, flags[0], flags[1],
                              rng.choice([1.0, 4.0, 32.0]), rng.choice([0, _log_int(rng, 1, 131072)]))
        else:
            samples = _log_int(rng, 1, 64)
            n_hi = rng.choice([1, _log_int(rng, 1, 128), _log_int(rng, 16, 2520)])
            n_lo = rng.randint(1, n_hi)
            if kind == "append":
                past_hi = _log_int(rng, 1, 4000)
                case = _append(None, dtype, samples, n_lo, n_hi, heads, kv, dim, page, rng.randint(0, past_hi), past_hi, rot, flags[0],
                               flags[1])
            else:
                past_hi = _log_int(rng, 16, 131072)
                case = _paged(None, dtype, samples, n_lo, n_hi, heads, kv, dim, page, rng.randint(0, past_hi), past_hi, flags[0])
        # no more than the largest listed cases of the kind and type
        w = work(case)
        if kind != "paged" and w["bytes"] <= (3e7 if dtype == "f32" else 5e8):
            return case
        if kind == "paged" and w["flops"] <= (2e10 if dtype == "f32" else 8e11) and w["bytes"] <= 1.2e9:
            return case


def _spread(lo, hi, n):
    return [hi - (hi - lo) * i // max(1, n - 1) for i in range(n)]


def _lengths(case):
    """New tokens and tokens before them, per sample; the orders differ, so that long chunks meet short histories too."""
    n = case["samples"]
    new, past = _spread(case["n_lo"], case["n_hi"], n), _spread(case["past_lo"], case["past_hi"], n)
    return new, [past[(i * 7 + 3) % n] if math.gcd(7, n) == 1 else past[n - 1 - i] for i in range(n)]


def _frequencies(rot, axes, factor):
    """Radians per position of each pair, its axis, and the magnitude.  One axis: 10000^(-2i/rot), stretched by `factor` where a pair
    turns less than once in 4096 positions, not at all where it turns more than 32 times, in proportion between (Peng et
    al., YaRN, 2023).  Three axes: a quarter of the pairs for the frame, the rest for row and column, a ladder each."""
    half = rot // 2
    if axes == 3:
        frame = max(1, half // 4)
        row = max(1, (half - frame) // 2)
        sizes = [frame, row, half - frame - row]
    else:
        sizes = [half]
    freq, axis = [], []
    for a, size in enumerate(sizes):
        for i in range(size):
            f = 10000.0 ** (-i / size)
            turns = 4096 * f / (2 * math.pi)
            keep = min(1.0, max(0.0, (turns - 1) / 31))
            freq.append(f * (keep + (1 - keep) / factor))
            axis.append(a)
    return freq, axis, 1.0 if factor <= 1 else 0.1 * math.log(factor) + 1.0


def _rows(gen, shape, dtype):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)


def _weight(gen, dim):
    return 1.0 + 0.2 * torch.randn(dim, generator=gen, device="cuda", dtype=torch.float32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    host = torch.Generator()
    host.manual_seed(seed)
    dt, H, KV, D = _DTYPES[case["dtype"]], case["heads"], case["kv_heads"], case["dim"]
    s = {"case": case, "q_weight": None, "k_weight": None, "rope": None}
    if case["op"] != "paged":
        axes = case.get("axes", 1)
        s["freq"], s["axis"], s["magnitude"] = _frequencies(case["rot"], axes, case.get("factor", 1.0))
        if case["norm"]:
            s["q_weight"], s["k_weight"] = _weight(gen, D), _weight(gen, D)
    if case["op"] == "norm_rope":
        B, n = case["batch"], case["n"]
        # q and k as one projection writes them, read in place through their strides
        qkv = _rows(gen, (B, n, H + 2 * KV, D), dt)
        s["q"], s["k"] = qkv[:, :, :H], qkv[:, :, H:H + KV]
        first = torch.tensor(_spread(0, case["far"], B), dtype=torch.int32).flip(0).cuda()
        t = torch.arange(n, dtype=torch.int32, device="cuda")
        if case["axes"] == 3:
            side = 32
            grid = torch.stack([t // (side * side), t // side % side, t % side], dim=-1)
            s["positions"] = (grid[None] + first[:, None, None]).contiguous()
        else:
            s["positions"] = (first[:, None] + t)[:, :, None].contiguous()
    else:
        new, past = _lengths(case)
        order = torch.randperm(case["samples"], generator=host).tolist()
        new, past = [new[i] for i in order], [past[i] for i in order]
        page, total = case["page"], sum(new)
        kv_len = [a + b for a, b in zip(new, past)]
        pages = [(n + page - 1) // page for n in kv_len]
        n_pages = sum(pages) + 3
        # pages come from a pool in no order; table entries behind a sample's last page name none
        free = torch.randperm(n_pages, generator=host, dtype=torch.int32)
        table = torch.full((len(new), max(pages)), -1, dtype=torch.int32)
        at = 0
        for b, m in enumerate(pages):
            table[b, :m] = free[at:at + m]
            at += m
        starts = [0]
        for n in new:
            starts.append(starts[-1] + n)
        s["new"], s["past"] = new, past
        s["page_table"] = table.cuda()
        s["kv_len"] = torch.tensor(kv_len, dtype=torch.int32).cuda()
        s["q_start"] = torch.tensor(starts, dtype=torch.int32).cuda()
        s["sample"] = torch.repeat_interleave(torch.arange(len(new)), torch.tensor(new)).cuda()
        s["k_pages"] = _rows(gen, (n_pages, page, KV, D), dt)
        s["v_pages"] = _rows(gen, (n_pages, page, KV, D), dt)
        if case["op"] == "append":
            qkv = _rows(gen, (total, H + 2 * KV, D), dt)
            s["q"], s["k"], s["v"] = qkv[:, :H], qkv[:, H:H + KV], qkv[:, H + KV:]
        else:
            # normalised queries and keys with a few strong matches: logits of a trained layer spread over several units
            s["q"] = _rows(gen, (total, H, D), dt) * 1.5
    if own:
        from paper_2609_38984_b200 import swam
        # the layer's context: its joint sequence does not matter to these calls, its heads and type do
        s["ctx"] = swam.Swam(case.get("batch", 1), 16, 2, 64, 8, H, D, 14, 18, n_kv_heads=KV,
                             dtype=swam.F32 if case["dtype"] == "f32" else swam.BF16)
        if case["op"] != "paged":
            s["rope"] = swam.Rope(s["freq"], axes=s["axis"], interleaved=case["interleaved"], magnitude=s["magnitude"])
    return s


def _angles(s, positions):
    """positions [..., axes] -> cos and sin [..., 1, pairs] in 32 bits, from angles in 64."""
    freq = torch.tensor(s["freq"], dtype=torch.float64, device=positions.device)
    axis = torch.tensor(s["axis"], device=positions.device)
    a = (positions.double()[..., axis] * freq).unsqueeze(-2)
    return (torch.cos(a) * s["magnitude"]).float(), (torch.sin(a) * s["magnitude"]).float()


def _normed_rotated(s, x, weight, cos, sin):
    c = s["case"]
    y = x.float()
    if weight is not None:
        y = y * torch.rsqrt(y.square().mean(dim=-1, keepdim=True) + _EPS) * weight
    rot = c["rot"]
    head, rest = y[..., :rot], y[..., rot:]
    if c["interleaved"]:
        a, b = head[..., 0::2], head[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    else:
        a, b = head[..., :rot // 2], head[..., rot // 2:]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    return torch.cat([turned, rest], dim=-1).to(x.dtype)


def _numbers(s):
    """Number of each new token in its sample."""
    return s["kv_len"].long()[s["sample"]] - s["q_start"].long()[s["sample"] + 1] + torch.arange(s["sample"].numel(), device="cuda")


def _plain_paged(s):
    c = s["case"]
    q, H, KV, D, page = s["q"], c["heads"], c["kv_heads"], c["dim"], c["page"]
    g, total = H // KV, s["q"].shape[0]
    out = torch.empty_like(q)
    lse = torch.empty(H, total, dtype=torch.float32, device=q.device)
    at = 0
    for b, n in enumerate(s["new"]):
        length = s["past"][b] + n
        pages = s["page_table"][b, :(length + page - 1) // page].long()
        k = s["k_pages"][pages].flatten(0, 1)[:length].float().transpose(0, 1)        # [KV, length, D]
        v = s["v_pages"][pages].flatten(0, 1)[:length].float().transpose(0, 1)
        rows = q[at:at + n].float().reshape(n, KV, g, D).permute(1, 0, 2, 3).reshape(KV, n * g, D)
        step = max(1, int(2e9) // (n * g * length))                                     # key/value heads at a time
        for h in range(0, KV, step):
            x = torch.matmul(rows[h:h + step], k[h:h + step].transpose(1, 2)) * (1.0 / math.sqrt(D))
            if c["causal"]:
                last = (length - n + torch.arange(n, device=q.device)).repeat_interleave(g)
                x = torch.where(torch.arange(length, device=q.device)[None, :] <= last[:, None], x, torch.full_like(x, -math.inf))
            m = x.amax(dim=-1, keepdim=True)
            m = torch.where(m == -math.inf, torch.zeros_like(m), m)
            p = torch.exp(x - m)
            sums = p.sum(dim=-1, keepdim=True)
            o = torch.matmul(p, v[h:h + step]) / torch.where(sums > 0, sums, torch.ones_like(sums))
            m_ = o.shape[0]
            out[at:at + n, h * g:(h + m_) * g] = o.reshape(m_, n, g, D).transpose(0, 1).reshape(n, m_ * g, D).to(q.dtype)
            e = (m + torch.log(sums)).squeeze(-1)
            lse[h * g:(h + m_) * g, at:at + n] = e.reshape(m_, n, g).transpose(1, 2).reshape(m_ * g, n)
        at += n
    return out, lse


def run(state):
    s, c = state, state["case"]
    if own:
        if c["op"] == "norm_rope":
            return s["ctx"].norm_rope(s["q"], s["k"], s["rope"], positions=s["positions"], q_weight=s["q_weight"],
                                      k_weight=s["k_weight"], eps=_EPS)
        if c["op"] == "append":
            q = s["ctx"].append_kv(s["k"], s["v"], s["k_pages"], s["v_pages"], s["page_table"], s["kv_len"], q_start=s["q_start"],
                                   q=s["q"], rope=s["rope"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=_EPS)
            return q, s["k_pages"], s["v_pages"]
        return s["ctx"].paged_attn(s["q"], s["k_pages"], s["v_pages"], s["page_table"], s["kv_len"], q_start=s["q_start"],
                                   max_q=c["n_hi"], causal=c["causal"], want_lse=True)
    if c["op"] == "norm_rope":
        cos, sin = _angles(s, s["positions"])
        return _normed_rotated(s, s["q"], s["q_weight"], cos, sin), _normed_rotated(s, s["k"], s["k_weight"], cos, sin)
    if c["op"] == "append":
        number = _numbers(s)
        cos, sin = _angles(s, number[:, None])
        where = s["page_table"].long()[s["sample"], number // c["page"]], number % c["page"]
        s["k_pages"][where] = _normed_rotated(s, s["k"], s["k_weight"], cos, sin)
        s["v_pages"][where] = s["v"]
        return _normed_rotated(s, s["q"], s["q_weight"], cos, sin), s["k_pages"], s["v_pages"]
    return _plain_paged(s)


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    H, KV, D = case["heads"], case["kv_heads"], case["dim"]
    if case["op"] == "norm_rope":
        tokens = case["batch"] * case["n"]
        elements = tokens * (H + KV) * D
        return {"bytes": 2 * elements * size + 4 * tokens * case["axes"],
                "flops": elements * (4 if case["norm"] else 0) + 3 * tokens * (H + KV) * case["rot"]}
    new, past = _lengths(case)
    tokens = sum(new)
    if case["op"] == "append":
        turned = tokens * (H + KV) * D
        return {"bytes": 2 * tokens * (H + 2 * KV) * D * size + 16 * len(new),
                "flops": turned * (4 if case["norm"] else 0) + 3 * tokens * (H + KV) * case["rot"]}
    pairs = sum(n * (m + n) - (n * (n - 1) // 2 if case["causal"] else 0) for n, m in zip(new, past))
    return {"bytes": 2 * sum(n + m for n, m in zip(new, past)) * KV * D * size + 2 * tokens * H * D * size + 4 * tokens * H,
            "flops": 4 * pairs * H * D}


def _exact_turned(x, weight, angle, s):
    """x [tokens, heads, D], angle [tokens, pairs]: each pair as a complex number, multiplied by one on the circle."""
    c = s["case"]
    y = x.double()
    if weight is not None:
        y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / y.shape[-1] + _EPS) * weight.double()
    i = torch.arange(c["rot"] // 2, device=x.device)
    first, second = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + c["rot"] // 2)
    z = torch.complex(y[..., first], y[..., second]) * (s["magnitude"] * torch.exp(1j * angle))[:, None]
    y = y.clone()
    y[..., first], y[..., second] = z.real, z.imag
    return y


def exact(case, seed):
    """The definitions, in 64 bits: attention a sample and a head at a time."""
    s = prepare(case, seed)
    H, KV, D = case["heads"], case["kv_heads"], case["dim"]
    if case["op"] == "norm_rope":
        freq = torch.tensor(s["freq"], dtype=torch.float64, device="cuda")
        angle = s["positions"].double().flatten(0, 1)[:, s["axis"]] * freq
        return tuple(_exact_turned(s[x].flatten(0, 1), s[x + "_weight"], angle, s).view(s[x].shape) for x in "qk")
    if case["op"] == "append":
        freq = torch.tensor(s["freq"], dtype=torch.float64, device="cuda")
        number = torch.cat([torch.arange(m, m + n) for n, m in zip(s["new"], s["past"])]).cuda()
        angle = number.double()[:, None] * freq
        k_pages, v_pages = s["k_pages"].double(), s["v_pages"].double()
        k = _exact_turned(s["k"], s["k_weight"], angle, s)
        at, table = 0, s["page_table"].tolist()
        for b, n in enumerate(s["new"]):
            m = s["past"][b]
            while n > 0:                                        # the stretch up to the end of a page
                row = m % case["page"]
                step = min(n, case["page"] - row)
                k_pages[table[b][m // case["page"]], row:row + step] = k[at:at + step]
                v_pages[table[b][m // case["page"]], row:row + step] = s["v"][at:at + step].double()
                m, n, at = m + step, n - step, at + step
        return _exact_turned(s["q"], s["q_weight"], angle, s), k_pages, v_pages
    if len(s["new"]) * H > 4096:
        return None
    total, page, table = sum(s["new"]), case["page"], s["page_table"].tolist()
    out = torch.zeros(total, H, D, dtype=torch.float64, device="cuda")
    lse = torch.full((H, total), -math.inf, dtype=torch.float64, device="cuda")
    at = 0
    for b, n in enumerate(s["new"]):
        length = s["past"][b] + n
        ids = table[b][:(length + page - 1) // page]
        for h in range(H):
            k = s["k_pages"][ids, :, h * KV // H].reshape(-1, D)[:length].double()
            v = s["v_pages"][ids, :, h * KV // H].reshape(-1, D)[:length].double()
            logits = (s["q"][at:at + n, h].double() @ k.T) / D ** 0.5
            if case["causal"]:
                behind = torch.arange(length, device="cuda")[None] - torch.arange(length - n, length, device="cuda")[:, None]
                logits.masked_fill_(behind > 0, -math.inf)
            e = torch.logsumexp(logits, dim=1)
            out[at:at + n, h] = torch.exp(logits - e[:, None]) @ v
            lse[h, at:at + n] = e
        at += n
    return out, lse

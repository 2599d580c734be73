"""What the two attention operators with keys outside the joint sequence are measured on.

Cross attention: every query of a sample attends an encoder's states of another length (the instruction's text states, for
instance), of which the first kv_len[b] of sample b are real and the rest is padding:
    out[b,t,h] = sum_c softmax_c(scale q[b,t,h] . k[b,c,h']) v[b,c,h'],   c < kv_len[b],   h' = h / (n_heads / n_kv_heads)
Prefix attention: samples that share a long prefix (the same observation, denoised into several candidate chunks) attend
that prefix's keys, which exist once per group of samples, and keys of their own behind it; with `causal` the query t of
n_q sees its own keys up to own_len[b] - n_q + t only.
A row that sees no key gives zeros and a log-sum-exp of -inf.  Both return (out, lse), lse [B, n_heads, n_q] in natural-log
units.
"""
import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _cross(name, dtype, batch, n_q, heads, kv_heads, dim, n_kv, lo):
    """Encoder lengths spread evenly over lo .. n_kv, one per sample."""
    c = dict(op="cross", dtype=dtype, batch=batch, n_q=n_q, heads=heads, kv_heads=kv_heads, dim=dim, n_kv=n_kv, lo=lo)
    return c if name is None else dict(name=name, **c)


def _prefix(name, dtype, batch, groups, n_q, heads, kv_heads, dim, n_prefix, n_own, lo, causal):
    """Prefixes of full length, own lengths spread evenly over lo .. n_own, one per sample."""
    c = dict(op="prefix", dtype=dtype, batch=batch, groups=groups, n_q=n_q, heads=heads, kv_heads=kv_heads, dim=dim,
             n_prefix=n_prefix, n_own=n_own, lo=lo, causal=causal)
    return c if name is None else dict(name=name, **c)


def listed():
    return [
        # the action tokens of one sample read a short instruction: the smallest call, all latency
        _cross("cross_actions_short_text", "bf16", 1, 32, 24, 24, 64, 77, 77),
        # one new token for each of 16 robots against its own encoder output (grouped-query heads): serving
        _cross("cross_single_tokens", "bf16", 16, 1, 32, 8, 128, 1500, 300),
        # every token of the single-view joint sequence reads a padded text of 512 states
        _cross("cross_single_view", "bf16", 1, 2912, 24, 24, 64, 512, 512),
        # guided denoising at the larger-imagination shape: the conditional sample has a text, the unconditional one none
        _cross("cross_guided_larger_imagination", "bf16", 2, 9280, 32, 32, 128, 1024, 0),
        # the multi-view batch, eight instructions of different lengths: the largest cross attention
        _cross("cross_multi_view", "bf16", 8, 8672, 24, 24, 64, 512, 64),
        # fp32 tensors, odd sizes
        _cross("cross_f32", "f32", 4, 1000, 8, 8, 64, 333, 100),
        # one new token for each of 64 samples behind one shared observation history
        _prefix("prefix_single_tokens", "bf16", 64, 1, 1, 32, 8, 128, 8192, 1024, 16, False),
        # one new token for each of 16 samples behind a very long history
        _prefix("prefix_long_history", "bf16", 16, 1, 1, 32, 8, 128, 131072, 300, 1, False),
        # 16 candidate action chunks, causal among themselves, behind the observed and imagined tokens they all share
        _prefix("prefix_action_chunks", "bf16", 16, 1, 64, 32, 32, 128, 9216, 64, 64, True),
        # eight candidates of a sparse step at the single-view shape: two observations, four candidates each
        _prefix("prefix_sparse_step", "bf16", 8, 2, 608, 24, 24, 64, 576, 608, 608, False),
        # four candidates of a sparse step at the larger-imagination shape: the largest prefix attention
        _prefix("prefix_sparse_step_large", "bf16", 4, 1, 2520, 32, 32, 128, 1024, 2520, 2520, False),
        # fp32 tensors, odd sizes, grouped-query heads
        _prefix("prefix_f32", "f32", 6, 2, 24, 8, 2, 32, 1001, 130, 7, True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _heads(rng):
    heads, kv = rng.choice([(24, 24), (32, 32), (32, 8), (16, 16), (16, 2), (12, 4), (15, 5)])
    return heads, kv, rng.choice([32, 64, 64, 128, 128])


def draw(rng):
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    while True:
        heads, kv, dim = _heads(rng)
        if rng.random() < 0.5:
            batch = _log_int(rng, 1, 16)
            n_q = rng.choice([1, _log_int(rng, 1, 128), _log_int(rng, 64, 9280)])
            n_kv = _log_int(rng, 1, 1500)
            case = _cross(None, dtype, batch, n_q, heads, kv, dim, n_kv, rng.randint(0, n_kv))
        else:
            groups = rng.choice([1, 1, 2, 3])
            batch = groups * _log_int(rng, 1, 32)
            n_q = rng.choice([1, _log_int(rng, 1, 64), _log_int(rng, 16, 2520)])
            n_prefix = _log_int(rng, 16, 131072)
            n_own = _log_int(rng, 1, 2520)
            causal = rng.random() < 0.5
            case = _prefix(None, dtype, batch, groups, n_q, heads, kv, dim, n_prefix, n_own, rng.randint(0, n_own), causal)
        w = work(case)
        # no more work than the largest listed case of the type, and a plain form that stays within seconds
        pairs = _pairs(case)[0] * heads
        if w["flops"] <= (2e10 if dtype == "f32" else 5e11) and w["bytes"] <= 6e8 and pairs <= 1.2e9:
            return case


def _spread(lo, hi, n):
    return [hi - (hi - lo) * i // max(1, n - 1) for i in range(n)]


def _rows(gen, shape, dtype):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    host = torch.Generator()
    host.manual_seed(seed)
    dt, B, D = _DTYPES[case["dtype"]], case["batch"], case["dim"]
    s = {"case": case}
    # normalised queries and keys with a few strong matches: logits of a trained layer spread over several units
    s["q"] = _rows(gen, (B, case["n_q"], case["heads"], D), dt) * 1.5
    hi = case["n_kv"] if case["op"] == "cross" else case["n_own"]
    lens = torch.tensor(_spread(case["lo"], hi, B), dtype=torch.int32)[torch.randperm(B, generator=host)].cuda()
    if case["op"] == "cross":
        # keys and values as one projection writes them: interleaved per state, read in place through their strides
        kv = _rows(gen, (B, case["n_kv"], 2, case["kv_heads"], D), dt)
        s["k"], s["v"], s["kv_len"] = kv[:, :, 0], kv[:, :, 1], lens
    else:
        G = case["groups"]
        s["k_prefix"] = _rows(gen, (G, case["n_prefix"], case["kv_heads"], D), dt)
        s["v_prefix"] = _rows(gen, (G, case["n_prefix"], case["kv_heads"], D), dt)
        s["k"] = _rows(gen, (B, case["n_own"], case["kv_heads"], D), dt)
        s["v"] = _rows(gen, (B, case["n_own"], case["kv_heads"], D), dt)
        s["own_len"] = lens
    if own:
        from paper_2609_38984_b200 import swam
        # the layer's context: its joint sequence does not matter to these calls, its batch, heads and type do
        s["ctx"] = swam.Swam(B, 16, 2, 64, 8, case["heads"], D, 14, 18, n_kv_heads=case["kv_heads"],
                             dtype=swam.F32 if case["dtype"] == "f32" else swam.BF16)
    return s


def _plain(q, keys, values, seen):
    """q [N, R, D]; keys, values [N, C, D] fp32; seen [N, R, C] truth values: softmax attention and its log-sum-exp."""
    x = torch.matmul(q, keys.transpose(1, 2)) * (1.0 / math.sqrt(q.shape[-1]))
    x = torch.where(seen, x, torch.full_like(x, -math.inf))
    m = x.amax(dim=-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = torch.exp(x - m)
    total = p.sum(dim=-1, keepdim=True)
    out = torch.matmul(p, values) / torch.where(total > 0, total, torch.ones_like(total))
    return out, (m + torch.log(total)).squeeze(-1)


def run(state):
    c = state["case"]
    if own:
        if c["op"] == "cross":
            return state["ctx"].cross_attn(state["q"], state["k"], state["v"], kv_len=state["kv_len"], want_lse=True)
        return state["ctx"].prefix_attn(state["q"], state["k_prefix"], state["v_prefix"], state["k"], state["v"],
                                        own_len=state["own_len"], causal=c["causal"], want_lse=True)
    q = state["q"]
    B, n_q, H, D = q.shape
    n_kv_heads = c["kv_heads"]
    g = H // n_kv_heads
    out = torch.empty_like(q)
    lse = torch.empty(B, H, n_q, dtype=torch.float32, device=q.device)
    t = torch.arange(n_q, device=q.device).repeat_interleave(g)          # the query of each (query, head of the group) row
    for h in range(n_kv_heads):
        rows = q[:, :, h * g:(h + 1) * g].float().reshape(B, n_q * g, D)
        k, v = state["k"][:, :, h].float(), state["v"][:, :, h].float()
        pos = torch.arange(k.shape[1], device=q.device)
        if c["op"] == "cross":
            limit = state["kv_len"][:, None].expand(B, n_q * g)
        else:
            limit = state["own_len"][:, None].expand(B, n_q * g)
            if c["causal"]:
                limit = limit - n_q + 1 + t[None, :]
        seen = pos[None, None, :] < limit[:, :, None]
        if c["op"] == "prefix":
            per = B // c["groups"]
            k = torch.cat([state["k_prefix"][:, :, h].float().repeat_interleave(per, 0), k], dim=1)
            v = torch.cat([state["v_prefix"][:, :, h].float().repeat_interleave(per, 0), v], dim=1)
            seen = torch.cat([torch.ones(B, n_q * g, c["n_prefix"], dtype=torch.bool, device=q.device), seen], dim=2)
        o, e = _plain(rows, k, v, seen)
        out[:, :, h * g:(h + 1) * g] = o.reshape(B, n_q, g, D).to(q.dtype)
        lse[:, h * g:(h + 1) * g] = e.reshape(B, n_q, g).transpose(1, 2)
    return out, lse


def _pairs(case):
    """(query, key) pairs per head and the number of real keys per key/value head."""
    lens = _spread(case["lo"], case["n_kv"] if case["op"] == "cross" else case["n_own"], case["batch"])
    if case["op"] == "cross":
        return case["n_q"] * sum(lens), sum(lens)
    pairs = case["batch"] * case["n_q"] * case["n_prefix"]
    for n in lens:
        if case["causal"]:
            pairs += sum(max(0, n - case["n_q"] + 1 + t) for t in range(case["n_q"]))
        else:
            pairs += case["n_q"] * n
    return pairs, case["groups"] * case["n_prefix"] + sum(lens)


def work(case):
    pairs, keys = _pairs(case)
    size = 4 if case["dtype"] == "f32" else 2
    rows = case["batch"] * case["n_q"] * case["heads"]
    return {"bytes": 2 * keys * case["kv_heads"] * case["dim"] * size + 2 * rows * case["dim"] * size + 4 * rows,
            "flops": 4 * pairs * case["heads"] * case["dim"]}


def exact(case, seed):
    """The definition, one sample and head at a time over the keys that are really there, in 64 bits."""
    s = prepare(case, seed)
    q = s["q"].double()
    B, n_q, H, D = q.shape
    if B * H > 4096:
        return None
    out = torch.zeros(B, n_q, H, D, dtype=torch.float64, device=q.device)
    lse = torch.full((B, H, n_q), -math.inf, dtype=torch.float64, device=q.device)
    lens = (s["kv_len"] if case["op"] == "cross" else s["own_len"]).tolist()
    for b in range(B):
        for h in range(H):
            hk = h * case["kv_heads"] // H
            k, v = s["k"][b, :lens[b], hk].double(), s["v"][b, :lens[b], hk].double()
            ahead = 0
            if case["op"] == "prefix":
                gi = b * case["groups"] // B
                k, v = torch.cat([s["k_prefix"][gi, :, hk].double(), k]), torch.cat([s["v_prefix"][gi, :, hk].double(), v])
                ahead = case["n_prefix"]
            if k.shape[0] == 0:
                continue
            logits = (q[b, :, h] @ k.T) / D ** 0.5
            if case["op"] == "prefix" and case["causal"]:
                # the last key that each query sees; the prefix is before every query
                last = ahead + (lens[b] - n_q + torch.arange(n_q, device=q.device)).clamp(min=-1)
                logits.masked_fill_(torch.arange(k.shape[0], device=q.device)[None] > last[:, None], -math.inf)
            e = torch.logsumexp(logits, dim=1)
            weights = torch.exp(logits - torch.where(torch.isinf(e), torch.zeros_like(e), e)[:, None])
            out[b, :, h] = weights @ v
            lse[b, h] = e
    return out, lse

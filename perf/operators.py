"""Cases of the operators that fill the paged cache and draw tokens: what is
timed and compared for rotary append, chunk attention and sampling.

A prompt reaches the cache in chunks (``simsd_rope_append``), every chunk
attends to all that is cached (``simsd_chunk_attention``), and drafts are
drawn from logits (``simsd_sample``).  ``run`` makes one of these calls, or
with ``own`` false computes the same thing from elementary torch operations.
"""
import math
import random

import torch

own = False

#: head shapes of the SDAR layers (query heads, KV heads, head dimension)
HEADS = {"1.7B": (16, 8, 128), "4B": (32, 8, 128)}
VOCAB = 151936  # the SDAR vocabulary


def _lengths(n, lo, hi, salt):
    """n whole numbers in [lo, hi], the same for every seed (so that a case
    has one amount of work); both ends occur where n allows it."""
    r = random.Random(1000003 * salt + 8191 * lo + hi + n)
    v = [lo + round((hi - lo) * i / max(1, n - 1)) for i in range(n)] if n > 1 else [hi]
    r.shuffle(v)
    return v


def listed():
    return [
        # one token of each of eight sequences in fp32: the smallest append of a decoding loop
        dict(name="append single f32", op="append", dtype="f32", seqs=8, lo=1, hi=1, prefix_lo=512, prefix_hi=1024,
             Hq=16, Hkv=8, d=64, page=16, layout="interleaved", rot=32, scaling="linear", fused=False),
        # a batch of long prompt chunks in a context stretched four times, cut out of one projection's output
        dict(name="append chunks bf16", op="append", dtype="bf16", seqs=8, lo=1501, hi=2600, prefix_lo=0,
             prefix_hi=8192, Hq=32, Hkv=8, d=128, page=64, layout="half", rot=128, scaling="yarn", fused=True),
        # token by token decoding of a small batch at the 1.7B heads: latency
        dict(name="attend single few", op="attend", dtype="bf16", seqs=8, lo=1, hi=1, prefix_lo=512, prefix_hi=1024,
             Hq=16, Hkv=8, d=128, page=64, block=1, window=0, skip=0, lse=False),
        # token by token decoding of a full batch: reading the cache is all there is
        dict(name="attend single many", op="attend", dtype="bf16", seqs=64, lo=1, hi=1, prefix_lo=2048,
             prefix_hi=8192, Hq=32, Hkv=8, d=128, page=64, block=1, window=0, skip=0, lse=False),
        # the model's own block decoding: 16 tokens that see each other and 4096 cached ones
        dict(name="attend blocks of 16", op="attend", dtype="bf16", seqs=32, lo=16, hi=16, prefix_lo=4096,
             prefix_hi=4096, Hq=32, Hkv=8, d=128, page=64, block=16, window=0, skip=0, lse=False),
        # a whole prompt at once, causal, nothing cached before it
        dict(name="attend prompt 8192", op="attend", dtype="bf16", seqs=1, lo=8192, hi=8192, prefix_lo=0,
             prefix_hi=0, Hq=32, Hkv=8, d=128, page=64, block=1, window=0, skip=0, lse=False),
        # the last chunk of a long prompt, block-causal, over a long cache
        dict(name="attend chunk over 32768", op="attend", dtype="bf16", seqs=1, lo=2048, hi=2048, prefix_lo=32768,
             prefix_hi=32768, Hq=32, Hkv=8, d=128, page=64, block=32, window=0, skip=0, lse=False),
        # a mixed batch: odd lengths, seven query heads to a KV head, small pages and heads, a window, and
        # sequences whose first cached rows (for some all that a token could see) are hidden
        dict(name="attend ragged window", op="attend", dtype="bf16", seqs=13, lo=1, hi=777, prefix_lo=0,
             prefix_hi=2500, Hq=28, Hkv=4, d=64, page=16, block=1, window=1000, skip=1, lse=True),
        # the fp32 path at odd lengths, for a user who checks a model in full precision
        dict(name="attend f32", op="attend", dtype="f32", seqs=3, lo=45, hi=203, prefix_lo=0, prefix_hi=1003, Hq=8,
             Hkv=2, d=128, page=32, block=4, window=0, skip=0, lse=True),
        # the next token of a few sequences: latency
        dict(name="sample few", op="sample", dtype="f32", rows=8, vocab=VOCAB, spread=3.0, k=50, p=0.95, min_p=0.0,
             dist=False),
        # every masked position of a full batch in one denoising step (64 sequences of 16)
        dict(name="sample blocks", op="sample", dtype="f32", rows=1024, vocab=VOCAB, spread=2.0, k=0, p=0.9,
             min_p=0.0, dist=False),
        # drafts with the distribution that they are drawn from, as stochastic acceptance wants it; odd vocabulary
        dict(name="sample with distribution", op="sample", dtype="bf16", rows=132, vocab=32003, spread=3.0, k=1000,
             p=0.98, min_p=0.001, dist=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49))))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "sample"])
    if op == "sample":
        vocab = _log(rng, 1000, VOCAB)
        rows = _log(rng, 1, min(2000, 1024 * VOCAB // vocab))
        return dict(op=op, dtype=rng.choice(["f32", "f32", "bf16"]), rows=rows, vocab=vocab,
                    spread=rng.choice([2.0, 3.0, 4.0]), k=rng.choice([0, 0, _log(rng, 1, 1000)]),
                    p=rng.choice([1.0, rng.choice([0.8, 0.9, 0.95, 0.99])]), min_p=rng.choice([0.0, 0.0, 0.01, 0.1]),
                    dist=rng.random() < 0.3)
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    Hq, Hkv, d = rng.choice([(16, 8, 128), (32, 8, 128), (32, 8, 64), (28, 4, 64), (8, 8, 128), (40, 8, 128)])
    hi = rng.choice([1, _log(rng, 2, 64), _log(rng, 65, 4096)])
    lo = rng.choice([hi, max(1, hi // 3)])
    seqs = _log(rng, 1, max(1, min(64, (4096 if op == "attend" else 16384) // hi)))
    prefix_hi = rng.choice([0, _log(rng, 16, 8192 if hi * seqs > 512 else 32768)])
    # fp32 runs without tensor cores: a sixteenth of the tokens
    if dtype == "f32" and op == "attend":
        hi, lo, seqs = max(1, hi // 8), max(1, lo // 8), max(1, seqs // 2)
    # the pool of a drawn case stays below 8 GB
    while seqs > 1 and seqs * (prefix_hi + hi) * Hkv * d > (1 << 30):
        seqs //= 2
    case = dict(op=op, dtype=dtype, seqs=seqs, lo=lo, hi=hi, prefix_lo=prefix_hi // 4, prefix_hi=prefix_hi, Hq=Hq,
                Hkv=Hkv, d=d, page=rng.choice([16, 64, 64, 128]))
    if op == "append":
        return dict(case, layout=rng.choice(["half", "interleaved"]), rot=rng.choice([d, d, d // 2, 24]),
                    scaling=rng.choice(["none", "linear", "ntk", "yarn"]), fused=rng.random() < 0.5)
    window = rng.choice([0, 0, 0, _log(rng, 16, 4096)])
    return dict(case, block=rng.choice([1, 1, 4, 16, 32, 0]), window=window, skip=int(rng.random() < 0.25),
                lse=rng.random() < 0.5)


# ------------------------------------------------------------------ inputs
ROPE = dict(theta=1.0e6, factor=4.0, context=8192, beta_fast=32.0, beta_slow=1.0)


class State:
    pass


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _normal(shape, gen, dtype, std):
    return torch.randn(shape, generator=gen, device="cuda").mul_(std).to(dtype)


def prepare(case, seed):
    s = State()
    s.case = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if case["op"] == "sample":
        _prepare_sample(s, case, gen)
    else:
        _prepare_cache(s, case, seed, gen)
    if own:
        from paper_2606_02544_gb300 import simsd
        s.err = torch.zeros(1, dtype=torch.int32, device="cuda")
        if case["op"] == "append":
            s.plan = simsd.simsd_rope_plan_init(case["layout"], case["rot"], ROPE["theta"], case["scaling"],
                                                factor=ROPE["factor"], context=ROPE["context"],
                                                beta_fast=ROPE["beta_fast"], beta_slow=ROPE["beta_slow"])
        elif case["op"] == "attend":
            n = simsd.simsd_chunk_workspace_bytes(simsd.SIMSD_F32 if case["dtype"] == "f32" else simsd.SIMSD_BF16,
                                                  s.q.shape[0], case["seqs"], case["Hq"], case["Hkv"], case["d"],
                                                  s.table.shape[1], case["page"])
            s.ws = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
    return s


def _prepare_cache(s, case, seed, gen):
    """Chunks of new tokens, a page pool in random order with spare pages,
    and per sequence the rows cached before the chunk."""
    dt, n, P = _dtype(case), case["seqs"], case["page"]
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    s.chunk = _lengths(n, case["lo"], case["hi"], 1)
    s.prefix = _lengths(n, case["prefix_lo"], case["prefix_hi"], 2)
    start = [0]
    for c in s.chunk:
        start.append(start[-1] + c)
    T = start[-1]
    pages = [(p + c + P - 1) // P for p, c in zip(s.prefix, s.chunk)]
    pool = sum(pages) + 3
    perm = torch.randperm(pool, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    table = torch.full((n, max(pages)), -1, dtype=torch.int32)
    at = 0
    for b, c in enumerate(pages):
        table[b, :c] = perm[at:at + c]
        at += c
    i32 = dict(dtype=torch.int32, device="cuda")
    s.start = torch.tensor(start, **i32)
    s.prefix_len = torch.tensor(s.prefix, **i32)
    s.table = table.cuda()
    s.k_cache = _normal((pool, Hkv, P, d), gen, dt, 1.0)
    s.v_cache = _normal((pool, Hkv, P, d), gen, dt, 1.0)
    # what the plain form indexes with: sequence and offset of every token
    s.seq = torch.repeat_interleave(torch.arange(n), torch.tensor(s.chunk)).cuda()
    s.off = (torch.arange(T) - torch.tensor(start)[s.seq.cpu()]).cuda()
    if case["op"] == "append":
        if case["fused"]:  # q, k and v are parts of one projection's rows
            qkv = _normal((T, Hq + 2 * Hkv, d), gen, dt, 1.0)
            s.q, s.k, s.v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        else:
            s.q, s.k, s.v = (_normal((T, h, d), gen, dt, 1.0) for h in (Hq, Hkv, Hkv))
        s.q_out = torch.empty((T, Hq, d), dtype=dt, device="cuda")
    else:
        s.q = _normal((T, Hq, d), gen, dt, 1.0)
        s.out = torch.empty((T, Hq, d), dtype=dt, device="cuda")
        s.lse = torch.empty((T, Hq), dtype=torch.float32, device="cuda") if case["lse"] else None
        s.key_start = torch.tensor(_starts(case, s.prefix, s.chunk), **i32) if case["skip"] else None


def _starts(case, prefix, chunk):
    """First visible cache row of every sequence: for every third one of them
    past its first new tokens, which then see nothing."""
    if not case["skip"]:
        return [0] * len(prefix)
    return [(0, p // 3, p + c // 2)[i % 3] for i, (p, c) in enumerate(zip(prefix, chunk))]


def _prepare_sample(s, case, gen):
    """Logits with 1% of the vocabulary forbidden, and for each row its
    temperature, limits and random number.  A token count or a token that
    hangs on the last bit of a sum of 150,000 terms has no one answer in
    floating point, so each row's top_p, min_p and random number are moved
    to the middle of the interval in which they give the same result."""
    R, V = case["rows"], case["vocab"]
    x = torch.randn((R, V), generator=gen, device="cuda").mul_(case["spread"])
    x.masked_fill_(torch.rand((V,), generator=gen, device="cuda") < 0.01, float("-inf"))
    s.logits = x.to(_dtype(case))
    rows = torch.arange(R, device="cuda")
    s.temperature = torch.rand((R,), generator=gen, device="cuda") * 0.5 + 0.6
    s.temperature[rows % 16 == 15] = 0.0  # greedy rows
    s.top_k = torch.full((R,), case["k"], dtype=torch.int32, device="cuda") if case["k"] else None
    if case["k"]:
        s.top_k -= (rows % 3).to(torch.int32) * (case["k"] // 4)
    s.top_p = torch.full((R,), case["p"], device="cuda") if case["p"] < 1 else None
    s.min_p = torch.full((R,), case["min_p"], device="cuda") if case["min_p"] else None
    s.u = torch.rand((R,), generator=gen, device="cuda")
    for a in range(0, R, 128):
        _settle(s, slice(a, min(R, a + 128)))
    s.token = torch.empty(R, dtype=torch.int32, device="cuda")
    s.kept = torch.empty(R, dtype=torch.int32, device="cuda")
    s.log_prob = torch.empty(R, dtype=torch.float32, device="cuda")
    s.log_probs = torch.empty((R, V), dtype=torch.float32, device="cuda") if case["dist"] else None


def _settle(s, at):
    x = s.logits[at].double()
    T = s.temperature[at].double().clamp(min=1e-3)[:, None]
    w, idx = torch.sort(torch.exp((x - x.amax(1, keepdim=True)) / T), dim=1, descending=True, stable=True)
    if s.top_k is not None:
        w = w * (torch.arange(w.shape[1], device="cuda") < s.top_k[at][:, None])
    if s.top_p is not None:
        c = torch.cumsum(w, 1) / w.sum(1, keepdim=True)
        j = (c < s.top_p[at].double()[:, None]).sum(1, keepdim=True)
        edge = c.gather(1, j)
        s.top_p[at] = (edge - 0.5 * w.gather(1, j) / w.sum(1, keepdim=True))[:, 0].float()
        w = w * (torch.arange(w.shape[1], device="cuda") <= j)
    if s.min_p is not None:
        j = (w >= s.min_p[at].double()[:, None]).sum(1, keepdim=True)
        nxt = w.gather(1, j.clamp(max=w.shape[1] - 1))
        mid = torch.sqrt(w.gather(1, j - 1) * nxt)
        s.min_p[at] = torch.where(nxt > 0, mid, s.min_p[at].double()[:, None])[:, 0].float()
        w = w * (torch.arange(w.shape[1], device="cuda") < j)
    c = torch.cumsum(torch.zeros_like(w).scatter_(1, idx, w), 1)
    total = c[:, -1:]
    t = torch.searchsorted(c, s.u[at].double()[:, None] * total, right=True).clamp(max=c.shape[1] - 1)
    below = torch.where(t > 0, c.gather(1, (t - 1).clamp(min=0)), torch.zeros_like(total))
    s.u[at] = ((below + c.gather(1, t)) / (2 * total))[:, 0].float().clamp(max=1 - 2.0 ** -24)


# --------------------------------------------------------------- one pass
def run(s):
    return (_own if own else _plain)[s.case["op"]](s)


def _own_append(s):
    from paper_2606_02544_gb300 import simsd
    simsd.simsd_rope_append(s.plan, s.q, s.k, s.v, s.start, s.prefix_len, s.q_out, s.k_cache, s.v_cache, s.table,
                            err_word=s.err)
    return s.q_out, s.k_cache, s.v_cache


def _own_attend(s):
    from paper_2606_02544_gb300 import simsd
    c = s.case
    simsd.simsd_chunk_attention(s.q, s.start, s.prefix_len, s.k_cache, s.v_cache, s.table, s.out, lse=s.lse,
                                mask_block=c["block"], window=c["window"], key_start=s.key_start, workspace=s.ws,
                                err_word=s.err)
    return s.out, s.lse


def _own_sample(s):
    from paper_2606_02544_gb300 import simsd
    simsd.simsd_sample(s.logits, s.u, s.token, temperature=s.temperature, top_k=s.top_k, top_p=s.top_p,
                       min_p=s.min_p, kept=s.kept, log_prob=s.log_prob, log_probs=s.log_probs, err_word=s.err)
    return s.token, s.kept, s.log_prob, s.log_probs


def _frequencies(case):
    """Radians a position for each pair, in 64 bits: a position times a
    frequency rounded to 32 bits is off by whole degrees in a long context."""
    r = case["rot"]
    i = torch.arange(r // 2, dtype=torch.float64, device="cuda")
    s, theta = ROPE["factor"], ROPE["theta"]
    if case["scaling"] == "ntk":
        theta = theta * s ** (r / (r - 2))
    f = theta ** (-2.0 * i / r)
    if case["scaling"] == "linear":
        return f / s, 1.0
    if case["scaling"] == "yarn":
        turns = ROPE["context"] * f / (2 * math.pi)
        g = ((turns - ROPE["beta_slow"]) / (ROPE["beta_fast"] - ROPE["beta_slow"])).clamp(0, 1)
        return (1 - g) * f / s + g * f, 0.1 * math.log(s) + 1
    return f, 1.0


def _plain_rotate(x, pos, case):
    f, scale = _frequencies(case)
    angle = pos.double()[:, None, None] * f
    cos, sin = (torch.cos(angle) * scale).float(), (torch.sin(angle) * scale).float()
    r = case["rot"]
    y = x.float()
    if case["layout"] == "half":
        a, b = y[..., :r // 2], y[..., r // 2:r]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    else:
        a, b = y[..., 0:r:2], y[..., 1:r:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    return torch.cat([turned, y[..., r:]], -1).to(x.dtype)


def _plain_append(s):
    P = s.case["page"]
    pos = s.prefix_len[s.seq].long() + s.off
    page = s.table[s.seq, pos // P].long()
    s.k_cache[page, :, pos % P] = _plain_rotate(s.k, pos, s.case)
    s.v_cache[page, :, pos % P] = s.v
    return _plain_rotate(s.q, pos, s.case), s.k_cache, s.v_cache


def _plain_attend(s):
    c = s.case
    n, Hq, Hkv, d, P = c["seqs"], c["Hq"], c["Hkv"], c["d"], c["page"]
    g, C = Hq // Hkv, max(s.chunk)
    N = max(p + m for p, m in zip(s.prefix, s.chunk))
    j = torch.arange(N, device="cuda")
    page = s.table[:, j // P].clamp(min=0).long()                   # [n][N]
    k = s.k_cache[page, :, j % P].float().permute(0, 2, 3, 1)       # [n][Hkv][d][N]
    v = s.v_cache[page, :, j % P].float().permute(0, 2, 1, 3)       # [n][Hkv][N][d]
    q = torch.zeros((n, C, Hq, d), device="cuda")
    q[s.seq, s.off] = s.q.float()
    q = q.view(n, C, Hkv, g, d).permute(0, 2, 3, 1, 4).reshape(n, Hkv, g * C, d)
    x = torch.matmul(q, k).mul_(1 / math.sqrt(d)).view(n, Hkv, g, C, N)
    total = s.start[1:] - s.start[:-1] + s.prefix_len
    pos = s.prefix_len[:, None] + torch.arange(C, device="cuda")    # [n][C]
    hi = total[:, None].expand_as(pos)
    if c["block"]:
        hi = torch.minimum(hi, (pos // c["block"] + 1) * c["block"])
    lo = torch.zeros_like(pos) if s.key_start is None else s.key_start[:, None].expand_as(pos)
    if c["window"]:
        lo = torch.maximum(lo, pos + 1 - c["window"])
    seen = (j >= lo[..., None]) & (j < hi[..., None])               # [n][C][N]
    x.masked_fill_(~seen[:, None, None], float("-inf"))
    m = x.amax(-1, keepdim=True).clamp(min=-3.0e38)
    x.sub_(m).exp_()
    z = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(n, Hkv, g * C, N), v).view(n, Hkv, g, C, d) / torch.where(z > 0, z, torch.ones_like(z))
    o = o.permute(0, 3, 1, 2, 4).reshape(n, C, Hq, d)[s.seq, s.off].to(s.q.dtype)
    if s.lse is None:
        return o, None
    lse = (m + torch.log(z))[..., 0].permute(0, 3, 1, 2).reshape(n, C, Hq)[s.seq, s.off]
    return o, torch.where(torch.isfinite(lse) & (lse > -1e38), lse, torch.full_like(lse, float("-inf")))


def _plain_sample(s):
    """Weights in 32 bits; their running sums in 64, since a sum of the whole
    vocabulary decides which token a random number falls on."""
    x = s.logits.float()
    R, V = x.shape
    greedy = s.temperature == 0
    T = torch.where(greedy, torch.ones_like(s.temperature), s.temperature)[:, None]
    top, idx = torch.sort(x, dim=1, descending=True, stable=True)
    z = (top - top[:, :1]) / T
    w = torch.exp(z)
    at = torch.arange(V, device="cuda")
    keep = (w > 0) & ~(greedy[:, None] & (at > 0))
    if s.top_k is not None:
        keep &= at < s.top_k[:, None]
    if s.top_p is not None:
        c = torch.cumsum(torch.where(keep, w, torch.zeros_like(w)), 1, dtype=torch.float64)
        before = c - torch.where(keep, w, torch.zeros_like(w)).double()
        keep &= before < s.top_p.double()[:, None] * c[:, -1:]
    if s.min_p is not None:
        keep &= w >= s.min_p[:, None]
    w = torch.where(keep, w, torch.zeros_like(w))
    c = torch.cumsum(torch.zeros_like(w).scatter_(1, idx, w), 1, dtype=torch.float64)
    total = c[:, -1:]
    token = (c <= s.u.double()[:, None] * total).sum(1, keepdim=True).clamp(max=V - 1)
    logz = torch.log(total).float()
    picked = (x.gather(1, token) - top[:, :1]) / T - logz
    dist = None
    if s.log_probs is not None:
        dist = torch.empty_like(x).scatter_(1, idx, torch.where(keep, z - logz, torch.full_like(z, float("-inf"))))
    return token[:, 0].to(torch.int32), keep.sum(1).to(torch.int32), picked[:, 0], dist


_own = {"append": _own_append, "attend": _own_attend, "sample": _own_sample}
_plain = {"append": _plain_append, "attend": _plain_attend, "sample": _plain_sample}


# -------------------------------------------------------------------- work
def _visible(case, p, C, start):
    """(visible pairs, distinct visible keys) of one sequence."""
    N, B, W = p + C, case["block"], case["window"]
    pairs, first, last = 0, None, 0
    for i in range(p, N):
        hi = min(N, (i // B + 1) * B) if B else N
        lo = max(start, i + 1 - W if W else 0)
        if hi > lo:
            pairs += hi - lo
            first = lo if first is None else min(first, lo)
            last = max(last, hi)
    return pairs, last - first if first is not None else 0


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "sample":
        n = case["rows"] * case["vocab"]
        # a difference, a product, an exponential and a sum for each logit
        return {"bytes": n * e + (4 * n if case["dist"] else 0) + 28 * case["rows"], "flops": 4 * n}
    chunk, prefix = _lengths(case["seqs"], case["lo"], case["hi"], 1), _lengths(case["seqs"], case["prefix_lo"],
                                                                               case["prefix_hi"], 2)
    T, Hq, Hkv, d = sum(chunk), case["Hq"], case["Hkv"], case["d"]
    pages = sum((p + c + case["page"] - 1) // case["page"] for p, c in zip(prefix, chunk))
    if case["op"] == "append":
        pages = sum((c + case["page"] - 1) // case["page"] for c in chunk)
        return {"bytes": 2 * T * (Hq + 2 * Hkv) * d * e + 4 * (pages + 2 * len(chunk) + 1),
                "flops": 3 * T * (Hq + Hkv) * case["rot"]}
    seen = [_visible(case, p, c, s) for p, c, s in zip(prefix, chunk, _starts(case, prefix, chunk))]
    return {"bytes": 2 * T * Hq * d * e + sum(k for _, k in seen) * 2 * Hkv * d * e + (4 * T * Hq if case["lse"] else 0)
            + 4 * (pages + 2 * len(chunk) + 1), "flops": 4 * d * Hq * sum(n for n, _ in seen)}


# ------------------------------------------------------ the same in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "sample": _exact_sample}[case["op"]](s, case)


def _exact_turn(x, pos, case):
    """Every pair as a complex number, times m e^(i pos f)."""
    r, stretch = case["rot"], ROPE["factor"]
    f = []
    for i in range(r // 2):
        base = ROPE["theta"] * (stretch ** (r / (r - 2)) if case["scaling"] == "ntk" else 1.0)
        w = math.exp(-2.0 * i / r * math.log(base))
        if case["scaling"] == "linear":
            w /= stretch
        if case["scaling"] == "yarn":
            rho = ROPE["context"] * w / (2 * math.pi)
            g = min(1.0, max(0.0, (rho - ROPE["beta_slow"]) / (ROPE["beta_fast"] - ROPE["beta_slow"])))
            w = w / stretch * (1 - g) + w * g
        f.append(w)
    m = 1 + 0.1 * math.log(stretch) if case["scaling"] == "yarn" else 1.0
    turn = torch.polar(torch.full((len(pos), r // 2), m, dtype=torch.float64, device="cuda"),
                       torch.outer(pos.double(), torch.tensor(f, dtype=torch.float64, device="cuda")))[:, None]
    y = x.double().clone()
    first, second = (slice(0, r // 2), slice(r // 2, r)) if case["layout"] == "half" else (slice(0, r, 2),
                                                                                          slice(1, r, 2))
    z = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * turn
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_append(s, case):
    kc, vc, q = s.k_cache.double(), s.v_cache.double(), []
    at, P, table = 0, case["page"], s.table.cpu().tolist()
    for b, (p, c) in enumerate(zip(s.prefix, s.chunk)):
        rows = torch.arange(p, p + c, device="cuda")
        q.append(_exact_turn(s.q[at:at + c], rows, case))
        page = torch.tensor([table[b][r // P] for r in range(p, p + c)], device="cuda")
        kc[page, :, rows % P] = _exact_turn(s.k[at:at + c], rows, case)
        vc[page, :, rows % P] = s.v[at:at + c].double()
        at += c
    return torch.cat(q), kc, vc


def _exact_attend(s, case):
    Hq, Hkv, d, P = case["Hq"], case["Hkv"], case["d"], case["page"]
    if work(case)["flops"] > 4e12:  # more than some seconds at this card's rate in 64 bits
        return None
    g, at = Hq // Hkv, 0
    out = torch.zeros(s.q.shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s.q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    for b, (p, c, first) in enumerate(zip(s.prefix, s.chunk, _starts(case, s.prefix, s.chunk))):
        N = p + c
        pages = s.table[b, :(N + P - 1) // P].long()
        step = max(1, (1 << 28) // N)
        for h in range(Hkv):
            k = s.k_cache[pages, h].reshape(-1, d)[:N].double()
            v = s.v_cache[pages, h].reshape(-1, d)[:N].double()
            for i0 in range(0, c, step):
                i1 = min(c, i0 + step)
                i = torch.arange(p + i0, p + i1, device="cuda")[:, None]
                key = torch.arange(N, device="cuda")[None]
                hidden = key < first
                if case["block"]:
                    hidden = hidden | (key // case["block"] > i // case["block"])
                if case["window"]:
                    hidden = hidden | (i - key >= case["window"])
                for u in range(h * g, h * g + g):
                    x = s.q[at + i0:at + i1, u].double() @ k.T / math.sqrt(d)
                    x = torch.where(hidden, -math.inf, x)
                    l = torch.logsumexp(x, 1, keepdim=True)
                    out[at + i0:at + i1, u] = torch.where(l > -math.inf, torch.exp(x - l), 0.0) @ v
                    lse[at + i0:at + i1, u] = l[:, 0]
        at += c
    return out, lse if case["lse"] else None


def _exact_sample(s, case):
    tokens, counts, picked, dists = [], [], [], []
    for r in range(case["rows"]):
        x = s.logits[r].double()
        T = float(s.temperature[r])
        order = torch.argsort(x, descending=True, stable=True)
        order = order[x[order] > -math.inf]
        if T == 0:
            order, T = order[:1], 1.0
        if s.top_k is not None:
            order = order[:int(s.top_k[r])]
        logw = (x[order] - x[order[0]]) / T
        if s.top_p is not None:
            share = torch.cumsum(torch.softmax(logw, 0), 0)
            order = order[:int((share < float(s.top_p[r])).sum()) + 1]
            logw = logw[:len(order)]
        if s.min_p is not None and float(s.min_p[r]) > 0:
            order = order[logw >= math.log(float(s.min_p[r]))]
            logw = logw[:len(order)]
        logp = logw - torch.logsumexp(logw, 0)
        by_index, perm = torch.sort(order)
        cum = torch.cumsum(torch.exp(logp[perm]), 0)
        j = min(int((cum <= float(s.u[r])).sum()), len(order) - 1)
        tokens.append(by_index[j])
        counts.append(len(order))
        picked.append(logp[perm[j]])
        if s.log_probs is not None:
            dists.append(torch.full_like(x, -math.inf).index_put_((order,), logp))
    return (torch.stack(tokens).to(torch.int32), torch.tensor(counts, dtype=torch.int32, device="cuda"),
            torch.stack(picked), torch.stack(dists) if dists else None)

"""Cases of the operators that keep long caches small: what is timed and
compared for the 4-bit paged cache, windows with visible first rows, and the
pages of forked and compacted sequences.

A chunk's keys and values go to the cache in 4 bits (``simsd_rope_append_q4``)
and are read as such (``simsd_chunk_attention_q4``) or expanded
(``simsd_q4_expand``); a token sees a window and the first rows of its
sequence (``simsd_chunk_attention_sinks``), so that the pages between can be
released; sequences share pages (``simsd_pages_fork``), grow, let go of them,
and the pool is made dense again (``simsd_pages_compact``).  ``run`` makes
these calls, or with ``own`` false computes the same things from elementary
torch operations.
"""
import math
import random

import torch

own = False

GROUP = 16  # components that share a scale
EDGES = (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)  # between the magnitudes of 4 bits
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
TINY = 2.0 ** -9  # the smallest scale


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
        dict(name="append4 single f32", op="append", dtype="f32", seqs=8, lo=1, hi=1, prefix_lo=512, prefix_hi=1024,
             Hq=16, Hkv=8, d=64, page=16, layout="interleaved", rot=32, scaling="linear"),
        # a batch of long prompt chunks in a stretched context, cut out of one projection's output
        dict(name="append4 chunks bf16", op="append", dtype="bf16", seqs=8, lo=1501, hi=2600, prefix_lo=0,
             prefix_hi=8192, Hq=32, Hkv=8, d=128, page=64, layout="half", rot=128, scaling="yarn"),
        # token by token decoding of a small batch: latency
        dict(name="attend4 single few", op="attend", dtype="bf16", seqs=8, lo=1, hi=1, prefix_lo=512, prefix_hi=1024,
             Hq=16, Hkv=8, d=128, page=64, block=1, window=0, sinks=0, skip=0, lse=False),
        # token by token decoding of a full batch: reading the cache is all there is
        dict(name="attend4 single many", op="attend", dtype="bf16", seqs=64, lo=1, hi=1, prefix_lo=2048,
             prefix_hi=8192, Hq=32, Hkv=8, d=128, page=64, block=1, window=0, sinks=0, skip=0, lse=False),
        # block decoding: 16 tokens that see each other and 4096 cached ones
        dict(name="attend4 blocks of 16", op="attend", dtype="bf16", seqs=32, lo=16, hi=16, prefix_lo=4096,
             prefix_hi=4096, Hq=32, Hkv=8, d=128, page=64, block=16, window=0, sinks=0, skip=0, lse=False),
        # prompt chunks of odd lengths over long caches, small pages and heads, a window with visible first rows, and
        # sequences whose first rows (for some all that a token could see) are hidden
        dict(name="attend4 ragged chunks", op="attend", dtype="bf16", seqs=7, lo=97, hi=1501, prefix_lo=0,
             prefix_hi=12289, Hq=28, Hkv=4, d=64, page=16, block=1, window=3001, sinks=20, skip=1, lse=True),
        # decoding of a full batch over long contexts of which a window and four first rows are kept
        dict(name="sinks single many", op="sinks", dtype="bf16", seqs=64, lo=1, hi=1, prefix_lo=4096,
             prefix_hi=32768, Hq=32, Hkv=8, d=128, page=64, block=1, window=1024, sinks=4, skip=0, lse=False),
        # a whole prompt, block-causal, through a window: the first rows stay visible to all of it
        dict(name="sinks prompt 8192", op="sinks", dtype="bf16", seqs=1, lo=8192, hi=8192, prefix_lo=0, prefix_hi=0,
             Hq=32, Hkv=8, d=128, page=64, block=16, window=1024, sinks=64, skip=0, lse=True),
        # four sequences forked once each in a small fp32 cache: latency
        dict(name="fork few", op="fork", kind="f32", seqs=4, children=1, len_lo=30, len_hi=200, add=1, layers=2,
             Hkv=8, d=64, page=16),
        # 32 continuations of each of four prompts, in the caches of eight layers
        dict(name="fork 32 ways", op="fork", kind="bf16", seqs=4, children=31, len_lo=2000, len_hi=8100, add=70,
             layers=8, Hkv=8, d=128, page=64),
        # a small pool in 4 bits after a few sequences ended
        dict(name="compact few", op="compact", kind="q4", pages=60, live=0.5, seqs=4, layers=2, Hkv=4, d=128, page=16),
        # a pool of eight layers of which 40% is still in use
        dict(name="compact 500 pages", op="compact", kind="bf16", pages=500, live=0.4, seqs=16, layers=8, Hkv=8,
             d=128, page=64),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49))))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "sinks", "fork", "compact"])
    if op in ("fork", "compact"):
        kind = rng.choice(["bf16", "f32", "q4"])
        shape = dict(op=op, kind=kind, Hkv=rng.choice([2, 4, 8]), d=rng.choice([64, 128]),
                     page=rng.choice([8, 16, 64, 128]))
        row = shape["Hkv"] * shape["page"] * shape["d"] * {"bf16": 4, "f32": 8, "q4": 1.125}[kind]
        if op == "fork":
            seqs, children, add = _log(rng, 1, 12), _log(rng, 1, 24), rng.choice([1, _log(rng, 2, 300)])
            layers = max(1, min(_log(rng, 1, 16), int(2 ** 28 / (row * seqs * children))))
            hi = _log(rng, 20, 6000)
            return dict(shape, seqs=seqs, children=children, len_lo=max(1, hi // 3), len_hi=hi, add=add,
                        layers=max(1, min(layers, int(2 ** 30 / (row * seqs * (hi / shape["page"] + 2 * children))))))
        pages = _log(rng, 20, 2000)
        return dict(shape, pages=pages, live=rng.choice([0.2, 0.4, 0.6, 0.9]), seqs=_log(rng, 1, 40),
                    layers=max(1, min(_log(rng, 1, 16), int(2 ** 29 / (row * pages)))))
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    Hq, Hkv, d = rng.choice([(16, 8, 128), (32, 8, 128), (32, 8, 64), (28, 4, 64), (8, 8, 128), (40, 8, 128)])
    hi = rng.choice([1, _log(rng, 2, 64), _log(rng, 65, 2048)])
    lo = rng.choice([hi, max(1, hi // 3)])
    seqs = _log(rng, 1, max(1, min(64, (4096 if op != "append" else 16384) // hi)))
    prefix_hi = rng.choice([0, _log(rng, 16, 6000 if hi * seqs > 512 else 16384)])
    # fp32 runs without tensor cores: a sixteenth of the tokens
    if dtype == "f32" and op != "append":
        hi, lo, seqs = max(1, hi // 8), max(1, lo // 8), max(1, seqs // 2)
    # what the plain form spreads out of a drawn case stays below 8 GB
    while seqs > 1 and seqs * (prefix_hi + hi) * Hkv * d > (1 << 29):
        seqs //= 2
    case = dict(op=op, dtype=dtype, seqs=seqs, lo=lo, hi=hi, prefix_lo=prefix_hi // 4, prefix_hi=prefix_hi, Hq=Hq,
                Hkv=Hkv, d=d, page=rng.choice([8, 16, 64, 64, 128]))
    if op == "append":
        return dict(case, layout=rng.choice(["half", "interleaved"]), rot=rng.choice([d, d, d // 2, 24]),
                    scaling=rng.choice(["none", "linear", "ntk", "yarn"]))
    windowed = op == "sinks" or rng.random() < 0.3
    return dict(case, block=rng.choice([1, 1, 4, 16, 32, 0]), window=_log(rng, 16, 4096) if windowed else 0,
                sinks=rng.choice([1, 4, _log(rng, 2, 300)]) if windowed else 0, skip=int(rng.random() < 0.25),
                lse=rng.random() < 0.5)


# ------------------------------------------------------------------ inputs
ROPE = dict(theta=1.0e6, factor=4.0, context=8192, beta_fast=32.0, beta_slow=1.0)


class State:
    pass


def _dtype(case):
    return torch.float32 if case.get("dtype", case.get("kind")) == "f32" else torch.bfloat16


def _normal(shape, gen, dtype, std=1.0):
    return torch.randn(shape, generator=gen, device="cuda").mul_(std).to(dtype)


def prepare(case, seed):
    s = State()
    s.case = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if case["op"] == "fork":
        _prepare_fork(s, case, seed, gen)
    elif case["op"] == "compact":
        _prepare_compact(s, case, seed, gen)
    else:
        _prepare_chunks(s, case, seed, gen)
    if own:
        from paper_2606_02544_gb300 import simsd
        s.err = torch.zeros(1, dtype=torch.int32, device="cuda")
        if case["op"] in ("fork", "compact"):
            s.pages = simsd.PageSet(s.caches)
            n = simsd.simsd_pages_workspace_bytes(len(s.refs), len(s.src) if case["op"] == "fork" else 0)
            s.ws = torch.empty(n, dtype=torch.uint8, device="cuda")
            return s
        if case["op"] != "sinks":
            s.cache = simsd.Q4Cache(*s.q4)
        if case["op"] == "append":
            s.plan = simsd.simsd_rope_plan_init(case["layout"], case["rot"], ROPE["theta"], case["scaling"],
                                                factor=ROPE["factor"], context=ROPE["context"],
                                                beta_fast=ROPE["beta_fast"], beta_slow=ROPE["beta_slow"])
            return s
        code = simsd.SIMSD_F32 if case["dtype"] == "f32" else simsd.SIMSD_BF16
        sizes = (s.q.shape[0], case["seqs"], case["Hq"], case["Hkv"], case["d"], s.table.shape[1], case["page"])
        n = (simsd.simsd_chunk_workspace_bytes(code, *sizes) if case["op"] == "sinks" else
             simsd.simsd_chunk_q4_workspace_bytes(code, *sizes, s.q4[0].shape[0]))
        s.ws = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
    return s


def _kept_pages(case, p, c, first):
    """Pages of one sequence that hold a row which one of its tokens sees
    (appending: that it writes)."""
    P, N = case["page"], p + c
    if case["op"] == "append":
        return [i for i in range((N + P - 1) // P) if (i + 1) * P > p]
    if not case["window"]:
        return list(range((N + P - 1) // P))
    lo = max(first, p + 1 - case["window"])
    return [i for i in range((N + P - 1) // P)
            if (i + 1) * P > lo or (i * P < first + case["sinks"] and (i + 1) * P > first)]


def _prepare_chunks(s, case, seed, gen):
    """Chunks of new tokens, and a page pool in random order with spare pages;
    of each sequence the pages that its tokens need, no others."""
    dt, n, P = _dtype(case), case["seqs"], case["page"]
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    s.chunk = _lengths(n, case["lo"], case["hi"], 1)
    s.prefix = _lengths(n, case["prefix_lo"], case["prefix_hi"], 2)
    start = [0]
    for c in s.chunk:
        start.append(start[-1] + c)
    T = start[-1]
    s.first = _starts(case, s.prefix, s.chunk)
    kept = [_kept_pages(case, p, c, f) for p, c, f in zip(s.prefix, s.chunk, s.first)]
    pool = sum(map(len, kept)) + 3
    perm = torch.randperm(pool, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    table = torch.full((n, max((p + c + P - 1) // P for p, c in zip(s.prefix, s.chunk))), -1, dtype=torch.int32)
    at = 0
    for b, k in enumerate(kept):
        table[b, k] = perm[at:at + len(k)]
        at += len(k)
    i32 = dict(dtype=torch.int32, device="cuda")
    s.start = torch.tensor(start, **i32)
    s.prefix_len = torch.tensor(s.prefix, **i32)
    s.table = table.cuda()
    # what the plain form indexes with: sequence and offset of every token
    s.seq = torch.repeat_interleave(torch.arange(n), torch.tensor(s.chunk)).cuda()
    s.off = (torch.arange(T) - torch.tensor(start)[s.seq.cpu()]).cuda()
    rows = (pool, Hkv, P, d)
    if case["op"] == "append":
        # q, k and v are parts of one projection's rows
        qkv = _normal((T, Hq + 2 * Hkv, d), gen, dt)
        s.q, s.k, s.v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        _settle(s, case, gen)
        s.q_out = torch.empty((T, Hq, d), dtype=dt, device="cuda")
        s.q4 = [torch.zeros((*rows[:3], w), dtype=torch.uint8, device="cuda") for w in (d // 2, d // GROUP) * 2]
        s.new_len = s.prefix_len + (s.start[1:] - s.start[:-1])
        s.k_cache, s.v_cache = (torch.zeros(rows, dtype=dt, device="cuda") for _ in range(2))
        return
    if case["op"] == "sinks":
        s.k_cache, s.v_cache = _normal(rows, gen, dt), _normal(rows, gen, dt)
    else:
        s.q4 = []
        for _ in range(2):
            parts = [_pack(*_quantise(_normal((min(256, pool - a), *rows[1:]), gen, torch.bfloat16).float()))
                     for a in range(0, pool, 256)]
            s.q4 += [torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts])]
    s.q = _normal((T, Hq, d), gen, dt)
    s.out = torch.empty((T, Hq, d), dtype=dt, device="cuda")
    s.lse = torch.empty((T, Hq), dtype=torch.float32, device="cuda") if case["lse"] else None
    s.key_start = torch.tensor(s.first, **i32) if case["skip"] else None


def _starts(case, prefix, chunk):
    """First row of every sequence that may be seen: for every third one of
    them past its first new tokens, which then see nothing."""
    if not case.get("skip"):
        return [0] * len(prefix)
    return [(0, p // 3, p + c // 2)[i % 3] for i, (p, c) in enumerate(zip(prefix, chunk))]


def _settle(s, case, gen):
    """A component whose quotient by its group's scale lies within fp32's
    rounding of a border between two codes (or a group's largest by that of a
    border between two scales) has no one code in floating point: rows of k
    and v that hold such a component are drawn again."""
    pos = (s.prefix_len[s.seq].double() + s.off)
    for x, turned in ((s.k, True), (s.v, False)):
        for _ in range(8):
            y = (_turn64(x, pos, case) if turned else x.double()).unflatten(-1, (-1, GROUP))
            top = y.abs().amax(-1, keepdim=True)
            sc = _scale(top)
            grid = torch.exp2(torch.floor(torch.log2((top / 6).clamp(min=2.0 ** -6))) - 3)
            near = (((top / 6 / grid) % 1 - 0.5).abs() < 1e-4).any(-1)
            ratio = (y.abs() / sc.double())[..., None]
            near |= ((ratio - torch.tensor(EDGES, dtype=torch.float64, device="cuda")).abs() < 2e-5).flatten(-2).any(-1)
            at = near.any(-1)
            if not turned:  # (the quotients of bf16 values are exact there)
                at &= x.dtype == torch.float32
            if not bool(at.any()):
                break
            x[at] = _normal((int(at.sum()), x.shape[-1]), gen, x.dtype)


def _sizes(case):
    """Layers' arrays of a page, as shapes after [layers][pages]."""
    Hkv, P, d = case["Hkv"], case["page"], case["d"]
    if case["kind"] == "q4":
        return [((Hkv, P, w), torch.uint8) for w in (d // 2, d // GROUP) * 2]
    return [((Hkv, P, d), _dtype(case))] * 2


def _fill(s, case, pool, gen):
    s.caches = []
    for shape, dt in _sizes(case):
        whole = (case["layers"], pool, *shape)
        s.caches.append(torch.randint(0, 256, whole, dtype=dt, generator=gen, device="cuda") if dt == torch.uint8
                        else torch.randn(whole, generator=gen, device="cuda").to(dt))


def _fork_layout(case):
    """Lengths of the prompts, pages of each, table width and pool size."""
    P = case["page"]
    lens = _lengths(case["seqs"], case["len_lo"], case["len_hi"], 3)
    held = [(n + P - 1) // P for n in lens]
    most = (max(lens) + case["add"] + P - 1) // P + 1
    return lens, held, most, sum(held) + case["seqs"] * case["children"] * (2 + case["add"] // P) + 5


def _prepare_fork(s, case, seed, gen):
    """Prompts in a pool of random order, each followed by the places of its
    children, which hold nothing yet."""
    lens, held, most, pool = _fork_layout(case)
    each = case["children"] + 1
    perm = torch.randperm(pool, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    table = torch.full((case["seqs"] * each, most), -1, dtype=torch.int32)
    full, at = [0] * (case["seqs"] * each), 0
    for i, h in enumerate(held):
        table[i * each, :h] = perm[at:at + h]
        full[i * each] = lens[i]
        at += h
    refs = torch.zeros(pool, dtype=torch.int32)
    refs[perm[:at].long()] = 1
    src = [i * each for i in range(case["seqs"]) for _ in range(case["children"])]
    dst = [i * each + 1 + j for i in range(case["seqs"]) for j in range(case["children"])]
    i32 = dict(dtype=torch.int32, device="cuda")
    s.table, s.refs, s.lens = table.cuda(), refs.cuda(), torch.tensor(full, **i32)
    s.src, s.dst = torch.tensor(src, **i32), torch.tensor(dst, **i32)
    s.zero, s.end = torch.zeros(len(dst), **i32), torch.full((len(dst),), 2 ** 31 - 1, **i32)
    s.add = torch.zeros(len(full), **i32)
    s.add[s.dst.long()] = case["add"]
    _fill(s, case, pool, gen)


def _compact_layout(case):
    """Which pages are in use, in the order in which the sequences hold them,
    and for each page how many further sequences share it."""
    r = random.Random(7919 * case["pages"] + case["seqs"])
    live = max(1, round(case["pages"] * case["live"]))
    order = r.sample(range(case["pages"]), live)
    return order, [r.choice([0, 0, 0, 1]) for _ in order]


def _prepare_compact(s, case, seed, gen):
    order, shared = _compact_layout(case)
    n = case["seqs"]
    rows = [order[b::n] for b in range(n)]
    for i, (page, more) in enumerate(zip(order, shared)):
        if more:
            rows[(i + 1) % n].append(page)
    table = torch.full((n, max(map(len, rows)) + 2), -1, dtype=torch.int32)
    for b, row in enumerate(rows):
        table[b, :len(row)] = torch.tensor(row, dtype=torch.int32)
    shift = torch.randperm(n, generator=torch.Generator().manual_seed(seed))
    s.table0 = table[shift].contiguous().cuda()
    used = s.table0[s.table0 >= 0].long()
    s.refs0 = torch.bincount(used, minlength=case["pages"]).to(torch.int32)
    s.table, s.refs = s.table0.clone(), s.refs0.clone()
    s.live = torch.zeros(1, dtype=torch.int32, device="cuda")
    _fill(s, case, case["pages"], gen)


# --------------------------------------------------------------- one pass
def run(s):
    return (_own if own else _plain)[s.case["op"]](s)


def _own_append(s):
    from paper_2606_02544_gb300 import simsd
    simsd.simsd_rope_append_q4(s.plan, s.q, s.k, s.v, s.start, s.prefix_len, s.q_out, s.cache, s.table,
                               err_word=s.err)
    simsd.simsd_q4_expand(s.cache, s.table, s.prefix_len, s.new_len, s.k_cache, s.v_cache, err_word=s.err)
    return s.q_out, s.k_cache, s.v_cache


def _own_attend(s):
    from paper_2606_02544_gb300 import simsd
    c = s.case
    simsd.simsd_chunk_attention_q4(s.q, s.start, s.prefix_len, s.cache, s.table, s.out, lse=s.lse,
                                   mask_block=c["block"], window=c["window"], sinks=c["sinks"],
                                   key_start=s.key_start, workspace=s.ws, err_word=s.err)
    return s.out, s.lse


def _own_sinks(s):
    from paper_2606_02544_gb300 import simsd
    c = s.case
    simsd.simsd_chunk_attention_sinks(s.q, s.start, s.prefix_len, s.k_cache, s.v_cache, s.table, s.out,
                                      window=c["window"], sinks=c["sinks"], lse=s.lse, mask_block=c["block"],
                                      key_start=s.key_start, workspace=s.ws, err_word=s.err)
    return s.out, s.lse


def _own_fork(s):
    """The children of the last pass let go of their pages, then the prompts
    are forked again and the children get room for their next rows."""
    from paper_2606_02544_gb300 import simsd
    P = s.case["page"]
    simsd.simsd_pages_release(s.table, s.refs, s.zero, s.end, P, seq=s.dst, err_word=s.err)
    simsd.simsd_pages_fork(s.pages, s.src, s.dst, s.lens, s.table, s.refs, P, workspace=s.ws, err_word=s.err)
    simsd.simsd_pages_extend(s.lens, s.add, s.table, s.refs, P, err_word=s.err)
    return s.table, s.refs, s.lens, s.caches


def _own_compact(s):
    from paper_2606_02544_gb300 import simsd
    s.table.copy_(s.table0)
    s.refs.copy_(s.refs0)
    simsd.simsd_pages_compact(s.pages, s.table, s.refs, s.live, workspace=s.ws, err_word=s.err)
    return s.table, s.refs, s.live, s.caches


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


def _rotate(x, pos, case):
    """In 32 bits, not rounded to the type."""
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
    return torch.cat([turned, y[..., r:]], -1)


def _scale(top):
    """A sixth of a group's largest magnitude in 8 bits (4 for the exponent, 3
    for the fraction), at least the smallest such number where it is not 0."""
    sc = (top / 6).clamp(max=448.0).to(torch.float32).to(torch.float8_e4m3fn).float()
    return torch.where(sc == 0, torch.full_like(sc, TINY), sc)


def _quantise(x):
    """Codes (sign, then three bits of magnitude) and scales of x's groups."""
    y = x.unflatten(-1, (-1, GROUP))
    sc = _scale(y.abs().amax(-1, keepdim=True))
    a = y.abs() / sc
    code = torch.zeros_like(a, dtype=torch.uint8)
    for i, e in enumerate(EDGES):  # a tie goes to the even code
        code += (a >= e) if i % 2 else (a > e)
    return (code + 8 * (y < 0)).flatten(-2).to(torch.uint8), sc[..., 0]


def _pack(code, sc):
    return code[..., 0::2] | (code[..., 1::2] << 4), sc.to(torch.float8_e4m3fn).view(torch.uint8)


def _values(codes, scales):
    """What codes and scales in memory stand for, in 32 bits."""
    level = torch.tensor([*LEVELS, *(-x for x in LEVELS)], device=codes.device)
    both = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).int()
    return level[both].unflatten(-1, (-1, GROUP)).mul_(scales.view(torch.float8_e4m3fn).float()[..., None]).flatten(-2)


def _plain_append(s):
    P = s.case["page"]
    pos = s.prefix_len[s.seq].long() + s.off
    page = s.table[s.seq, pos // P].long()
    for i, x, image in ((0, _rotate(s.k, pos, s.case), s.k_cache), (2, s.v.float(), s.v_cache)):
        codes, scales = _pack(*_quantise(x))
        s.q4[i][page, :, pos % P], s.q4[i + 1][page, :, pos % P] = codes, scales
        image[page, :, pos % P] = _values(codes, scales).to(image.dtype)
    return _rotate(s.q, pos, s.case).to(s.q.dtype), s.k_cache, s.v_cache


def _columns(s):
    """The rows that a sequence's tokens see, side by side: the first ones
    that stay visible, then all from the window of the first token on.
    [n][N] row numbers, and which of these places count."""
    c = s.case
    first = torch.zeros_like(s.prefix_len) if s.key_start is None else s.key_start
    total = s.start[1:] - s.start[:-1] + s.prefix_len
    lo = torch.maximum(first, s.prefix_len + 1 - c["window"]) if c["window"] else first
    N = max(p + m - (max(f, p + 1 - c["window"]) if c["window"] else 0)
            for p, m, f in zip(s.prefix, s.chunk, s.first))
    j = torch.arange(max(1, N), device="cuda") + (lo if c["window"] else torch.zeros_like(lo))[:, None]
    real = j < total[:, None]
    if c["sinks"]:
        k = torch.arange(c["sinks"], device="cuda") + first[:, None]
        j, real = torch.cat([k, j], 1), torch.cat([k < torch.minimum(lo, total)[:, None], real], 1)
    return j, real, first, total


def _plain_attend(s):
    c = s.case
    n, Hq, Hkv, d, P = c["seqs"], c["Hq"], c["Hkv"], c["d"], c["page"]
    g, C = Hq // Hkv, max(s.chunk)
    j, real, first, total = _columns(s)
    N = j.shape[1]
    at = torch.where(real, j, torch.zeros_like(j))
    page = s.table.gather(1, (at // P).long()).clamp(min=0).long()  # [n][N]
    if c["op"] == "sinks":
        k, v = (x[page, :, at % P].float() for x in (s.k_cache, s.v_cache))
    else:
        k, v = (_values(s.q4[i][page, :, at % P], s.q4[i + 1][page, :, at % P]) for i in (0, 2))
    k, v = k.permute(0, 2, 3, 1), v.permute(0, 2, 1, 3)             # [n][Hkv][d][N], [n][Hkv][N][d]
    q = torch.zeros((n, C, Hq, d), device="cuda")
    q[s.seq, s.off] = s.q.float()
    q = q.view(n, C, Hkv, g, d).permute(0, 2, 3, 1, 4).reshape(n, Hkv, g * C, d)
    x = torch.matmul(q, k).mul_(1 / math.sqrt(d)).view(n, Hkv, g, C, N)
    pos = s.prefix_len[:, None] + torch.arange(C, device="cuda")    # [n][C]
    hi = total[:, None].expand_as(pos)
    if c["block"]:
        hi = torch.minimum(hi, (pos // c["block"] + 1) * c["block"])
    lo = first[:, None].expand_as(pos)
    if c["window"]:
        lo = torch.maximum(lo, pos + 1 - c["window"])
    j = j[:, None]
    seen = (j >= lo[..., None]) | ((j >= first[:, None, None]) & (j < first[:, None, None] + c["sinks"]))
    seen &= (j < hi[..., None]) & real[:, None]                     # [n][C][N]
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


def _plain_fork(s):
    P = s.case["page"]
    src, dst = s.src.long(), s.dst.long()
    held = s.table[dst]
    s.refs.index_add_(0, held.clamp(min=0).flatten().long(), -(held >= 0).flatten().int())
    s.table[dst] = -1
    # whole pages are shared, a page that is filled in part is copied
    n = s.lens[src]
    j = torch.arange(s.table.shape[1], device="cuda")
    row = s.table[src]
    whole = (j < (n // P)[:, None]) & (row >= 0)
    s.refs.index_add_(0, row.clamp(min=0).flatten().long(), whole.flatten().int())
    part = (n % P > 0).nonzero()[:, 0]
    old = row[part, (n[part] // P).long()].long()
    new = (s.refs == 0).nonzero()[:len(part), 0]
    s.refs[new] = 1
    row = torch.where(whole, row, torch.full_like(row, -1))
    row[part, (n[part] // P).long()] = new.int()
    s.table[dst] = row
    s.lens[dst] = n
    for x in s.caches:
        x[:, new] = x[:, old]
    # room for the next rows, sequence by sequence
    need = (j * P < (s.lens + s.add)[:, None]) & ((j + 1) * P > s.lens[:, None]) & (s.table < 0) & (s.add > 0)[:, None]
    b, k = need.nonzero(as_tuple=True)
    new = (s.refs == 0).nonzero()[:len(b), 0]
    s.refs[new] = 1
    s.table[b, k] = new.int()
    return s.table, s.refs, s.lens, s.caches


def _plain_compact(s):
    s.table.copy_(s.table0)
    s.refs.copy_(s.refs0)
    used = s.refs > 0
    count = used.sum()
    at = torch.arange(len(s.refs), device="cuda")
    free, out = (~used & (at < count)).nonzero()[:, 0], (used & (at >= count)).nonzero()[:, 0]
    for x in s.caches:
        x[:, free] = x[:, out]
    to = at.int()
    to[out] = free.int()
    s.table.copy_(torch.where(s.table >= 0, to[s.table.clamp(min=0).long()], s.table))
    s.refs[free], s.refs[out] = s.refs[out], 0
    s.live[0] = count
    return s.table, s.refs, s.live, s.caches


_own = {"append": _own_append, "attend": _own_attend, "sinks": _own_sinks, "fork": _own_fork, "compact": _own_compact}
_plain = {"append": _plain_append, "attend": _plain_attend, "sinks": _plain_attend, "fork": _plain_fork,
          "compact": _plain_compact}


# -------------------------------------------------------------------- work
def _visible(case, p, C, start):
    """(visible pairs, distinct visible keys) of one sequence."""
    N, B, W, S = p + C, case["block"], case["window"], case["sinks"]
    pairs, first, last = 0, None, 0
    for i in range(p, N):
        hi = min(N, (i // B + 1) * B) if B else N
        lo = max(start, i + 1 - W if W else 0)
        if hi > lo:
            pairs += hi - lo + max(0, min(start + S, lo) - start)
            first = lo if first is None else min(first, lo)
            last = max(last, hi)
    return pairs, last - first + max(0, min(start + S, first) - start) if first is not None else 0


def work(case):
    if case["op"] in ("fork", "compact"):
        page = sum(math.prod(shape) * (1 if dt == torch.uint8 else 4 if dt == torch.float32 else 2)
                   for shape, dt in _sizes(case)) * case["layers"]
        if case["op"] == "compact":
            order, shared = _compact_layout(case)
            moved = sum(p >= len(order) for p in order)
            return {"bytes": 2 * moved * page + 8 * case["pages"] + 8 * (len(order) + sum(shared)), "flops": 0}
        lens, held, _, pool = _fork_layout(case)
        P, each = case["page"], case["children"]
        part = [n % P > 0 for n in lens]
        # a prompt's last page is read once and written for each child; of the tables, the children's
        more = sum(len([k for k in range((n + case["add"] + P - 1) // P) if k >= h]) for n, h in zip(lens, held))
        return {"bytes": sum(part) * (1 + each) * page + 4 * (2 * each * sum(held) + each * more + 2 * pool),
                "flops": 0}
    e = 4 if case["dtype"] == "f32" else 2
    chunk, prefix = _lengths(case["seqs"], case["lo"], case["hi"], 1), _lengths(case["seqs"], case["prefix_lo"],
                                                                               case["prefix_hi"], 2)
    T, Hq, Hkv, d = sum(chunk), case["Hq"], case["Hkv"], case["d"]
    four = d // 2 + d // GROUP  # bytes of a row in 4 bits
    if case["op"] == "append":
        pages = sum((c + case["page"] - 1) // case["page"] for c in chunk)
        # rows in, q out; codes written and read again, their values written
        return {"bytes": T * ((2 * Hq + 2 * Hkv) * d * e + 2 * Hkv * (2 * four + d * e)) + 4 * (pages + 3 * len(chunk)),
                "flops": 3 * T * (Hq + Hkv) * case["rot"] + 6 * T * Hkv * d}
    seen = [_visible(case, p, c, s) for p, c, s in zip(prefix, chunk, _starts(case, prefix, chunk))]
    row = four if case["op"] == "attend" else d * e
    pages = sum(k // case["page"] + 1 for _, k in seen)
    return {"bytes": 2 * T * Hq * d * e + sum(k for _, k in seen) * 2 * Hkv * row + (4 * T * Hq if case["lse"] else 0)
            + 4 * (pages + 2 * len(chunk) + 1), "flops": 4 * d * Hq * sum(n for n, _ in seen)}


# ------------------------------------------------------ the same in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "sinks": _exact_attend, "fork": _exact_fork,
            "compact": _exact_compact}[case["op"]](s, case)


def _turn64(x, pos, case):
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


def _nearest(y):
    """What the groups of y are rounded to: the nearest of the numbers that a
    scale in 8 bits and 4 bits a component can hold."""
    y = y.unflatten(-1, (-1, GROUP))
    sixth = y.abs().amax(-1, keepdim=True) / 6
    scales = [i * TINY for i in range(1, 8)] + [m * 2.0 ** (x - 10) for x in range(1, 16) for m in range(8, 16)][:-1]
    scales = torch.tensor(scales, dtype=torch.float64, device="cuda")
    k = torch.searchsorted(scales, sixth).clamp(1, len(scales) - 1)
    below, above = scales[k - 1], scales[k]
    # (a tie goes to the even one, and the number at k has the last bit of k + 1)
    sc = torch.where((sixth - below < above - sixth) | ((sixth - below == above - sixth) & (k % 2 == 0)), below, above)
    a = y.abs() / sc
    level = torch.tensor(LEVELS, dtype=torch.float64, device="cuda")
    k = torch.searchsorted(level, a.contiguous()).clamp(1, 7)
    down, up = a - level[k - 1], level[k] - a
    v = torch.where((down < up) | ((down == up) & (k % 2 == 1)), level[k - 1], level[k])
    return (torch.where(y < 0, -v, v) * sc).flatten(-2)


def _exact_append(s, case):
    kc, vc, q = s.k_cache.double(), s.v_cache.double(), []
    at, P, table = 0, case["page"], s.table.cpu().tolist()
    for b, (p, c) in enumerate(zip(s.prefix, s.chunk)):
        rows = torch.arange(p, p + c, device="cuda")
        q.append(_turn64(s.q[at:at + c], rows, case))
        page = torch.tensor([table[b][r // P] for r in range(p, p + c)], device="cuda")
        kc[page, :, rows % P] = _nearest(_turn64(s.k[at:at + c], rows, case))
        vc[page, :, rows % P] = _nearest(s.v[at:at + c].double())
        at += c
    return torch.cat(q), kc, vc


def _exact_rows(s, case, i, pages, h):
    """Keys (i = 0) or values (1) of one head in the given pages."""
    if case["op"] == "sinks":
        return (s.k_cache, s.v_cache)[i][pages, h].double().flatten(0, 1)
    codes, scales = s.q4[2 * i][pages, h].flatten(0, 1).long(), s.q4[2 * i + 1][pages, h].flatten(0, 1).long()
    out = torch.empty((codes.shape[0], case["d"]), dtype=torch.float64, device="cuda")
    for half in range(2):
        c = (codes >> (4 * half)) & 15
        m, e = c & 1, (c >> 1) & 3
        mag = torch.where(e > 0, (2 + m) * 2.0 ** (e.double() - 2), m * 0.5)
        out[:, half::2] = torch.where(c >= 8, -mag, mag)
    e, m = scales >> 3, scales & 7
    sc = torch.where(e > 0, (8 + m) * 2.0 ** (e.double() - 10), m * 2.0 ** -9)
    return out * sc.repeat_interleave(GROUP, 1)


def _exact_attend(s, case):
    Hq, Hkv, d, P = case["Hq"], case["Hkv"], case["d"], case["page"]
    if work(case)["flops"] > 4e12:  # more than some seconds at this card's rate in 64 bits
        return None
    g, at = Hq // Hkv, 0
    out = torch.zeros(s.q.shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s.q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    for b, (p, c, first) in enumerate(zip(s.prefix, s.chunk, s.first)):
        N = p + c
        # the pages that are there, and the rows in them
        have = (s.table[b, :(N + P - 1) // P] >= 0).nonzero()[:, 0]
        pages = s.table[b, have].long()
        key = (have[:, None] * P + torch.arange(P, device="cuda")).flatten()[None]
        step = max(1, (1 << 28) // key.shape[1])
        for h in range(Hkv):
            k, v = _exact_rows(s, case, 0, pages, h), _exact_rows(s, case, 1, pages, h)
            for i0 in range(0, c, step):
                i1 = min(c, i0 + step)
                i = torch.arange(p + i0, p + i1, device="cuda")[:, None]
                hidden = key >= N
                if case["block"]:
                    hidden = hidden | (key // case["block"] > i // case["block"])
                if case["window"]:
                    hidden = hidden | ((i - key >= case["window"]) & (key >= first + case["sinks"]))
                hidden = hidden | (key < first)
                for u in range(h * g, h * g + g):
                    x = s.q[at + i0:at + i1, u].double() @ k.T / math.sqrt(d)
                    x = torch.where(hidden, -math.inf, x)
                    l = torch.logsumexp(x, 1, keepdim=True)
                    out[at + i0:at + i1, u] = torch.where(l > -math.inf, torch.exp(x - l), 0.0) @ v
                    lse[at + i0:at + i1, u] = l[:, 0]
        at += c
    return out, lse if case["lse"] else None


def _exact_fork(s, case):
    P, table, refs, lens = case["page"], s.table.cpu().tolist(), s.refs.cpu().tolist(), s.lens.cpu().tolist()
    caches = [x.clone() for x in s.caches]

    def take():
        page = refs.index(0)
        refs[page] = 1
        return page

    for a, b in zip(s.src.tolist(), s.dst.tolist()):
        lens[b] = lens[a]
        for k in range(lens[a] // P):
            table[b][k] = table[a][k]
            refs[table[a][k]] += 1
        if lens[a] % P:
            k = lens[a] // P
            table[b][k] = take()
            for x in caches:
                x[:, table[b][k]] = x[:, table[a][k]]
    for b, more in enumerate(s.add.tolist()):
        for k in range(lens[b] // P, (lens[b] + more + P - 1) // P if more else 0):
            if table[b][k] < 0:
                table[b][k] = take()
    i32 = dict(dtype=torch.int32, device="cuda")
    return torch.tensor(table, **i32), torch.tensor(refs, **i32), torch.tensor(lens, **i32), caches


def _exact_compact(s, case):
    table, refs = s.table0.cpu().tolist(), s.refs0.cpu().tolist()
    caches = [x.clone() for x in s.caches]
    used = sum(r > 0 for r in refs)
    holes, to = [p for p in range(used) if refs[p] == 0], {}
    for p in range(used, len(refs)):
        if refs[p]:
            to[p] = holes.pop(0)
            refs[to[p]], refs[p] = refs[p], 0
            for x in caches:
                x[:, to[p]] = x[:, p]
    table = [[to.get(p, p) for p in row] for row in table]
    i32 = dict(dtype=torch.int32, device="cuda")
    return torch.tensor(table, **i32), torch.tensor(refs, **i32), torch.tensor([used], **i32), caches

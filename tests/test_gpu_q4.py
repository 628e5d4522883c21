"""The cache in 4 bits on the GPU: append and expansion, and attention by codes
and through the image, against plain 64-bit forms."""
import math

import numpy as np
import pytest
import torch

from paper_2606_02544_gb300 import simsd
from tests import _longcache as ref
from tests import _prompt
from tests.test_gpu_sinks import compare

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
THETA = 1.0e6


def layout(chunk, prefix, P, g, spare=2):
    start = np.concatenate([[0], np.cumsum(chunk)]).astype(np.int32)
    pages = [(n + c + P - 1) // P for n, c in zip(prefix, chunk)]
    pool = sum(pages) + spare
    perm = torch.randperm(pool, generator=g).int()
    table = torch.full((len(chunk), max(max(pages), 1)), -1, dtype=torch.int32)
    at = 0
    for b, c in enumerate(pages):
        table[b, :c] = perm[at:at + c]
        at += c
    return start, pool, table


def make(dtype, chunk, prefix, Hq, Hkv, d, P, seed, units=(1.0, 1.0)):
    g = torch.Generator().manual_seed(seed)
    start, pool, table = layout(chunk, prefix, P, g)
    T = sum(chunk)
    # rows of one projection; magnitudes from tiny to large
    x = torch.randn(T, Hq + 2 * Hkv, d, generator=g) * torch.exp2(torch.randint(-7, 6, (T, Hq + 2 * Hkv, 1), generator=g))
    x = x.to(dtype).cuda()
    codes = [torch.randint(0, 256, (pool, Hkv, P, w), dtype=torch.uint8, generator=g).cuda() for w in (d // 2, d // 16) * 2]
    i32 = dict(dtype=torch.int32, device="cuda")
    return dict(q=x[:, :Hq], k=x[:, Hq:Hq + Hkv], v=x[:, Hq + Hkv:], token_start=torch.tensor(start, **i32),
                prefix_len=torch.tensor(prefix, **i32), cache=simsd.Q4Cache(*codes, *units),
                q_out=torch.full((T, Hq, d), float("nan"), dtype=dtype, device="cuda"), block_table=table.cuda(),
                err_word=torch.zeros(1, **i32))


def check_append(a, plan_args, positions=None):
    before = [t.clone() for t in a["cache"].tensors]
    plan = simsd.simsd_rope_plan_init(*plan_args[:3], **plan_args[3])
    simsd.simsd_rope_append_q4(plan, **a, positions=positions)
    assert simsd.simsd_check_error(a["err_word"]) == 0
    lay, rot, theta, kw = plan_args
    freq = _prompt.frequencies(rot, theta, **kw)
    dtype = a["q"].dtype
    start, prefix = a["token_start"].tolist(), a["prefix_len"].tolist()
    pos = np.concatenate([np.arange(n, n + start[b + 1] - start[b]) for b, n in enumerate(prefix)] or [[]]).astype(int)
    at = positions.cpu().numpy() if positions is not None else pos
    P = a["cache"].P
    seq = np.repeat(np.arange(len(prefix)), np.diff(start))
    page = torch.as_tensor(a["block_table"].cpu().numpy()[seq, pos // P]).cuda()
    off = torch.as_tensor(pos % P).cuda()
    want, size = _prompt.rotate(a["q"].double().cpu().numpy(), at, lay, rot, freq)
    assert np.all(np.abs(a["q_out"].double().cpu().numpy() - want) <= _prompt.rope_tolerance(want, size, dtype == BF16))
    kcodes, kscales, vcodes, vscales = (t[page, :, off].cpu().numpy() for t in a["cache"].tensors)
    want, size = _prompt.rotate(a["k"].double().cpu().numpy(), at, lay, rot, freq)
    ref.check_codes(kcodes, kscales, want, 2.0 ** -20 * size, a["cache"].k_unit)
    v = a["v"].double().cpu().numpy()
    if dtype == BF16 and math.log2(a["cache"].v_unit) % 1 == 0:
        assert np.array_equal(ref.decode(vcodes, vscales), ref.encode(v / a["cache"].v_unit))
    else:
        ref.check_codes(vcodes, vscales, v, 2.0 ** -23 * np.abs(v), a["cache"].v_unit)
    # nothing else is written
    for t, b in zip(a["cache"].tensors, before):
        b[page, :, off] = t[page, :, off]
        assert torch.equal(t, b)


PLANS = [("half", 128, {}), ("interleaved", 128, dict(scaling="linear", factor=4.0)),
         ("half", 64, dict(scaling="ntk", factor=2.0)), ("half", 24, {}), ("interleaved", 6, {}), ("half", 2, {}),
         ("half", 52, dict(scaling="yarn", factor=4.0, context=4096)), ("half", 126, {}), ("half", 10, {})]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("lay,rot,kw", PLANS)
@pytest.mark.parametrize("d", [64, 128])
def test_append(dtype, lay, rot, kw, d):
    a = make(dtype, [1, 37, 0, 5], [70, 0, 9, 130], 8, 2, d, 16, rot)
    check_append(a, (lay, min(rot, d), THETA, kw))


@pytest.mark.parametrize("chunk,prefix,Hq,Hkv,P", [([1], [0], 1, 1, 8), ([1] * 9, [3, 64, 100, 7, 8, 9, 0, 1, 1000], 7, 7, 64),
                                                   ([513, 1, 260], [31, 5000, 0], 5, 3, 128), ([2000], [77], 32, 8, 192)])
def test_append_sizes(chunk, prefix, Hq, Hkv, P):
    for dtype, d in ((BF16, 128), (F32, 64)):
        check_append(make(dtype, chunk, prefix, Hq, Hkv, d, P, len(chunk)), ("half", d, THETA, {}))


@pytest.mark.parametrize("units", [(0.25, 8.0), (1.7, 0.003)])
def test_append_units(units):
    for dtype in (BF16, F32):
        check_append(make(dtype, [9, 40], [11, 0], 8, 2, 128, 16, 1, units), ("half", 128, THETA, {}))


def test_append_positions_and_in_place():
    a = make(BF16, [5, 9], [100, 3], 4, 2, 64, 16, 3)
    pos = torch.tensor([7, 2 ** 27, 0, 123456, 9, -5, 1, 2, 3, 10 ** 6, 5, 2 ** 30, 31, 32], dtype=torch.int32, device="cuda")
    check_append(a, ("half", 64, THETA, {}), positions=pos)
    b = make(BF16, [5, 9], [100, 3], 4, 2, 64, 16, 3)
    q = b["q"].contiguous()
    plan = simsd.simsd_rope_plan_init("half", 64, THETA)
    simsd.simsd_rope_append_q4(plan, **(b | dict(q=q, q_out=q)), positions=pos)
    assert torch.equal(q, a["q_out"])


def test_append_special_values():
    """Zeros, the smallest and largest groups, infinities and NaN."""
    a = make(F32, [7], [3], 1, 1, 64, 8, 2)
    a["v"].zero_()
    v = a["v"]
    v[1, 0, 0] = float("nan")
    v[2, 0, 5] = float("inf")
    v[3, 0, :16] = 1e-6
    v[4, 0, 16:32] = 1e30
    v[5, 0, 63] = -2688.0
    v[6, 0, :] = -0.0
    a["k"].copy_(v)
    a["prefix_len"].zero_()
    simsd.simsd_rope_append_q4(simsd.simsd_rope_plan_init("half", 2, THETA), **a,
                               positions=torch.zeros(7, dtype=torch.int32, device="cuda"))
    assert simsd.simsd_check_error(a["err_word"]) == 0
    t = a["cache"].tensors
    page = int(a["block_table"][0, 0])
    for c, s in ((t[0], t[1]), (t[2], t[3])):
        got = ref.decode(c[page, 0, :7].cpu().numpy(), s[page, 0, :7].cpu().numpy())
        assert np.all(got[0] == 0) and np.isnan(got[1, :16]).all() and np.all(got[1, 16:] == 0)
        assert got[2, 5] == 2688 and np.all(np.delete(got[2], 5) == 0)
        assert np.all(got[3] == 0) and np.all(got[4, 16:32] == 2688) and np.all(got[4, 32:] == 0)
        assert got[5, 63] == -2688 and np.all(got[5, :63] == 0) and np.all(got[6] == 0)


def test_append_errors():
    """Bad lengths, pages and offsets: as simsd_rope_append."""
    plan = simsd.simsd_rope_plan_init("half", 64, THETA)
    for what, bit in (("len", simsd.EW_PREFIX_LEN), ("page", simsd.EW_PAGE), ("start", simsd.EW_TOKENS)):
        a = make(BF16, [4, 5, 6], [20, 30, 10], 4, 2, 64, 16, 7)
        if what == "len":
            a["prefix_len"][1] = 1000
        if what == "page":
            a["block_table"][1, 2] = 99
        if what == "start":
            a["token_start"][2] = 2  # sequences 1: reversed
        before = [t.clone() for t in a["cache"].tensors]
        simsd.simsd_rope_append_q4(plan, **a)
        assert simsd.simsd_check_error(a["err_word"]) & bit
        qo = a["q_out"].float()
        if what == "len":
            assert bool((qo[4:9] == 0).all())
        if what != "start":
            assert bool(torch.isfinite(qo).all())
            page = int(a["block_table"][1, 1])
            for t, b in zip(a["cache"].tensors, before):
                if what == "len":
                    assert torch.equal(t[page], b[page])
        spare = np.setdiff1d(np.arange(a["cache"].num_pages), a["block_table"].cpu().numpy())
        for t, b in zip(a["cache"].tensors, before):
            assert torch.equal(t[torch.as_tensor(spare).cuda()], b[torch.as_tensor(spare).cuda()])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d,P,units", [(128, 64, (1.0, 1.0)), (64, 8, (0.5, 1.7)), (128, 192, (3.3, 4.0))])
def test_expand(dtype, d, P, units):
    """Every byte of scale and code, ranges that begin and end inside pages."""
    g = torch.Generator().manual_seed(d + P)
    _, pool, table = layout([0] * 5, [300, 33, 1, 0, 130], P, g)
    codes = [torch.randint(0, 256 if w == d // 2 else 127, (pool, 3, P, w), dtype=torch.uint8, generator=g).cuda()
             for w in (d // 2, d // 16) * 2]
    cache = simsd.Q4Cache(*codes, *units)
    i32 = dict(dtype=torch.int32, device="cuda")
    first, last = [7, 0, 0, 0, 65], [300, 33, 1, 0, 66]
    out = [torch.full((pool, 3, P, d), 5.0, dtype=dtype, device="cuda") for _ in range(2)]
    err = torch.zeros(1, **i32)
    simsd.simsd_q4_expand(cache, table.cuda(), torch.tensor(first, **i32), torch.tensor(last, **i32), *out, err_word=err)
    assert simsd.simsd_check_error(err) == 0
    for i in range(2):
        val = torch.from_numpy(ref.decode(codes[2 * i].cpu().numpy(), codes[2 * i + 1].cpu().numpy())).float()
        want = torch.full((pool, 3, P, d), 5.0).to(dtype)
        val = (val * torch.tensor(units[i], dtype=F32)).to(dtype)  # one product in fp32, rounded once
        for b in range(5):
            r = np.arange(first[b], last[b])
            pg = table[b].numpy()[r // P]
            want[pg, :, r % P] = val[pg, :, r % P]
        assert torch.equal(out[i].cpu(), want)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_expand_to_arrays_at_odd_multiples_of_16_bytes(dtype):
    g = torch.Generator().manual_seed(11)
    cache = simsd.Q4Cache(*(torch.randint(0, 120, (5, 2, 16, w), dtype=torch.uint8, generator=g).cuda() for w in (32, 4) * 2))
    i32 = dict(dtype=torch.int32, device="cuda")
    table, first, last = torch.arange(5, **i32)[None], torch.tensor([3], **i32), torch.tensor([77], **i32)
    n, shift = 5 * 2 * 16 * 64, 16 // dtype.itemsize
    outs = []
    for k, v in ((0, 0), (shift, 0), (shift, shift)):
        pair = [torch.full((n + 16,), 5.0, dtype=dtype, device="cuda")[at:at + n].view(5, 2, 16, 64) for at in (k, v)]
        simsd.simsd_q4_expand(cache, table, first, last, *pair)
        outs.append(torch.stack(pair))
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2]) and bool((outs[0] != 5).any())


def test_expand_errors():
    g = torch.Generator().manual_seed(1)
    _, pool, table = layout([0] * 3, [40, 40, 40], 8, g)
    cache = simsd.Q4Cache.zeros(pool, 2, 8, 64)
    i32 = dict(dtype=torch.int32, device="cuda")
    t = table.cuda()
    for first, last, bit in (([0, -1, 0], [40, 8, 40], simsd.EW_PREFIX_LEN), ([0, 0, 0], [40, 41, 40], simsd.EW_PREFIX_LEN)):
        out = [torch.full((pool, 2, 8, 64), 5.0, dtype=BF16, device="cuda") for _ in range(2)]
        err = torch.zeros(1, **i32)
        simsd.simsd_q4_expand(cache, t, torch.tensor(first, **i32), torch.tensor(last, **i32), *out, err_word=err)
        assert simsd.simsd_check_error(err) == bit
        for x in out:
            assert bool((x[t[1].long()] == 5).all()) and bool((x[t[0].long()] == 0).all())
    t[1, 2] = pool
    out = [torch.full((pool, 2, 8, 64), 5.0, dtype=BF16, device="cuda") for _ in range(2)]
    err = torch.zeros(1, **i32)
    simsd.simsd_q4_expand(cache, t, torch.zeros(3, **i32), torch.full((3,), 40, **i32), *out, err_word=err)
    assert simsd.simsd_check_error(err) == simsd.EW_PAGE
    assert bool((out[0][t[1, [0, 1, 3, 4]].long()] == 0).all()) and bool((out[0][table[1, 2]] == 5).all())


# ---------------------------------------------------------------- attention
def attention_case(dtype, chunk, prefix, Hq, Hkv, d, P, seed, window=0, sinks=0, block=1, key_start=None, std=1.0,
                   units=(1.0, 1.0), hide=True):
    """Codes of normal rows; rows that no token sees hold NaN scales, their
    pages, where no row of them is seen, are not in the table."""
    g = torch.Generator().manual_seed(seed)
    start, pool, table = layout(chunk, prefix, P, g)
    ks = key_start or [0] * len(chunk)
    codes = []
    for _ in range(2):
        y = torch.randn(pool, Hkv, P, d, generator=g) * std
        grp = y.unflatten(-1, (-1, 16))
        s = torch.from_numpy(np.abs(ref.SCALES[None, 1:] - (grp.abs().amax(-1) / 6).numpy().reshape(-1, 1)).argmin(1) + 1)
        s = s.view(pool, Hkv, P, d // 16).to(torch.uint8)
        q = (grp / torch.from_numpy(ref.SCALES)[s.long()][..., None].float()).flatten(-2)
        c = (q.abs()[..., None] - torch.from_numpy(ref.LEVELS).float()).abs().argmin(-1) + 8 * (q < 0)
        codes += [(c[..., 0::2] | c[..., 1::2] << 4).to(torch.uint8), s]
    keep = torch.zeros(pool, P, dtype=torch.bool)
    for b, (n, C) in enumerate(zip(prefix, chunk)):
        rows = [ref.visible(n, C, i, block, window, ks[b], sinks) for i in range(C)]
        r = torch.as_tensor(np.unique(np.concatenate(rows)) if rows else np.array([], dtype=int))
        keep[table[b, r // P].long(), r % P] = True
    if hide:
        for s in (codes[1], codes[3]):
            s.masked_fill_(~keep[:, None, :, None], 127)
        gone = ~keep.any(1)
        table[(table >= 0) & gone[table.clamp(min=0).long()]] = -1
    i32 = dict(dtype=torch.int32, device="cuda")
    q = torch.randn(sum(chunk), Hq, d, generator=g).mul_(std).to(dtype).cuda()
    return dict(q=q, token_start=torch.tensor(start, **i32), prefix_len=torch.tensor(prefix, **i32),
                cache=simsd.Q4Cache(*(c.cuda() for c in codes), *units), block_table=table.cuda(),
                key_start=torch.tensor(ks, **i32) if key_start else None)


def run(a, stream=None, **kw):
    T, Hq, d = a["q"].shape
    c = a["cache"]
    out = torch.full((T, Hq, d), float("nan"), dtype=a["q"].dtype, device="cuda")
    lse = torch.full((T, Hq), float("nan"), device="cuda")
    code = simsd.SIMSD_F32 if a["q"].dtype == F32 else simsd.SIMSD_BF16
    n = simsd.simsd_chunk_q4_workspace_bytes(code, T, len(a["prefix_len"]), Hq, c.Hkv, d, a["block_table"].shape[1],
                                             c.P, c.num_pages)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")  # NaN bits: it needs no initial value
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    simsd.simsd_chunk_attention_q4(**a, out=out, lse=lse, workspace=ws, err_word=err, stream=stream, **kw)
    return out, lse, simsd.simsd_check_error(err)


def check(a, window=0, sinks=0, mask_block=1, softmax_scale=0.0):
    out, lse, word = run(a, window=window, sinks=sinks, mask_block=mask_block, softmax_scale=softmax_scale)
    assert word == 0
    c, (T, Hq, d) = a["cache"], a["q"].shape
    bf16 = a["q"].dtype == BF16
    kc, ks, vc, vs = (t.cpu().numpy() for t in c.tensors)
    kd, vd = ref.decode(kc, ks, c.k_unit), ref.decode(vc, vs, c.v_unit)
    few = bf16 and T * Hq <= (768 if d == 128 else 512) * len(a["prefix_len"]) * c.Hkv  # by codes
    if not few:  # a unit that is no power of two rounds the image
        kd, vd = (torch.from_numpy(x).float().to(a["q"].dtype).double().numpy() for x in (kd, vd))

    def tolerance(o, av, qk, N, vm):
        return ref.q4_tolerance(o, av, qk, N, vm) if few else _prompt.attention_tolerance(o, av, qk, N, bf16)

    compare(a, out, lse, kd, vd, window, sinks, mask_block, softmax_scale, tolerance)


@pytest.mark.parametrize("Hq,Hkv", [(4, 2), (8, 1), (7, 1), (16, 1), (6, 2), (32, 1), (40, 1), (64, 1), (3, 3)])
@pytest.mark.parametrize("d,P", [(128, 64), (64, 16), (128, 8), (64, 192), (128, 128)])
def test_single_tokens(Hq, Hkv, d, P):
    """One token a sequence, lengths around pages and tiles."""
    prefix = [0, 1, 7, 63, 64, 127, 128, 129, 255, 300, 511, 700]
    check(attention_case(BF16, [1] * 12, prefix, Hq, Hkv, d, P, Hq + P))


@pytest.mark.parametrize("chunk,Hq,Hkv", [([2] * 5, 4, 1), ([4, 1, 3, 4, 0], 8, 2), ([16] * 5, 8, 2), ([9, 16, 1, 12, 20], 4, 1),
                                          ([33, 1, 1, 1, 0], 4, 2), ([5, 64, 1, 0, 2], 2, 2)])
@pytest.mark.parametrize("block", [1, 16, 0])
def test_short_chunks(chunk, Hq, Hkv, block):
    """2 to 64 query rows a unit, units of part of a chunk."""
    prefix = [130, 0, 500, 77, 256]
    check(attention_case(BF16, chunk, prefix, Hq, Hkv, 128, 16, sum(chunk), block=block), mask_block=block)
    check(attention_case(BF16, chunk, prefix, Hq, Hkv, 64, 64, sum(chunk), block=block), mask_block=block)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("window,sinks,block", [(1, 0, 1), (5, 3, 1), (130, 4, 1), (128, 128, 16), (300, 129, 0),
                                                (64, 700, 1), (97, 1, 7), (50, 0, 4)])
def test_windows(dtype, window, sinks, block):
    chunk, prefix = [1, 1, 6, 9, 1, 0, 3], [700, 3, 511, 0, 0, 40, 385]
    check(attention_case(dtype, chunk, prefix, 8, 2, 128, 16, window + sinks, window, sinks, block), window, sinks, block)
    check(attention_case(dtype, chunk, prefix, 3, 1, 64, 8, window + sinks, window, sinks, block), window, sinks, block)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_key_start(dtype):
    chunk, prefix, ks = [5, 14, 3, 9, 1], [300, 500, 100, 64, 0], [200, 129, 110, 80, 0]
    check(attention_case(dtype, chunk, prefix, 4, 2, 128, 16, 5, key_start=ks))
    check(attention_case(dtype, chunk, prefix, 4, 2, 64, 8, 6, 20, 100, 4, key_start=ks), 20, 100, 4)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("window,sinks", [(0, 0), (70, 9)])
def test_long_chunks(dtype, window, sinks):
    """Through the image; shared pages and pages of other sequences' rows."""
    chunk, prefix = [150, 40, 201], [100, 0, 33]
    a = attention_case(dtype, chunk, prefix, 8, 2, 128, 16, 3, window, sinks, 4, units=(0.5, 2.0))
    check(a, window, sinks, 4)
    a = attention_case(dtype, chunk, prefix, 6, 1, 64, 64, 4, window, sinks, units=(1.3, 0.7))
    check(a, window, sinks)
    a = attention_case(dtype, [400], [70], 8, 2, 128, 16, 7, window, sinks, 4, units=(0.7, 2.0))
    check(a, window, sinks, 4)


@pytest.mark.parametrize("d,Hq,Hkv", [(128, 8, 2), (64, 8, 2), (128, 7, 1), (64, 9, 3)])
def test_either_side_of_the_rule_of_ways(d, Hq, Hkv):
    """The most rows that are attended to by codes, and one token more."""
    most = (768 if d == 128 else 512) * Hkv // Hq
    for n in (most, most + 1):
        check(attention_case(BF16, [n], [100], Hq, Hkv, d, 16, n + Hq))


@pytest.mark.parametrize("n,Hq,Hkv,d,window,sinks", [(1, 32, 8, 128, 0, 0), (16, 32, 8, 128, 0, 0), (32, 32, 8, 128, 0, 0),
                                                     (16, 32, 8, 128, 1500, 40), (29, 32, 8, 128, 1500, 40),
                                                     (9, 28, 4, 64, 0, 0), (17, 28, 4, 64, 900, 200)])
def test_long_runs(n, Hq, Hkv, d, window, sinks):
    """Tens of tiles and several units a CTA, with queries of their own for
    sequences that share their pages."""
    seqs = 40
    a = attention_case(BF16, [n], [2600], Hq, Hkv, d, 64, n + d, window, sinks)
    i32 = dict(dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(n)
    a["q"] = torch.randn(seqs * n, Hq + 2, d, generator=g, device="cuda").to(BF16)[:, 1:-1]
    a["token_start"] = torch.arange(seqs + 1, **i32) * n
    a["prefix_len"] = torch.full((seqs,), 2600, **i32)
    a["block_table"] = a["block_table"].repeat(seqs, 1)
    check(a, window, sinks)
    first, again = run(a, window=window, sinks=sinks), run(a, window=window, sinks=sinks)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("units,scale", [((0.25, 8.0), 0.0), ((1.7, 0.3), 0.02), ((1.0, 1.0), 0.5)])
def test_units_and_scale(units, scale):
    check(attention_case(BF16, [1, 3], [300, 140], 8, 2, 128, 64, 9, units=units), softmax_scale=scale)


def test_large_and_small_queries():
    """q from 2^-60 to 2^60 of ordinary, zero rows, components far below their
    row's largest; references that move."""
    a = attention_case(BF16, [1] * 6, [500, 300, 200, 100, 130, 64], 8, 2, 128, 64, 12, std=3.0)
    check(a)
    a["q"][1] *= 2.0 ** -60
    a["q"][2] = 0
    a["q"][3, :, ::2] *= 2.0 ** -20
    check(a)
    b = attention_case(BF16, [1, 1], [500, 300], 8, 2, 128, 64, 12)
    want, _, _ = run(b)
    b["q"] = b["q"] * 2.0 ** 60
    got, _, word = run(b, softmax_scale=2.0 ** -60 / math.sqrt(128))
    assert word == 0 and torch.equal(got, want)


def test_same_bits_every_time_and_on_another_stream():
    a = attention_case(BF16, [1, 4, 2, 1], [900, 30, 1500, 64], 8, 2, 128, 64, 2)
    want = run(a)
    s = torch.cuda.Stream()
    for _ in range(3):
        torch.cuda.synchronize()
        got = run(a, stream=s)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype,chunk", [(BF16, [1, 1, 1]), (F32, [1, 1, 1]), (BF16, [200, 30, 1])])
def test_bad_pages_and_lengths(dtype, chunk):
    for what, bit in (("page", simsd.EW_PAGE), ("len", simsd.EW_PREFIX_LEN), ("start", simsd.EW_TOKENS)):
        a = attention_case(dtype, chunk, [400, 390, 70], 8, 2, 64, 16, 4)
        want, _, _ = run(a)
        if what == "page":
            a["block_table"][1, 3] = -1
        if what == "len":
            a["prefix_len"][1] = 10 ** 6
        if what == "start":
            a["token_start"][3] = sum(chunk) + 1
        out, lse, word = run(a)
        assert word == bit
        s, e = sum(chunk[:1]), sum(chunk[:2])
        if what == "start":
            assert bool(torch.isnan(out[e:]).all())  # untouched
            assert torch.equal(out[:e], want[:e])
        else:
            assert bool((out[s:e] == 0).all()) and bool(torch.isneginf(lse[s:e]).all())
            assert torch.equal(out[:s], want[:s]) and torch.equal(out[e:], want[e:])


def test_empty_calls():
    c = simsd.Q4Cache.zeros(4, 2, 16, 64)
    i32 = dict(dtype=torch.int32, device="cuda")
    q = torch.empty(0, 8, 64, dtype=BF16, device="cuda")
    plan = simsd.simsd_rope_plan_init("half", 64, THETA)
    table = torch.zeros(2, 2, **i32)
    simsd.simsd_chunk_attention_q4(q, torch.zeros(3, **i32), torch.zeros(2, **i32), c, table, torch.empty_like(q))
    kv = torch.empty(0, 2, 64, dtype=BF16, device="cuda")
    simsd.simsd_rope_append_q4(plan, q, kv, kv, torch.zeros(3, **i32), torch.zeros(2, **i32), torch.empty_like(q), c, table)


def test_workspace_too_small_is_refused():
    a = attention_case(BF16, [1], [300], 8, 2, 128, 64, 2)
    out = torch.empty_like(a["q"])
    with pytest.raises(simsd.SimsdError):
        simsd.simsd_chunk_attention_q4(**a, out=out)
    with pytest.raises(simsd.SimsdError):
        simsd.simsd_chunk_attention_q4(**a, out=out, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        simsd.simsd_chunk_attention_q4(**a, out=out, workspace=torch.empty(1 << 24, dtype=torch.uint8))
    with pytest.raises(ValueError):
        simsd.simsd_chunk_attention_q4(**(a | dict(key_start=torch.zeros(2, dtype=torch.int32, device="cuda"))), out=out)


def test_pools_past_four_gigabytes():
    """Rows whose codes lie past 2^32 bytes and 2^31 rows of a head's scales:
    the same bits as from the pool's start."""
    n, Hq, Hkv, d, P = 70000, 8, 8, 128, 128
    cache = simsd.Q4Cache.zeros(n, Hkv, P, d)
    i32 = dict(dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(2)
    T = 300
    x = torch.randn(T, Hq + 2 * Hkv, d, generator=g, device="cuda").to(BF16)
    plan = simsd.simsd_rope_plan_init("half", d, THETA)
    start, zero, err = torch.tensor([0, T], **i32), torch.zeros(1, **i32), torch.zeros(1, **i32)
    got = []
    for first in (0, n - 3):
        table = torch.arange(first, first + 3, **i32)[None].contiguous()
        q = torch.empty(T, Hq, d, dtype=BF16, device="cuda")
        simsd.simsd_rope_append_q4(plan, x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], start, zero, q, cache, table,
                                   err_word=err)
        for t in cache.tensors:
            got.append(t[first:first + 3].clone())
        for rows in (1, 9, 100):  # from the registers, by tiles
            s, m = torch.tensor([0, rows], **i32), torch.tensor([T - rows], **i32)
            out = torch.empty(rows, Hq, d, dtype=BF16, device="cuda")
            ws = torch.empty(simsd.simsd_chunk_q4_workspace_bytes(simsd.SIMSD_BF16, rows, 1, Hq, Hkv, d, 3, P, n),
                             dtype=torch.uint8, device="cuda")
            simsd.simsd_chunk_attention_q4(q[T - rows:], s, m, cache, table, out, workspace=ws, err_word=err)
            got.append(out)
    half = len(got) // 2
    assert simsd.simsd_check_error(err) == 0
    assert all(torch.equal(a, b) for a, b in zip(got[:half], got[half:])) and bool(got[4].float().abs().sum() > 0)


def test_many_sequences():
    """More sequences than the kernel of few rows plans for, and chunks without
    a token."""
    Bt, Hq, Hkv, d, P = 9000, 2, 1, 64, 8
    i32 = dict(dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(4)
    has = torch.arange(Bt, device="cuda") % 3 != 1
    start = torch.cat([torch.zeros(1, **i32), torch.cumsum(has.int(), 0).int()])
    T = int(start[-1])
    cache = simsd.Q4Cache.zeros(Bt * 3, Hkv, P, d)
    table = torch.arange(Bt * 3, **i32).view(Bt, 3)
    x = torch.randn(Bt * 20, Hq + 2 * Hkv, d, generator=g, device="cuda").to(BF16)
    plan, err = simsd.simsd_rope_plan_init("half", d, THETA), torch.zeros(1, **i32)
    q = torch.empty(Bt * 20, Hq, d, dtype=BF16, device="cuda")
    simsd.simsd_rope_append_q4(plan, x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], torch.arange(Bt + 1, **i32) * 20,
                               torch.zeros(Bt, **i32), q, cache, table, err_word=err)
    q = torch.randn(T, Hq, d, generator=g, device="cuda").to(BF16)
    outs = []
    for part in (slice(0, Bt), slice(0, 3000), slice(3000, 6000), slice(6000, Bt)):
        b = table[part].contiguous()
        s = start[part.start:part.stop + 1]
        qq = q[int(s[0]):int(s[-1])].contiguous()
        out = torch.empty_like(qq)
        n = len(b)
        ws = torch.empty(simsd.simsd_chunk_q4_workspace_bytes(simsd.SIMSD_BF16, len(qq), n, Hq, Hkv, d, 3, P, Bt * 3),
                         dtype=torch.uint8, device="cuda")
        simsd.simsd_chunk_attention_q4(qq, s - s[0], torch.full((n,), 19, **i32), cache, b, out, workspace=ws,
                                       err_word=err)
        outs.append(out.float())
    assert simsd.simsd_check_error(err) == 0
    # two kernels, each off by 2^-11 of the probabilities and 2^-8 of the output at most
    diff = (outs[0] - torch.cat(outs[1:])).abs()
    assert bool((diff <= 2.0 ** -9 * 6.0 + 2.0 ** -7 * outs[0].abs()).all())


WAYS = [[1] * 6, [9, 2, 16], [60, 33, 1]]  # from the registers, lean tiles, wide tiles


@pytest.mark.parametrize("chunk", WAYS)
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("units,scale", [((2.0 ** -24, 1.0), 0.0), ((2.0 ** -64, 2.0 ** 64), 0.0), ((2.0 ** 64, 2.0 ** -64), 0.0),
                                         ((1.0, 1.0), 2.0 ** -60), ((2.0 ** -64, 1.0), 2.0 ** -140)])
def test_zero_and_small_queries_at_the_ends_of_the_units(chunk, d, units, scale):
    """Rows of q whose factor leaves fp32's normal numbers, with hidden keys
    beside them: the mean of the values that they see."""
    prefix = [300, 140, 5, 64, 0, 129][:len(chunk)]
    a = attention_case(BF16, chunk, prefix, 8, 2, d, 16, 21, units=units)
    if units[0] > 1:
        a["q"] = a["q"] / units[0]
    a["q"][0] = 0
    a["q"][1] *= 2.0 ** -100 if units[0] <= 1 else 2.0 ** -50
    a["q"][-1, :4] = 2.0 ** -126
    check(a, softmax_scale=scale)


@pytest.mark.parametrize("chunk", WAYS)
def test_large_queries_on_keys_of_zeros(chunk):
    """Scores are zero, though the factor of a row passes fp32."""
    a = attention_case(BF16, chunk, [300, 140, 5, 64, 0, 129][:len(chunk)], 8, 2, 128, 16, 22, units=(2.0 ** 64, 1.0))
    a["cache"].tensors[0].zero_()
    want = run(a | dict(q=torch.zeros_like(a["q"])))
    a["q"] = a["q"] * 2.0 ** 100
    got = run(a)
    assert got[2] == 0 and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    check(a | dict(q=torch.zeros_like(a["q"])))


@pytest.mark.parametrize("chunk", WAYS)
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("level", [20, 25, 29, 33, 60, 100, 126])
def test_scores_far_from_zero(chunk, sign, level):
    """Two levels of scores around 2^level in log2 units, of either sign: the
    mean of the values at the higher one.  Far apart as the two are, equal
    scores have weights of equal bits, so that what is left is 2^-11 for them
    in fp16, 2^-8 for the output and 2^-23 a sum."""
    prefix = [300, 140, 5, 64, 0, 129][:len(chunk)]
    a = attention_case(BF16, chunk, prefix, 8, 2, 128, 16, 23, units=(2.0 ** 64, 1.0))
    kc, ks = a["cache"].tensors[:2]
    kc.zero_()
    kc[..., 0] = torch.where(torch.arange(16, device="cuda") % 3 == 0, 7, 5).to(torch.uint8)  # 6 and 3
    ks[ks != 127] = 56  # 1
    a["q"].zero_()
    a["q"][..., 0] = sign * 1.3359375 * 2.0 ** (level - 64)
    out, lse, word = run(a, softmax_scale=0.1)
    assert word == 0
    start, table = a["token_start"].tolist(), a["block_table"].cpu().numpy()
    v = ref.decode(*(t.cpu().numpy() for t in a["cache"].tensors[2:]))
    unit = sign * float(np.float32(0.1)) * 1.3359375 * 2.0 ** level
    for b, n in enumerate(prefix):
        for i in range(chunk[b]):
            r = np.arange(n + i + 1)
            best = r % 16 % 3 == 0 if sign > 0 or len(r) == 1 else r % 16 % 3 != 0
            rows = v[table[b, r[best] // 16], :, r[best] % 16].repeat(4, 1)
            want, size = rows.mean(0), np.abs(rows).mean(0)
            got = out[start[b] + i].double().cpu().numpy()
            assert np.all(np.abs(got - want) <= (size * 2.0 ** -11 + np.abs(want) * 2.0 ** -8) * (1 + 2.0 ** -7)
                          + size * (len(r) // 128 + 72) * 2.0 ** -22), (b, i)
            score = unit * (6 if best[0] else 3)
            lw = score + math.log(best.sum())
            assert np.all(np.abs(lse[start[b] + i].double().cpu().numpy() - lw) <= 2.0 ** -21 * abs(lw)), (b, i)


@pytest.mark.parametrize("T", [1, 9, 40])  # from the registers, lean tiles, wide tiles
@pytest.mark.parametrize("d", [64, 128])
def test_many_keys_far_below_one(T, d):
    """A first row whose score is 25.5 log2 units above all others', which are
    2^18: what they add up to, 2^-7.5 of the whole, is not lost, though a CTA
    has all of a sequence.  A probability is off by 2^-32 of the largest one's
    (fp16's 2^-25, of weights of 2^7 for it), so their sum by 2^-14, the output
    by 2^-8.  A sum of weights is one of 2^11 tiles with two additions each to
    a thread's, all after the first row's 2^7: each is off by half a step, 2^-24
    of the whole, so the sum, and with it the output and e^lse, by 2^-12."""
    n, P, seqs = 2 ** 18, 128, 912
    i32 = dict(dtype=torch.int32, device="cuda")
    pages = n // P + 1
    cache = simsd.Q4Cache.zeros(pages, 1, P, d)
    kc, ks, vc, vs = cache.tensors
    ks.fill_(56)  # scale 1
    vs.fill_(56)
    vc.fill_(0x22)  # 1
    table = torch.randperm(pages, generator=torch.Generator().manual_seed(1)).int()[None].cuda()
    first = int(table[0, 0])
    kc[first, 0, 0, 0] = 7  # 6, in component 0
    vc[first, 0, 0] = 0
    q = torch.zeros(seqs * T, 4, d, dtype=BF16, device="cuda")
    q[..., 0] = 1
    scale = float(np.float32(25.5 * math.log(2) / 6))
    out, lse, word = run(dict(q=q, token_start=torch.arange(seqs + 1, **i32) * T, prefix_len=torch.full((seqs,), n, **i32),
                              cache=cache, block_table=table.repeat(seqs, 1)), softmax_scale=scale)
    assert word == 0
    rest = np.tile((n + np.arange(T)) * math.exp(-6 * scale), seqs)
    want = torch.from_numpy(rest / (1 + rest))[:, None, None].cuda()
    assert bool(((out.double() - want).abs() <= n * 2.0 ** -32 + (2.0 ** -8 + 2.0 ** -12) * want).all())
    total = 6 * scale + torch.from_numpy(np.log1p(rest))[:, None].cuda()
    assert bool(((lse.double() - total).abs() <= 2.0 ** -21 * (1 + total) + 2.0 ** -12).all())


def test_scales_next_to_their_borders():
    """Groups whose largest component lies on a border between two scales, or
    one step of fp32 beside it: the nearest scale, on the border the even one
    (a border times 6 is exact in fp32)."""
    borders = (ref.SCALES[1:126] + ref.SCALES[2:127]) / 2
    top = np.float32(6 * borders)
    assert np.array_equal(top.astype(np.float64), 6 * borders)
    x = np.concatenate([[np.nextafter(t, np.float32(0)), t, np.nextafter(t, np.float32(np.inf))] for t in top])
    x = np.concatenate([x, -x, [0] * (-2 * len(x) % 4)]).astype(np.float32)
    T = len(x) // 4
    v = torch.zeros(T, 4, 16)
    v[:, :, 5] = torch.from_numpy(x).view(T, 4)
    v = v.view(T, 1, 64).cuda()
    i32 = dict(dtype=torch.int32, device="cuda")
    pages = (T + 7) // 8
    cache = simsd.Q4Cache.zeros(pages, 1, 8, 64)
    q = torch.empty_like(v)
    # (at position 0 keys are turned by nothing)
    simsd.simsd_rope_append_q4(simsd.simsd_rope_plan_init("half", 64, THETA), v, v, v, torch.tensor([0, T], **i32),
                               torch.zeros(1, **i32), q, cache, torch.arange(pages, **i32)[None], positions=torch.zeros(T, **i32))
    want = ref.encode(v.double().cpu().numpy()[:, 0])
    for c, s in (cache.tensors[:2], cache.tensors[2:]):
        got = ref.decode(*(t.view(pages * 8, -1)[:T].cpu().numpy() for t in (c, s)))
        assert np.array_equal(got, want)


@pytest.mark.parametrize("unit", [0.7, 3.3, 1.7e-5, 1e10])
def test_quotients_by_the_unit(unit):
    """Components on the borders between two codes and next to them, times a
    unit that is no power of two: codes of x / unit as fp32 has it, correctly
    rounded, ties to the even code."""
    u = np.float32(unit)
    rng = np.random.RandomState(3)
    T = 300
    s = ref.SCALES[rng.randint(8, 126, (T, 4))]
    x = (((ref.LEVELS[1:] + ref.LEVELS[:-1]) / 2)[rng.randint(0, 7, (T, 4, 16))] * s[..., None]).astype(np.float32) * u
    x[..., 0] = np.float32(6 * s) * u
    step = rng.randint(-2, 3, x.shape)
    for k in (1, 2):
        x = np.where(step >= k, np.nextafter(x, np.float32(np.inf)), np.where(step <= -k, np.nextafter(x, np.float32(0)), x))
    x = (x * rng.choice([-1, 1], x.shape)).astype(np.float32)
    v = torch.from_numpy(x).view(T, 1, 64).cuda()
    i32 = dict(dtype=torch.int32, device="cuda")
    pages = (T + 7) // 8
    cache = simsd.Q4Cache.zeros(pages, 1, 8, 64, float(u), float(u))
    simsd.simsd_rope_append_q4(simsd.simsd_rope_plan_init("half", 64, THETA), v, v, v, torch.tensor([0, T], **i32),
                               torch.zeros(1, **i32), torch.empty_like(v), cache, torch.arange(pages, **i32)[None],
                               positions=torch.zeros(T, **i32))
    want = ref.encode((x / u).astype(np.float64)).reshape(T, 64)
    for c, s in (cache.tensors[:2], cache.tensors[2:]):
        got = ref.decode(*(t.view(pages * 8, -1)[:T].cpu().numpy() for t in (c, s)))
        assert np.array_equal(got, want)


def test_quotients_that_pass_fp32():
    """x / unit beyond fp32 is an infinity: the largest scale, 6 or -6."""
    v = torch.zeros(1, 1, 64, device="cuda")
    v[0, 0, 0], v[0, 0, 20] = 1e30, -3e38
    i32 = dict(dtype=torch.int32, device="cuda")
    cache = simsd.Q4Cache.zeros(1, 1, 8, 64, 2.0 ** -64, 2.0 ** -63 * 1.3)
    simsd.simsd_rope_append_q4(simsd.simsd_rope_plan_init("half", 64, THETA), v, v, v, torch.tensor([0, 1], **i32),
                               torch.zeros(1, **i32), torch.empty_like(v), cache, torch.zeros(1, 1, **i32))
    want = np.zeros(64)
    want[0], want[20] = 2688, -2688
    for c, s in (cache.tensors[:2], cache.tensors[2:]):
        assert np.array_equal(ref.decode(*(t[0, 0, 0].cpu().numpy() for t in (c, s))), want)


def test_expand_near_the_last_row():
    """Rows next to 2^31, where a row number plus a page passes 32 bits."""
    P, d = 704, 64
    max_pages = 0x7fffff00 // P
    top = max_pages * P
    assert top + P - 1 >= 2 ** 31
    i32 = dict(dtype=torch.int32, device="cuda")
    cache = simsd.Q4Cache.zeros(2, 1, P, d)
    for t in cache.tensors:
        t.random_(0, 127)
    table = torch.full((1, max_pages), -1, **i32)
    table[0, -2], table[0, -1] = 1, 0
    outs = []
    for tb, first, last in ((table, top - P - 9, top), (torch.tensor([[1, 0]], **i32), P - 9, 2 * P)):
        out = [torch.full((2, 1, P, d), 5.0, dtype=BF16, device="cuda") for _ in range(2)]
        err = torch.zeros(1, **i32)
        simsd.simsd_q4_expand(cache, tb, torch.tensor([first], **i32), torch.tensor([last], **i32), *out, err_word=err)
        assert simsd.simsd_check_error(err) == 0
        outs.append(torch.stack(out))
    assert torch.equal(outs[0], outs[1]) and bool((outs[0][:, 0] != 5).any()) and bool((outs[0][:, 1, 0, :P - 9] == 5).all())


def test_expand_of_more_than_2_to_the_31_pages_and_heads():
    """2^19 entries (of one page, but for the first and the last) of 4096
    heads: all that they name is written."""
    Hkv, P, d, n = 4096, 8, 64, 2 ** 19 + 3
    i32 = dict(dtype=torch.int32, device="cuda")
    cache = simsd.Q4Cache.zeros(3, Hkv, P, d)
    for t in cache.tensors:
        t.random_(0, 127)
    table = torch.ones(1, n, **i32)
    table[0, 0], table[0, -1] = 0, 2
    outs = []
    for tb in (table, torch.tensor([[0, 1, 2]], **i32)):
        out = [torch.full((3, Hkv, P, d), 5.0, dtype=BF16, device="cuda") for _ in range(2)]
        err = torch.zeros(1, **i32)
        last = tb.shape[1] * P
        simsd.simsd_q4_expand(cache, tb, torch.zeros(1, **i32), torch.tensor([last], **i32), *out, err_word=err)
        assert simsd.simsd_check_error(err) == 0
        outs.append(torch.stack(out))
    assert torch.equal(outs[0], outs[1]) and not bool((outs[0] == 5).flatten(2).all(2).any())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("window,sinks", [(0, 0), (90, 5)])
@pytest.mark.parametrize("chunk", [[200] + [0] * 63 + [1] * 6, [64] + [0] * 63, [0] * 30 + [300] + [1] * 40, [33, 1, 0, 0] * 9,
                                   [1] * 40 + [0] * 40, [600, 0, 0]])
def test_long_chunks_beside_single_tokens_and_empty_slots(dtype, window, sinks, chunk):
    """Averages over sequences that say little about any of them."""
    prefix = [(37 * b) % 300 for b in range(len(chunk))]
    check(attention_case(dtype, chunk, prefix, 4, 1, 64, 16, len(chunk), window, sinks), window, sinks)


@pytest.mark.parametrize("T", [1, 9, 60])
@pytest.mark.parametrize("level", [23, 24, 25, 26, 27, 28])
def test_scores_far_from_zero_that_rise(T, level):
    """Scores of about 2^level in log2 units, from the second tile on 5 to 30
    above those of the first, where a sum of such a score and a small number is
    rounded to a multiple of up to 32: no weight passes fp16, and the output is
    a mean of the values."""
    n, P, seqs = 300, 16, 64
    i32 = dict(dtype=torch.int32, device="cuda")
    pages = (n + T + P - 1) // P
    cache = simsd.Q4Cache.zeros(pages, 1, P, 64)
    kc, ks, vc, vs = cache.tensors
    ks.fill_(56)
    vs.fill_(56)
    kc[:, :, :, 0] = 2  # 1 in component 0
    kc[8:, :, :, 8] = 2  # and, from row 128 on, in component 16
    vc.fill_(0x22)  # 1
    vc[8:] = 0x44  # 2
    q = torch.zeros(seqs * T, 4, 64, dtype=BF16, device="cuda")
    sign = torch.where(torch.arange(seqs * T, device="cuda") % 2 == 0, 1.0, -1.0)[:, None]
    q[..., 0] = sign * 2.0 ** level * math.log(2)
    q[..., 16] = torch.linspace(5, 30, seqs * T * 4, device="cuda").view(seqs * T, 4) * math.log(2)
    out, lse, word = run(dict(q=q, token_start=torch.arange(seqs + 1, **i32) * T, prefix_len=torch.full((seqs,), n, **i32),
                              cache=cache, block_table=torch.arange(pages, **i32).repeat(seqs, 1)), softmax_scale=1.0)
    assert word == 0 and bool(torch.isfinite(lse).all())
    assert bool(((out >= 1) & (out <= 2)).all())

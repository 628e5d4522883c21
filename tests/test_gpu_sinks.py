"""Attention through a window whose first rows stay visible, on the GPU,
against the plain 64-bit form; rows that nobody sees are NaN and their pages
are released."""
import math

import numpy as np
import pytest
import torch

from paper_2606_02544_gb300 import simsd
from tests import _longcache as ref
from tests import _prompt

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def make(dtype, chunk, prefix, Hq, Hkv, d, P, seed, window, sinks, block=1, key_start=None, std=1.0, hide=True):
    """Chunks over a shuffled pool; pages of rows that no token sees are not
    in the table, rows beside those that are seen are NaN."""
    g = torch.Generator().manual_seed(seed)
    T = sum(chunk)
    start = np.concatenate([[0], np.cumsum(chunk)]).astype(np.int32)
    ks = key_start or [0] * len(chunk)
    seen = []
    for n, c, s in zip(prefix, chunk, ks):
        rows = [ref.visible(n, c, i, block, window, s, sinks) for i in range(c)]
        seen.append(np.unique(np.concatenate(rows)) if rows else np.array([], dtype=int))
    width = max((n + c + P - 1) // P for n, c in zip(prefix, chunk))
    table = torch.full((len(chunk), max(width, 1)), -1, dtype=torch.int32)
    pool = sum(len(np.unique(r // P)) for r in seen) + 3
    perm = torch.randperm(pool, generator=g).int()
    kc = torch.randn(pool, Hkv, P, d, generator=g).mul_(std).to(dtype)
    vc = torch.randn(pool, Hkv, P, d, generator=g).mul_(std).to(dtype)
    keep, at = torch.zeros(pool, P, dtype=torch.bool), 0
    for b, r in enumerate(seen):
        pages = np.unique(r // P)
        table[b, pages] = perm[at:at + len(pages)]
        at += len(pages)
        r = torch.as_tensor(r)
        keep[table[b, r // P].long(), r % P] = True
    if hide:
        kc.masked_fill_(~keep[:, None, :, None], float("nan"))
        vc.masked_fill_(~keep[:, None, :, None], float("nan"))
    i32 = dict(dtype=torch.int32, device="cuda")
    q = torch.randn(T, Hq, d, generator=g).mul_(std).to(dtype).cuda()
    return dict(q=q, token_start=torch.tensor(start, **i32), prefix_len=torch.tensor(prefix, **i32),
                k_cache=kc.cuda(), v_cache=vc.cuda(), block_table=table.cuda(),
                key_start=torch.tensor(ks, **i32) if key_start else None)


def run(a, **kw):
    T, Hq, d = a["q"].shape
    out = torch.full((T, Hq, d), float("nan"), dtype=a["q"].dtype, device="cuda")
    lse = torch.full((T, Hq), float("nan"), device="cuda")
    code = simsd.SIMSD_F32 if a["q"].dtype == F32 else simsd.SIMSD_BF16
    n = simsd.simsd_chunk_workspace_bytes(code, T, len(a["prefix_len"]), Hq, a["k_cache"].shape[1], d,
                                          a["block_table"].shape[1], a["k_cache"].shape[2])
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda") if n else None
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    simsd.simsd_chunk_attention_sinks(**a, out=out, lse=lse, workspace=ws, err_word=err, **kw)
    return out, lse, simsd.simsd_check_error(err)


def check(a, window, sinks, mask_block=1, softmax_scale=0.0):
    out, lse, word = run(a, window=window, sinks=sinks, mask_block=mask_block, softmax_scale=softmax_scale)
    assert word == 0
    compare(a, out, lse, a["k_cache"].double().cpu().numpy(), a["v_cache"].double().cpu().numpy(), window, sinks,
            mask_block, softmax_scale, lambda o, av, qk, N, vm: _prompt.attention_tolerance(o, av, qk, N, a["q"].dtype == BF16))


def compare(a, out, lse, kd, vd, window, sinks, mask_block, softmax_scale, tolerance):
    start, prefix = a["token_start"].tolist(), a["prefix_len"].tolist()
    P, d = kd.shape[2:]
    scale = softmax_scale or 1 / math.sqrt(d)
    q, table = a["q"].double().cpu().numpy(), a["block_table"].cpu().numpy()
    for b, n in enumerate(prefix):
        s, C = start[b], start[b + 1] - start[b]
        if C == 0:
            continue
        N = n + C
        rows = np.arange(N)
        k, v = kd[table[b, rows // P], :, rows % P], vd[table[b, rows // P], :, rows % P]
        first = int(a["key_start"][b]) if a["key_start"] is not None else 0
        want, wl, absv = ref.attention(q[s:s + C], k, v, n, C, scale, mask_block, window, first, sinks)
        qk = scale * np.linalg.norm(q[s:s + C], axis=-1).max() * np.nan_to_num(np.linalg.norm(k, axis=-1)).max()
        got, gl = out[s:s + C].double().cpu().numpy(), lse[s:s + C].double().cpu().numpy()
        assert np.isfinite(got).all()
        assert np.all(np.abs(got - want) <= tolerance(want, absv, qk, N, np.nan_to_num(np.abs(v)).max())), b
        none = np.isinf(wl)
        assert np.array_equal(np.isneginf(gl), none)
        assert np.all(got[none] == 0)
        assert np.all(np.abs(gl[~none] - wl[~none]) <= _prompt.lse_tolerance(wl[~none], qk, N)), b


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("window,sinks,block", [(1, 1, 1), (5, 3, 1), (130, 4, 1), (128, 128, 16), (300, 129, 0),
                                                (64, 700, 1), (256, 16, 32), (97, 1, 7)])
def test_windows(dtype, window, sinks, block):
    """Parts that touch, overlap or lie far apart; chunks of one token to
    several tiles; rows without a prefix."""
    chunk, prefix = [1, 1, 17, 70, 1, 0, 33], [700, 3, 511, 0, 0, 40, 385]
    check(make(dtype, chunk, prefix, 8, 2, 128, 16, window + sinks, window, sinks, block), window, sinks, block)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("Hq,Hkv,d,P", [(7, 1, 64, 8), (4, 4, 128, 64), (8, 1, 64, 192), (16, 2, 128, 128)])
def test_layouts(dtype, Hq, Hkv, d, P):
    chunk, prefix = [3, 1, 140], [900, 260, 131]
    check(make(dtype, chunk, prefix, Hq, Hkv, d, P, Hq + P, 100, 10), 100, 10)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_first_rows_after_key_start(dtype):
    """The first visible rows are those from key_start on; past a token's own
    row there is nothing to see."""
    chunk, prefix, ks = [5, 40, 30, 9, 1], [300, 500, 100, 64, 0], [200, 129, 110, 80, 0]
    check(make(dtype, chunk, prefix, 4, 2, 128, 16, 5, 50, 6, key_start=ks), 50, 6)
    check(make(dtype, chunk, prefix, 4, 2, 64, 8, 6, 20, 200, 4, key_start=ks), 20, 200, 4)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_without_a_window_or_first_rows(dtype):
    """sinks without a window, and a window without sinks: the bits of
    simsd_chunk_attention."""
    a = make(dtype, [40, 1], [200, 700], 8, 2, 128, 16, 3, 0, 0, hide=False)
    T, Hq, d = a["q"].shape
    code = simsd.SIMSD_F32 if dtype == F32 else simsd.SIMSD_BF16
    n = simsd.simsd_chunk_workspace_bytes(code, T, 2, Hq, 2, d, a["block_table"].shape[1], 16)
    for window, sinks in ((0, 9), (77, 0)):
        out, lse, word = run(a, window=window, sinks=sinks)
        o2, l2 = torch.empty_like(out), torch.empty_like(lse)
        ws = torch.empty(max(1, n), dtype=torch.uint8, device="cuda")
        simsd.simsd_chunk_attention(**a, out=o2, lse=l2, window=window, workspace=ws)
        assert word == 0 and torch.equal(out, o2) and torch.equal(lse, l2)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_first_rows_that_reach_the_window_change_nothing(dtype):
    """With as many first rows as the sequence has, every earlier row is seen."""
    a = make(dtype, [20, 1, 130], [300, 600, 5], 8, 2, 128, 16, 8, 0, 0, hide=False)
    check(a, 30, 10 ** 9)
    a["key_start"] = torch.tensor([2 ** 31 - 5, 100, 0], dtype=torch.int32, device="cuda")
    check(a, 30, 2 ** 31 - 1)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_bad_pages_and_lengths(dtype):
    """A missing page of the first rows or of the window zeroes what sees it
    and raises; the other sequence is right."""
    for gone in (0, 20):
        a = make(dtype, [1, 1], [400, 390], 8, 2, 64, 16, 4, 90, 8)
        page = int(a["block_table"][0, gone])
        assert (page >= 0) == (gone == 0 or gone >= (400 - 89) // 16)
        a["block_table"][0, gone] = 10 ** 6
        out, lse, word = run(a, window=90, sinks=8)
        assert word == simsd.EW_PAGE and bool((out[0] == 0).all()) and bool(torch.isneginf(lse[0]).all())
        assert bool((out[1] != 0).any()) and bool(torch.isfinite(out[1].float()).all())
    a = make(dtype, [1, 1], [400, 390], 8, 2, 64, 16, 4, 90, 8)
    a["prefix_len"][0] = -1
    out, lse, word = run(a, window=90, sinks=8)
    assert word == simsd.EW_PREFIX_LEN and bool((out[0] == 0).all())
    assert bool(torch.isfinite(out[1].float()).all())


def test_long_cache_few_pages():
    """A window over a table of 131072 rows of which a few pages exist."""
    check(make(BF16, [1, 2], [131000, 70001], 8, 2, 128, 64, 9, 256, 4), 256, 4)
    check(make(F32, [1, 2], [131000, 70001], 8, 2, 128, 64, 9, 256, 4), 256, 4)


def test_large_scores():
    """References that move: scores of some hundreds, first rows above and
    below the window's."""
    a = make(BF16, [2, 60], [500, 300], 8, 2, 128, 16, 11, 64, 20, std=3.0)
    check(a, 64, 20)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("window,sinks", [(0, 0), (90, 5)])
@pytest.mark.parametrize("chunk", [[70] + [0] * 63 + [1] * 6, [64] + [0] * 63, [65] + [0] * 63, [0] * 30 + [300] + [1] * 40,
                                   [33, 1, 0, 0] * 9, [1] * 40 + [0] * 40, [2] + [1] * 38 + [0]])
def test_long_chunks_beside_single_tokens_and_empty_slots(dtype, window, sinks, chunk):
    """Averages over sequences that say little about any of them."""
    prefix = [(37 * b) % 300 for b in range(len(chunk))]
    check(make(dtype, chunk, prefix, 4, 1, 64, 16, len(chunk), window, sinks), window, sinks)


@pytest.mark.parametrize("dtype,level", [(BF16, 20), (BF16, 25), (BF16, 29), (F32, 29), (F32, 120)])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("chunk", [[1] * 4, [60, 33, 1, 90]])
def test_scores_far_from_zero(dtype, level, sign, chunk):
    """Two levels of scores of either sign, the higher one of magnitude up to
    2^29 (fp32: further): the mean of the values at it."""
    prefix = [300, 140, 5, 64]
    a = make(dtype, chunk, prefix, 8, 2, 64, 16, 31, 0, 0, hide=False)
    a["k_cache"].zero_()
    a["k_cache"][..., 0] = torch.where(torch.arange(16, device="cuda") % 3 == 0, 1.0, 0.5).to(dtype)
    a["q"].zero_()
    a["q"][..., 0] = sign * 1.3359375 * 2.0 ** level
    scale = float(np.float32(0.7))
    out, lse, word = run(a, window=0, sinks=0, softmax_scale=scale)
    assert word == 0
    start, table = a["token_start"].tolist(), a["block_table"].cpu().numpy()
    v = a["v_cache"].double().cpu().numpy()
    for b, n in enumerate(prefix):
        for i in range(chunk[b]):
            r = np.arange(n + i + 1)
            best = r % 16 % 3 == 0 if sign > 0 or len(r) == 1 else r % 16 % 3 != 0
            rows = v[table[b, r[best] // 16], :, r[best] % 16].repeat(4, 1)
            want, size = rows.mean(0), np.abs(rows).mean(0)
            got = out[start[b] + i].double().cpu().numpy()
            # equal weights in bf16 are off by 2^-8 of their like in the sum, outputs by 2^-8
            tol = (size + np.abs(want)) * 2.0 ** -8 * (1 + 2.0 ** -7) if dtype == BF16 else size * 2.0 ** -20
            assert np.all(np.abs(got - want) <= tol + size * (len(r) // 64 + 72) * 2.0 ** -22), (b, i)
            lw = sign * scale * 1.3359375 * 2.0 ** level * (1.0 if best[0] else 0.5) + math.log(best.sum())
            assert np.all(np.abs(lse[start[b] + i].double().cpu().numpy() - lw) <= 2.0 ** -21 * abs(lw)), (b, i)

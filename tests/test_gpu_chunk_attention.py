"""Attention of chunks of new tokens over the paged cache on the GPU, against
the plain 64-bit form."""
import math

import numpy as np
import pytest
import torch

from paper_2606_02544_gb300 import simsd
from tests import _prompt as ref

pytestmark = pytest.mark.gpu


def make(dtype, chunk, prefix, Hq, Hkv, d, P, seed, std=1.0, poison=True, key_start=None):
    """Chunks over a shuffled page pool; rows that no token may see (past the
    end, before key_start, spare pages) are NaN."""
    g = torch.Generator().manual_seed(seed)
    T = sum(chunk)
    start = np.concatenate([[0], np.cumsum(chunk)]).astype(np.int32)
    pages = [(n + c + P - 1) // P for n, c in zip(prefix, chunk)]
    pool = sum(pages) + 2
    perm = torch.randperm(pool, generator=g)
    table = torch.full((len(chunk), max(max(pages), 1)), -1, dtype=torch.int32)
    kc = torch.randn(pool, Hkv, P, d, generator=g).mul_(std).to(dtype)
    vc = torch.randn(pool, Hkv, P, d, generator=g).mul_(std).to(dtype)
    seen = torch.zeros(pool, P, dtype=torch.bool)
    at = 0
    for b, c in enumerate(pages):
        table[b, :c] = perm[at:at + c]
        at += c
        rows = torch.arange(max(0, key_start[b] if key_start else 0), prefix[b] + chunk[b])
        if len(rows):
            seen[table[b, rows // P].long(), rows % P] = True
    if poison:
        kc.masked_fill_(~seen[:, None, :, None], float("nan"))
        vc.masked_fill_(~seen[:, None, :, None], float("nan"))
    i32 = dict(dtype=torch.int32, device="cuda")
    q = torch.randn(T, Hq, d, generator=g).mul_(std).to(dtype).cuda()
    return dict(q=q, token_start=torch.tensor(start, **i32), prefix_len=torch.tensor(prefix, **i32),
                k_cache=kc.cuda(), v_cache=vc.cuda(), block_table=table.cuda(),
                key_start=torch.tensor(key_start, **i32) if key_start else None)


def run(a, **kw):
    T, Hq, d = a["q"].shape
    out = torch.full((T, Hq, d), float("nan"), dtype=a["q"].dtype, device="cuda")
    lse = torch.full((T, Hq), float("nan"), device="cuda")
    code = simsd.SIMSD_F32 if a["q"].dtype == torch.float32 else simsd.SIMSD_BF16
    n = simsd.simsd_chunk_workspace_bytes(code, T, len(a["prefix_len"]), Hq, a["k_cache"].shape[1], d,
                                          a["block_table"].shape[1], a["k_cache"].shape[2])
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda") if n else None  # NaN bits: it needs no initial value
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    simsd.simsd_chunk_attention(**a, out=out, lse=lse, workspace=ws, err_word=err, **kw)
    return out, lse, simsd.simsd_check_error(err)


def check(a, **kw):
    out, lse, word = run(a, **kw)
    assert word == 0
    start, prefix = a["token_start"].tolist(), a["prefix_len"].tolist()
    P, d = a["k_cache"].shape[2:]
    scale = kw.get("softmax_scale") or 1 / math.sqrt(d)
    bf16 = a["q"].dtype == torch.bfloat16
    kd, vd = a["k_cache"].double().cpu().numpy(), a["v_cache"].double().cpu().numpy()
    q, table = a["q"].double().cpu().numpy(), a["block_table"].cpu().numpy()
    for b, n in enumerate(prefix):
        s, C = start[b], start[b + 1] - start[b]
        if C == 0:
            continue
        N = n + C
        rows = np.arange(N)
        k, v = kd[table[b, rows // P], :, rows % P], vd[table[b, rows // P], :, rows % P]
        first = int(a["key_start"][b]) if a["key_start"] is not None else 0
        want, wl, absv = ref.attention(q[s:s + C], k, v, n, C, scale, kw.get("mask_block", 1), kw.get("window", 0),
                                       first)
        qk = scale * np.linalg.norm(q[s:s + C], axis=-1).max() * np.nan_to_num(np.linalg.norm(k, axis=-1)).max()
        got, gl = out[s:s + C].double().cpu().numpy(), lse[s:s + C].double().cpu().numpy()
        assert np.isfinite(got).all()
        assert np.all(np.abs(got - want) <= ref.attention_tolerance(want, absv, qk, N, bf16)), b
        empty = np.isneginf(wl)
        assert np.array_equal(np.isneginf(gl), empty)
        assert (got[empty] == 0).all()
        assert np.all(np.abs(gl[~empty] - wl[~empty]) <= ref.lse_tolerance(wl, qk, N)[~empty]), b
    return out, lse


DTYPES = [torch.bfloat16, torch.float32]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("chunk,prefix", [([1], [0]), ([1], [1]), ([2, 1, 1], [127, 128, 129]), ([33, 1, 64], [0, 200, 63]),
                                          ([0, 5, 0], [9, 0, 0]), ([150], [300])])
def test_lengths(dtype, d, chunk, prefix):
    check(make(dtype, chunk, prefix, 4, 2, d, 64, 1))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (3, 3), (8, 1), (14, 2), (40, 8), (128, 1), (66, 2)])
def test_heads(dtype, Hq, Hkv):
    check(make(dtype, [5, 18], [70, 3], Hq, Hkv, 64, 16, 2))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("P", [8, 16, 32, 64, 128, 192])
def test_page_sizes(dtype, P):
    check(make(dtype, [40, 3], [301, 127], 4, 2, 64, P, 3))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("block", [0, 1, 4, 16, 100])
@pytest.mark.parametrize("window", [0, 1, 30, 200])
def test_masks(dtype, block, window):
    check(make(dtype, [45, 7], [33, 260], 4, 2, 64, 16, 4), mask_block=block, window=window)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("window", [0, 20])
def test_hidden_keys_and_empty_rows(dtype, window):
    """Hidden rows hold NaN; in the second sequence the first tokens see
    nothing, in the third none does."""
    check(make(dtype, [20, 30, 10, 3], [100, 40, 5, 300], 4, 2, 64, 16, 5, key_start=[60, 55, 15, 290]), window=window)


@pytest.mark.parametrize("dtype", DTYPES)
def test_hidden_pages_need_no_page(dtype):
    a = make(dtype, [4], [500], 4, 2, 64, 16, 6, key_start=[300])
    a["block_table"][0, :300 // 16] = -1  # evicted
    check(a)


@pytest.mark.parametrize("dtype", DTYPES)
def test_many_single_tokens(dtype):
    r = np.random.default_rng(7)
    check(make(dtype, [1] * 70, [int(x) for x in r.integers(0, 400, 70)], 8, 2, 64, 32, 7))


@pytest.mark.parametrize("dtype", DTYPES)
def test_long_cache_is_cut_over_ctas(dtype):
    """One token over 20000 rows: its units are cut over all SMs and merged."""
    check(make(dtype, [1], [20000], 4, 2, 128, 64, 8, std=0.3))


@pytest.mark.parametrize("dtype", DTYPES)
def test_units_cut_by_run_ends(dtype):
    """Chunks whose runs end inside units with both row blocks."""
    check(make(dtype, [333, 1, 190], [700, 900, 0], 4, 2, 64, 64, 9))


@pytest.mark.parametrize("dtype", DTYPES)
def test_growing_scores_move_the_reference(dtype):
    """Scores that rise along the keys by far more than 2^8."""
    a = make(dtype, [3], [900], 2, 1, 64, 64, 10)
    ramp = torch.linspace(0.0, 6.0, 903)
    P = 64
    rows = torch.arange(903)
    page = a["block_table"][0].cpu()[rows // P].long()
    k = a["k_cache"].cpu()
    k[page, :, rows % P] = (k[page, :, rows % P].float() * 0.1 + ramp[:, None, None]).to(dtype)
    a["k_cache"] = k.cuda()
    a["q"] = a["q"].abs() + 1.0
    check(a, softmax_scale=0.5)


@pytest.mark.parametrize("dtype", DTYPES)
def test_strided_queries_and_scale(dtype):
    a = make(dtype, [9, 40], [100, 0], 4, 2, 128, 64, 11)
    wide = torch.randn(49, 8, 128, device="cuda").to(dtype)
    wide[:, :4] = a["q"]
    dense = check(a, softmax_scale=0.05)
    a["q"] = wide[:, :4]
    strided = check(a, softmax_scale=0.05)
    assert torch.equal(dense[0], strided[0]) and torch.equal(dense[1], strided[1])


@pytest.mark.parametrize("dtype", DTYPES)
def test_same_bits_every_time_and_on_another_stream(dtype):
    a = make(dtype, [64, 5, 200], [1000, 30, 0], 8, 2, 128, 64, 12)
    o1, l1, _ = run(a)
    o2, l2, _ = run(a)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        o3, l3, _ = run(a)
    s.synchronize()
    assert torch.equal(o1, o2) and torch.equal(o1, o3) and torch.equal(l1, l2) and torch.equal(l1, l3)


@pytest.mark.parametrize("dtype", DTYPES)
def test_data_errors(dtype):
    a = make(dtype, [3, 4, 5], [30, 70, 0], 4, 2, 64, 16, 13)
    good, _, _ = run(a)
    b = dict(a, prefix_len=a["prefix_len"].clone())
    b["prefix_len"][1] = 80  # no room for the chunk
    out, lse, word = run(b)
    assert word == simsd.EW_PREFIX_LEN
    assert (out[3:7] == 0).all() and torch.isneginf(lse[3:7]).all()
    assert torch.equal(out[:3], good[:3]) and torch.equal(out[7:], good[7:])
    c = dict(a, block_table=a["block_table"].clone())
    c["block_table"][1, 2] = a["k_cache"].shape[0]
    out, lse, word = run(c)
    assert word == simsd.EW_PAGE
    assert (out[3:7] == 0).all() and torch.equal(out[:3], good[:3]) and torch.equal(out[7:], good[7:])
    e = dict(a, token_start=a["token_start"].clone())
    e["token_start"][:] = torch.tensor([0, 3, 2, 12])
    out, lse, word = run(e)
    assert word == simsd.EW_TOKENS
    assert torch.equal(out[:2], good[:2])


def test_bad_page_in_one_piece_of_a_cut_unit():
    """A unit cut over several CTAs is zero as a whole."""
    a = make(torch.bfloat16, [1], [9000], 4, 2, 64, 64, 14, std=0.3)
    a["block_table"][0, 100] = -7
    out, lse, word = run(a)
    assert word == simsd.EW_PAGE
    assert (out == 0).all() and torch.isneginf(lse).all()


def test_workspace_is_checked():
    a = make(torch.bfloat16, [4], [100], 4, 2, 64, 64, 15)
    out = torch.empty_like(a["q"])
    with pytest.raises(simsd.SimsdError) as e:
        simsd.simsd_chunk_attention(**a, out=out, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    assert e.value.status == simsd.SIMSD_ERR_INVALID_ARG
    with pytest.raises(simsd.SimsdError) as e:
        b = make(torch.bfloat16, [4], [100], 130, 1, 64, 64, 15)
        simsd.simsd_chunk_attention(**b, out=torch.empty_like(b["q"]),
                                    workspace=torch.empty(1 << 27, dtype=torch.uint8, device="cuda"))
    assert e.value.status == simsd.SIMSD_ERR_UNSUPPORTED


def test_chunks_of_a_prompt_equal_the_whole():
    """A prompt in chunks of any size sees what the whole prompt sees: each
    token's row agrees within the rounding of both."""
    a = make(torch.bfloat16, [500], [0], 4, 2, 128, 64, 16, std=0.5)
    whole, _ = check(a, mask_block=16)
    parts = []
    for lo, hi in ((0, 16), (16, 240), (240, 496), (496, 500)):
        b = dict(a, q=a["q"][lo:hi].contiguous(),
                 token_start=torch.tensor([0, hi - lo], dtype=torch.int32, device="cuda"),
                 prefix_len=torch.tensor([lo], dtype=torch.int32, device="cuda"))
        parts.append(run(b, mask_block=16)[0])
    got = torch.cat(parts).double()
    # each side rounds P and O to bf16: twice the bound's leading terms, |v| <= 3.5 std here
    assert (got - whole.double()).abs().max().item() <= 2 * 2.0 ** -8 * 2 * 3.5 * 0.5


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 2), (12, 2), (16, 2), (18, 2)])
def test_few_rows_over_long_caches(dtype, d, Hq, Hkv):
    """Single tokens and short drafts; the fp32 kernel for few rows takes its
    keys 256 at a time, four to a warp's step."""
    prefix = [255, 256, 1030, 3, 700]
    check(make(dtype, [1] * 5, prefix, Hq, Hkv, d, 16, 11))
    check(make(dtype, [2, 1, 0, 3, 1], prefix, Hq, Hkv, d, 8, 12, key_start=[0, 250, 0, 2, 699]), window=300)
    check(make(dtype, [1, 2, 1, 1, 1], prefix, Hq, Hkv, d, 128, 13), mask_block=2, window=7)


@pytest.mark.parametrize("dtype", DTYPES)
def test_many_heads_and_long_chunks(dtype):
    """So many query rows that the fp32 kernel takes them 128 at a time."""
    check(make(dtype, [300, 130, 40], [100, 0, 333], 64, 64, 64, 32, 14), mask_block=4)


# (chunk, prefix, Hq, Hkv, key_start, mask arguments): so many key tiles a SM that a CTA's run holds several units,
# a unit of one row block (few tokens, many keys) before one of two blocks whose first tile is seen in part
RUNS = {
    "single tokens before fresh chunks": ([1, 100] * 6, [600, 0, 333, 0, 1900, 0, 1000, 0, 256, 0, 1290, 27], 128, 64,
                                          None, {}),
    "short chunks before windows and hidden keys": (
        [3, 90, 1, 70, 5, 127, 2, 66], [1500, 333, 700, 50, 1100, 900, 2000, 0], 96, 48,
        [77, 0, 0, 51, 300, 901, 1000, 3], dict(window=200, mask_block=4)),
    "prompts that end in a short unit": ([1096, 8, 200], [0, 1000, 0], 64, 16, None, {}),
    "prompts that end in a short unit, unmasked": ([70, 520], [700, 24], 32, 8, [0, 100], dict(mask_block=0)),
}


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("case", list(RUNS))
def test_runs_of_several_units(case, d):
    chunk, prefix, Hq, Hkv, key_start, mask = RUNS[case]
    check(make(torch.bfloat16, chunk, prefix, Hq, Hkv, d, 16, 17, key_start=key_start), **mask)


@pytest.mark.parametrize("d", [64, 128])
def test_the_reference_moves_in_some_rows_of_every_tile(d):
    """Each tile of keys holds a few that lie far above all before them for
    some of the rows: the first half of the probabilities is stored against
    the old reference, then again against the new one."""
    a = make(torch.bfloat16, [150, 60], [900, 0], 8, 4, d, 64, 18)
    P, scale = 64, 0.5
    k = a["k_cache"].cpu()
    q = a["q"].cpu()
    for b, (n, C, s) in enumerate([(900, 150, 0), (0, 60, 150)]):
        for j in range(5, n + C, 37):
            page = a["block_table"][b].cpu()[j // P].long()
            # along the query of one token: its score grows from tile to tile
            k[page, :, j % P] = (q[s + (7 * j) % C, ::2].float() * (0.2 + 0.8 * j / 1050)).to(torch.bfloat16)
    a["k_cache"] = k.cuda()
    check(a, softmax_scale=scale, mask_block=16)


def test_offsets_that_overlap_many_times_over():
    """8192 chunks of the same 8192 tokens over 300,000 rows: about 5 10^9 key
    tiles, past the 32 bits that they are counted in.  Nothing is computed and
    nothing written."""
    Bt, T, Hkv, d, P = 16384, 8192, 8, 64, 1024
    i32 = dict(dtype=torch.int32, device="cuda")
    n = 300 * P
    tiles = Bt // 2 * sum(-(-(n + 256 * (j + 1)) // 128) for j in range(T // 256)) * Hkv
    assert tiles > 2 * 2 ** 31
    q = torch.zeros(T, Hkv, d, dtype=torch.bfloat16, device="cuda")
    out, lse = torch.full_like(q, 7.0), torch.full((T, Hkv), 7.0, device="cuda")
    start = torch.zeros(Bt + 1, **i32)
    start[1::2] = T
    kc = torch.zeros(1, Hkv, P, d, dtype=torch.bfloat16, device="cuda")
    table = torch.zeros(Bt, n // P + T // P, **i32)
    err = torch.zeros(1, **i32)
    nbytes = simsd.simsd_chunk_workspace_bytes(simsd.SIMSD_BF16, T, Bt, Hkv, Hkv, d, table.shape[1], P)
    ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    simsd.simsd_chunk_attention(q, start, torch.full((Bt,), n, **i32), kc, kc, table, out, lse=lse, workspace=ws,
                                err_word=err)
    assert simsd.simsd_check_error(err) == simsd.EW_TOKENS
    assert (out == 7).all() and (lse == 7).all()

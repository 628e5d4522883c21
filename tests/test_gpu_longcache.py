"""The calls for long caches together, as a serving loop makes them: windows,
4 bits, pools, forks and compaction, and the same in a CUDA graph."""
import pytest
import torch

from paper_2606_02544_gb300 import simsd
from paper_2606_02544_gb300.prompt import PromptCache, long_context

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
I32 = dict(dtype=torch.int32, device="cuda")
LAYERS, HQ, HKV, D, P = 2, 8, 2, 64, 16


def plan():
    return simsd.simsd_rope_plan_init("half", D, 1.0e6)


def chunk(g, dtype, *n):
    x = torch.randn(LAYERS, sum(n), HQ + 2 * HKV, D, generator=g, device="cuda").to(dtype)
    return x, torch.tensor([sum(n[:i]) for i in range(len(n) + 1)], **I32)


@pytest.mark.parametrize("dtype,bits", [(BF16, None), (BF16, 4), (F32, None), (F32, 4)])
def test_pool_and_place_for_every_row_agree(dtype, bits):
    """Pages that the window has left behind are taken again by other
    sequences; outputs have the bits that a place for every row gives."""
    kw = dict(mask_block=1, dtype=dtype, window=70, sinks=20, bits=bits)
    whole = PromptCache(LAYERS, 3, HQ, HKV, D, P, 1024, plan(), **kw)
    pool = PromptCache(LAYERS, 3, HQ, HKV, D, P, 1024, plan(), pages=37, **kw)
    for i, n in enumerate([(100, 1, 30), (50, 0, 1), (1, 1, 1), (140, 33, 1), (1, 1, 1), (70, 90, 100), (1, 1, 1)]):
        g = torch.Generator(device="cuda").manual_seed(i)
        x, start = chunk(g, dtype, *n)
        a, b = whole.append_chunk(x, start), pool.append_chunk(x, start)
        assert torch.equal(a, b), i
        if i == 4:
            pool.compact()
    assert simsd.simsd_check_error(pool.err) == 0 and simsd.simsd_check_error(whole.err) == 0
    assert int((pool.refs > 0).sum()) <= 3 * (2 + 6)
    assert pool.prefix_len.tolist() == [363, 127, 135]


@pytest.mark.parametrize("dtype,bits", [(BF16, None), (BF16, 4), (F32, 4)])
def test_forks_continue_as_their_source(dtype, bits):
    """A fork that gets the rows its source gets has its outputs, and one that
    gets others does not disturb it."""
    cache = PromptCache(LAYERS, 4, HQ, HKV, D, P, 512, plan(), dtype=dtype, bits=bits, pages=60)
    g = torch.Generator(device="cuda").manual_seed(0)
    cache.append_chunk(*chunk(g, dtype, 75, 0, 40, 0))
    cache.fork(torch.tensor([0, 0], **I32), torch.tensor([1, 3], **I32))
    assert cache.prefix_len.tolist() == [75, 75, 40, 75]
    shared = cache.refs.max().item()
    assert shared == 3  # four whole pages of three sequences
    for step in range(30):
        x, start = chunk(g, dtype, 1, 1, 1, 1)
        x[:, 1] = x[:, 0]
        out = cache.append_chunk(x, start)
        assert torch.equal(out[:, 0], out[:, 1]), step
        assert not torch.equal(out[:, 0], out[:, 3])
    before = cache.append_chunk(*chunk(g, dtype, 0, 0, 0, 0))
    assert before.numel() == 0
    cache.release(torch.tensor([0, 2], **I32))
    live = cache.compact()
    assert int(live) == int((cache.refs > 0).sum()) and int(cache.block_table.max()) == int(live) - 1
    x, start = chunk(g, dtype, 0, 1, 0, 1)
    out = cache.append_chunk(x, start)
    assert bool(torch.isfinite(out.float()).all()) and simsd.simsd_check_error(cache.err) == 0


def test_expanded_cache_is_what_the_codes_stand_for():
    """Attention by codes and attention over the expanded cache are the same
    up to the rounding of the probabilities (2^-9 and 2^-12 of them) and of
    the outputs (2^-8 at most)."""
    cache = PromptCache(LAYERS, 2, HQ, HKV, D, P, 512, plan(), bits=4)
    g = torch.Generator(device="cuda").manual_seed(3)
    cache.append_chunk(*chunk(g, BF16, 200, 77))
    before = cache.prefix_len.clone()
    x, start = chunk(g, BF16, 1, 1)
    out = cache.append_chunk(x, start)
    n = cache.refs.shape[0]
    for l in range(LAYERS):
        kc, vc = (torch.full((n, HKV, P, D), float("nan"), dtype=BF16, device="cuda") for _ in range(2))
        simsd.simsd_q4_expand(cache.q4[l], cache.block_table, torch.zeros_like(before), cache.prefix_len, kc, vc,
                              err_word=cache.err)
        q = torch.empty(2, HQ, D, dtype=BF16, device="cuda")
        simsd.simsd_rope_rotate(plan(), before, x[l][:, :HQ], q)
        o2 = torch.empty_like(q)
        ws = torch.empty(simsd.simsd_chunk_workspace_bytes(simsd.SIMSD_BF16, 2, 2, HQ, HKV, D, cache.max_pages, P),
                         dtype=torch.uint8, device="cuda")
        simsd.simsd_chunk_attention(q, start, before, kc, vc, cache.block_table, o2, workspace=ws)
        top = float(torch.nan_to_num(vc.float()).abs().max())
        err = (out[l].float() - o2.float()).abs()
        # A <= max |v|: 2^-8 (bf16 probabilities) + 2^-11 + scores' errors, and both roundings of the outputs
        assert bool((err <= top * (2.0 ** -8 + 2.0 ** -10) + 2 * 2.0 ** -8 * o2.float().abs()).all())
    assert simsd.simsd_check_error(cache.err) == 0


@pytest.mark.parametrize("bits", [None, 4])
def test_replayed_decoding_step(bits):
    """A step of every sequence captured once, with its pages taken and let go
    of, and replayed on other rows; the bits of calls made one by one."""
    caches = [PromptCache(LAYERS, 3, HQ, HKV, D, P, 512, plan(), window=50, sinks=10, bits=bits, pages=40) for _ in range(2)]
    g = torch.Generator(device="cuda").manual_seed(5)
    x, start = chunk(g, BF16, 61, 5, 100)
    for c in caches:
        c.append_chunk(x, start)
    static, one = chunk(g, BF16, 1, 1, 1)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    state = [t.clone() for t in (caches[1].block_table, caches[1].refs, caches[1].prefix_len)]
    with torch.cuda.stream(s):
        caches[1].append_chunk(static, one)  # warm-up, undone below
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            out = caches[1].append_chunk(static, one)
    torch.cuda.current_stream().wait_stream(s)
    for t, v in zip((caches[1].block_table, caches[1].refs, caches[1].prefix_len), state):
        t.copy_(v)
    for step in range(25):
        x, _ = chunk(g, BF16, 1, 1, 1)
        static.copy_(x)
        want = caches[0].append_chunk(x, one)
        graph.replay()
        assert torch.equal(out, want), step
    for a, b in ((caches[0].block_table, caches[1].block_table), (caches[0].refs, caches[1].refs)):
        assert torch.equal(a, b)
    assert all(simsd.simsd_check_error(c.err) == 0 for c in caches)


def test_verification_refuses_what_it_cannot_read():
    cache = PromptCache(LAYERS, 2, HQ, HKV, D, P, 512, plan(), bits=4)
    with pytest.raises(ValueError):
        cache.verify(*[torch.zeros(1)] * 8)


def test_example_runs():
    assert long_context(simsd.simsd_rope_plan_init("half", 128, 1.0e6))


def test_cache_without_a_pool_refuses_the_pools_calls():
    cache = PromptCache(1, 2, HQ, HKV, D, P, 64, plan())
    one = torch.tensor([1], **I32)
    for call in (lambda: cache.fork(one, one), lambda: cache.release(one), cache.compact):
        with pytest.raises(ValueError):
            call()
    for kw in (dict(bits=8), dict(window=-1), dict(window=4, sinks=-1)):
        with pytest.raises(ValueError):
            PromptCache(1, 2, HQ, HKV, D, P, 64, plan(), **kw)


def test_release_of_a_sequence_out_of_range():
    cache = PromptCache(LAYERS, 2, HQ, HKV, D, P, 64, plan(), pages=8)
    g = torch.Generator(device="cuda").manual_seed(3)
    cache.append_chunk(*chunk(g, BF16, 20, 30))
    cache.release(torch.tensor([1, 5, -1], **I32))
    assert simsd.simsd_check_error(cache.err) == simsd.EW_SEQ
    assert cache.prefix_len.tolist() == [20, 0] and int((cache.refs > 0).sum()) == 2


def test_graph_outlives_a_larger_workspace():
    """A step captured with a small workspace gives the same after a longer
    chunk has made a larger one."""
    x, start = chunk(torch.Generator(device="cuda").manual_seed(4), BF16, 1, 1)
    cache = PromptCache(LAYERS, 2, HQ, HKV, D, P, 2048, plan(), bits=4)
    cache.append_chunk(*chunk(torch.Generator(device="cuda").manual_seed(5), BF16, 300, 400))
    cache.workspace = None
    lens = cache.prefix_len.clone()
    want = cache.append_chunk(x, start)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = cache.append_chunk(x, start)
    small = cache.workspace
    cache.prefix_len.copy_(lens)
    cache.append_chunk(*chunk(torch.Generator(device="cuda").manual_seed(6), BF16, 600, 500))
    assert cache.workspace is not small and any(w is small for w in cache.captured)
    cache.prefix_len.copy_(lens)
    graph.replay()
    assert torch.equal(got, want) and simsd.simsd_check_error(cache.err) == 0


def near(a, b):
    """Rows of calls whose other rows differ (they may be cut elsewhere, or go
    another way): each off by 2^-8 (fp32: 2^-16) of values of 8 at most."""
    return bool(((a.double() - b.double()).abs() <= 16 * 2.0 ** (-8 if a.dtype == BF16 else -16)).all())


@pytest.mark.parametrize("dtype,bits", [(BF16, None), (BF16, 4), (F32, 4)])
def test_a_chunk_without_pages_can_be_made_again(dtype, bits):
    """Too few free pages: sequences that want one stay as they were, with
    outputs of zero, those that want none go on; after a release the same rows
    have the outputs that a larger pool gives."""
    small, large = (PromptCache(LAYERS, 4, HQ, HKV, D, P, 512, plan(), dtype=dtype, bits=bits, pages=n) for n in (12, 60))
    g = torch.Generator(device="cuda").manual_seed(8)
    x, start = chunk(g, dtype, 60, 33, 20, 40)  # 4 + 3 + 2 + 3 pages
    for c in (small, large):
        c.append_chunk(x, start)
    assert simsd.simsd_check_error(small.err) == 0 and int((small.refs == 0).sum()) == 0
    state = [t.clone() for t in (small.block_table, small.refs)]
    parts = [t.clone() for t in small.page_set.tensors]
    x, start = chunk(g, dtype, 2, 30, 1, 20)  # sequences 1 and 3 want pages
    got, want = small.append_chunk(x, start), large.append_chunk(x, start)
    assert simsd.simsd_check_error(small.err) & simsd.EW_POOL
    small.err.zero_()
    assert small.prefix_len.tolist() == [62, 33, 21, 40]
    assert near(got[:, :2], want[:, :2]) and near(got[:, 32:33], want[:, 32:33])
    assert bool((got[:, 2:32] == 0).all()) and bool((got[:, 33:] == 0).all())
    assert torch.equal(small.block_table, state[0]) and torch.equal(small.refs, state[1])
    for b in (1, 3):
        held = state[0][b][state[0][b] >= 0].long()
        # (bytes: rows that nobody has written may hold NaN)
        assert all(torch.equal(t.view(torch.uint8)[:, held], s.view(torch.uint8)[:, held]) for t, s in zip(small.page_set.tensors, parts))
    small.release(torch.tensor([2], **I32))
    again = torch.tensor([0, 0, 30, 30, 30], **I32)  # sequence 1 (2 pages), then 3
    out = small.append_chunk(x[:, 2:32], again)
    assert near(out, want[:, 2:32])
    small.release(torch.tensor([0], **I32))
    out = small.append_chunk(x[:, 33:], torch.tensor([0, 0, 0, 0, 20], **I32))
    assert near(out, want[:, 33:])
    assert simsd.simsd_check_error(small.err) == 0 and small.prefix_len.tolist() == [0, 63, 0, 60]


@pytest.mark.parametrize("bits", [None, 4])
def test_a_sequence_cut_back_into_shared_pages_writes_nothing(bits):
    """A fork cut back into a page that it shares with its source: its rows are
    refused, the source goes on with its own."""
    cache, alone = (PromptCache(LAYERS, 2, HQ, HKV, D, P, 256, plan(), bits=bits, pages=20) for _ in range(2))
    g = torch.Generator(device="cuda").manual_seed(9)
    x, start = chunk(g, BF16, 40, 0)
    for c in (cache, alone):
        c.append_chunk(x, start)
    cache.fork(torch.tensor([0], **I32), torch.tensor([1], **I32))
    cache.prefix_len[1] = 20  # in the second page of three
    x, start = chunk(g, BF16, 1, 1)
    out = cache.append_chunk(x, start)
    want = alone.append_chunk(x[:, :1].contiguous(), torch.tensor([0, 1, 1], **I32))
    assert simsd.simsd_check_error(cache.err) & simsd.EW_SHARED
    assert near(out[:, :1], want) and bool((out[:, 1] == 0).all()) and cache.prefix_len.tolist() == [41, 20]
    cache.err.zero_()
    x, start = chunk(g, BF16, 1, 0)
    assert near(cache.append_chunk(x, start), alone.append_chunk(x, start))
    assert simsd.simsd_check_error(cache.err) == 0

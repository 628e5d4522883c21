"""Rotary positions and the append to the paged cache on the GPU, against the
plain 64-bit form."""
import numpy as np
import pytest
import torch

from paper_2606_02544_gb300 import simsd
from tests import _prompt as ref

pytestmark = pytest.mark.gpu
THETA = 1.0e6


def make(dtype, chunk, prefix, Hq, Hkv, d, P, seed, fused=False, spare=2):
    g = torch.Generator().manual_seed(seed)
    T = sum(chunk)
    start = np.concatenate([[0], np.cumsum(chunk)]).astype(np.int32)
    pages = [(n + c + P - 1) // P for n, c in zip(prefix, chunk)]
    pool = sum(pages) + spare
    perm = torch.randperm(pool, generator=g)
    table = torch.full((len(chunk), max(max(pages), 1)), -1, dtype=torch.int32)
    at = 0
    for b, c in enumerate(pages):
        table[b, :c] = perm[at:at + c]
        at += c
    x = torch.randn(T, Hq + 2 * Hkv, d, generator=g).to(dtype).cuda()
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    if not fused:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    kc = torch.randn(pool, Hkv, P, d, generator=g).to(dtype).cuda()
    vc = torch.randn(pool, Hkv, P, d, generator=g).to(dtype).cuda()
    i32 = dict(dtype=torch.int32, device="cuda")
    return dict(q=q, k=k, v=v, token_start=torch.tensor(start, **i32), prefix_len=torch.tensor(prefix, **i32),
                q_out=torch.full((T, Hq, d), float("nan"), dtype=dtype, device="cuda"), k_cache=kc, v_cache=vc,
                block_table=table.cuda(), err_word=torch.zeros(1, **i32))


def check(a, plan_args, positions=None):
    """One append against the plain form; every cache row that is not a
    destination keeps its bits."""
    kc0, vc0 = a["k_cache"].clone(), a["v_cache"].clone()
    plan = simsd.simsd_rope_plan_init(*plan_args[:3], **plan_args[3])
    simsd.simsd_rope_append(plan, **a, positions=positions)
    assert simsd.simsd_check_error(a["err_word"]) == 0
    layout, rot, theta, kw = plan_args
    freq = ref.frequencies(rot, theta, **kw)
    bf16 = a["q"].dtype == torch.bfloat16
    start, prefix = a["token_start"].tolist(), a["prefix_len"].tolist()
    pos = np.concatenate([np.arange(n, n + start[b + 1] - start[b]) for b, n in enumerate(prefix)] or [[]]).astype(int)
    at = positions.cpu().numpy() if positions is not None else pos
    P = kc0.shape[2]
    seq = np.repeat(np.arange(len(prefix)), np.diff(start))
    page = a["block_table"].cpu().numpy()[seq, pos // P]
    want, size = ref.rotate(a["q"].double().cpu().numpy(), at, layout, rot, freq)
    got = a["q_out"].double().cpu().numpy()
    assert np.all(np.abs(got - want) <= ref.rope_tolerance(want, size, bf16))
    want, size = ref.rotate(a["k"].double().cpu().numpy(), at, layout, rot, freq)
    got = a["k_cache"][torch.as_tensor(page).cuda(), :, torch.as_tensor(pos % P).cuda()].double().cpu().numpy()
    assert np.all(np.abs(got - want) <= ref.rope_tolerance(want, size, bf16))
    vc0[torch.as_tensor(page).cuda(), :, torch.as_tensor(pos % P).cuda()] = a["v"]
    assert torch.equal(a["v_cache"], vc0)
    kc0[torch.as_tensor(page).cuda(), :, torch.as_tensor(pos % P).cuda()] = \
        a["k_cache"][torch.as_tensor(page).cuda(), :, torch.as_tensor(pos % P).cuda()]
    assert torch.equal(a["k_cache"], kc0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rot", [2, 6, 8, 24, 48, 64])
def test_layouts_and_partial_heads(dtype, layout, rot):
    check(make(dtype, [5, 1, 9], [0, 30, 15], 4, 2, 64, 16, rot), (layout, rot, THETA, {}))


@pytest.mark.parametrize("scaling", ["linear", "ntk", "yarn"])
@pytest.mark.parametrize("fused", [False, True])
def test_scaled_and_strided(scaling, fused):
    kw = dict(scaling=scaling, factor=8.0, context=4096)
    check(make(torch.bfloat16, [70, 130], [9000, 0], 8, 2, 128, 64, 3, fused), ("half", 128, THETA, kw))


@pytest.mark.parametrize("chunk,prefix", [([1], [0]), ([1] * 40, list(range(40))), ([0, 3, 0, 0, 2], [5, 0, 7, 1, 15]),
                                          ([700, 1, 333], [100, 64, 0])])
def test_chunk_lengths(chunk, prefix):
    check(make(torch.bfloat16, chunk, prefix, 6, 3, 64, 16, 7), ("half", 64, THETA, {}))


@pytest.mark.parametrize("d,Hq,Hkv", [(8, 3, 1), (40, 5, 5), (128, 40, 8), (256, 2, 1)])
def test_head_sizes(d, Hq, Hkv):
    check(make(torch.float32, [9, 4], [3, 17], Hq, Hkv, d, 8, d), ("interleaved", min(d, 128), THETA, {}))


def test_given_positions_far_and_negative():
    a = make(torch.float32, [6], [10], 2, 2, 64, 16, 11)
    pos = torch.tensor([0, -5, 1 << 20, (1 << 30) + 7, -(1 << 29), 123456789], dtype=torch.int32, device="cuda")
    check(a, ("half", 64, 1.0e4, {}), positions=pos)


def test_rotate_in_place_and_strided():
    g = torch.Generator().manual_seed(1)
    x = torch.randn(37, 6, 128, generator=g).cuda()
    pos = torch.randint(0, 5000, (37,), generator=g, dtype=torch.int32).cuda()
    plan = simsd.simsd_rope_plan_init("interleaved", 32, THETA)
    f = ref.frequencies(32, THETA)
    wq, sq = ref.rotate(x[:, :4].double().cpu().numpy(), pos.cpu().numpy(), "interleaved", 32, f)
    wk, sk = ref.rotate(x[:, 4:].double().cpu().numpy(), pos.cpu().numpy(), "interleaved", 32, f)
    qo = torch.full((37, 4, 128), float("nan"), device="cuda")
    ko = torch.full((37, 2, 128), float("nan"), device="cuda")
    simsd.simsd_rope_rotate(plan, pos, x[:, :4], qo, x[:, 4:], ko)
    assert np.all(np.abs(qo.double().cpu().numpy() - wq) <= ref.rope_tolerance(wq, sq, False))
    assert np.all(np.abs(ko.double().cpu().numpy() - wk) <= ref.rope_tolerance(wk, sk, False))
    y = x.clone()
    simsd.simsd_rope_rotate(plan, pos, y[:, :4], y[:, :4], y[:, 4:], y[:, 4:])  # in place, on strided views
    assert torch.equal(y[:, :4], qo) and torch.equal(y[:, 4:], ko)
    z = x.clone()
    simsd.simsd_rope_rotate(plan, pos, z[:, :4], z[:, :4])  # q alone
    assert torch.equal(z[:, :4], qo) and torch.equal(z[:, 4:], x[:, 4:])


def test_rotation_matches_the_verification_kernels():
    """Rotating q and the new keys first (rope_pos None) and letting the
    verification rotate them give the same attention: one rotation, two
    kernels (fp32; each is within 1e-5 of the oracle)."""
    from paper_2606_02544_gb300 import inputs
    from tests import _gpu
    w = inputs.Workload("t", "f32", 2, 4, 2, 64, 4, (30, 90), 1, 64, 0.5, 1 / 8.0, 1.0, 3)
    si = inputs.make_step_inputs(w, device="cuda", with_logits=False)
    mask = _gpu.gpu_mask(si)
    rope = mask[2]
    want, e0, _ = _gpu.gpu_attention(si, mask=mask, rope_pos=rope, rope_theta=THETA)
    plan = simsd.simsd_rope_plan_init("half", 64, THETA)
    q, k = si.q[0].view(-1, 4, 64), si.k_new[0].view(-1, 2, 64)
    simsd.simsd_rope_rotate(plan, rope.view(-1), q, q, k, k)
    got, e1, _ = _gpu.gpu_attention(si, mask=mask)
    assert e0 == e1 == 0
    assert (got - want).abs().max().item() <= 2e-5


def test_bad_prefix_pages_and_offsets():
    a = make(torch.bfloat16, [3, 4, 5], [0, 20, 8], 4, 2, 64, 16, 5)
    a["prefix_len"][1] = -1                      # bad prefix: zero rows, nothing cached
    a["block_table"][2, 0] = a["k_cache"].shape[0]  # rows 8..12 of sequence 2 lie in its page 0
    kc0, vc0 = a["k_cache"].clone(), a["v_cache"].clone()
    plan = simsd.simsd_rope_plan_init("half", 64, THETA)
    simsd.simsd_rope_append(plan, **a)
    assert simsd.simsd_check_error(a["err_word"]) == simsd.EW_PREFIX_LEN | simsd.EW_PAGE
    assert torch.isfinite(a["q_out"].float()).all()
    assert (a["q_out"][3:7] == 0).all() and (a["q_out"][7:] != 0).any()
    page = int(a["block_table"][0, 0])
    other = torch.ones(kc0.shape[0], dtype=torch.bool)
    other[page] = False
    assert torch.equal(a["k_cache"][other.cuda()], kc0[other.cuda()])
    assert torch.equal(a["v_cache"][other.cuda()], vc0[other.cuda()])
    # no room for the chunk in the block table
    b = make(torch.bfloat16, [3], [0], 4, 2, 64, 16, 5)
    b["prefix_len"][0] = 14
    simsd.simsd_rope_append(plan, **b)
    assert simsd.simsd_check_error(b["err_word"]) == simsd.EW_PREFIX_LEN
    assert (b["q_out"] == 0).all()
    # offsets out of order or range: those chunks are empty, their tokens untouched
    c = make(torch.bfloat16, [3, 4, 5], [0, 20, 8], 4, 2, 64, 16, 5)
    c["token_start"][:] = torch.tensor([0, 3, 2, 99])
    simsd.simsd_rope_append(plan, **c)
    assert simsd.simsd_check_error(c["err_word"]) == simsd.EW_TOKENS
    assert torch.isfinite(c["q_out"][:2].float()).all() and torch.isnan(c["q_out"][3:].float()).all()


def test_tokens_outside_every_chunk_are_untouched():
    a = make(torch.float32, [4, 4], [0, 0], 2, 2, 64, 16, 9)
    a["token_start"][:] = torch.tensor([2, 4, 7])
    plan = simsd.simsd_rope_plan_init("half", 64, THETA)
    simsd.simsd_rope_append(plan, **a)
    assert simsd.simsd_check_error(a["err_word"]) == 0
    bad = torch.isnan(a["q_out"]).flatten(1)
    assert bad[[0, 1, 7]].all() and not bad[2:7].any()


def test_on_a_stream_of_its_own():
    a = make(torch.bfloat16, [40], [100], 8, 2, 128, 64, 13)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    plan = simsd.simsd_rope_plan_init("half", 128, THETA)
    simsd.simsd_rope_append(plan, **a, stream=s)
    s.synchronize()
    first = a["q_out"].clone()
    simsd.simsd_rope_append(plan, **a)
    assert torch.equal(first, a["q_out"])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("layout,rot,d", [("half", 128, 128), ("interleaved", 128, 128), ("half", 24, 64), ("interleaved", 6, 64)])
def test_rotate_against_the_plain_form(dtype, layout, rot, d):
    """The rows of a verification step (many tokens, scaled frequencies) and a
    single one; the type's own vectors and rounding."""
    g = torch.Generator().manual_seed(2)
    kw = dict(scaling="yarn", factor=4.0, context=8192)
    plan, f = simsd.simsd_rope_plan_init(layout, rot, THETA, **kw), ref.frequencies(rot, THETA, **kw)
    for T in (1, 1025):
        x = torch.randn(T, 10, d, generator=g).to(dtype).cuda()
        pos = torch.randint(0, 40000, (T,), generator=g, dtype=torch.int32).cuda()
        qo, ko = torch.full_like(x[:, :8], float("nan")), torch.full_like(x[:, 8:], float("nan"))
        simsd.simsd_rope_rotate(plan, pos, x[:, :8], qo, x[:, 8:], ko)
        want, size = ref.rotate(x.double().cpu().numpy(), pos.cpu().numpy(), layout, rot, f)
        got = torch.cat([qo, ko], 1).double().cpu().numpy()
        assert np.all(np.abs(got - want) <= ref.rope_tolerance(want, size, dtype == torch.bfloat16))

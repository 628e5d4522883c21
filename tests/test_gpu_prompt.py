"""The prompt path as a whole: chunks into the cache, drafts with their
distribution, a verified block."""
import numpy as np
import pytest
import torch

from paper_2606_02544_gb300 import prompt, simsd
from tests import _prompt as ref

pytestmark = pytest.mark.gpu


def test_command_runs(capsys):
    assert prompt.main() == 0
    assert "error word 0" in capsys.readouterr().out


def _fill(sizes, dtype, seed=3):
    plan = simsd.simsd_rope_plan_init("interleaved", 64, 1.0e6, "yarn", factor=4.0, context=256)
    c = prompt.PromptCache(2, 2, 4, 2, 64, 16, 400, plan, mask_block=8, dtype=dtype)
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(2, 2, 300, 8, 64, generator=g) * 0.5).to(dtype).cuda()  # [layer][sequence][token]
    outs, done = [], 0
    for n in sizes:
        qkv = torch.cat([x[:, 0, done:done + n], x[:, 1, done:done + n]], 1)
        start = torch.tensor([0, n, 2 * n], dtype=torch.int32, device="cuda")
        o = c.append_chunk(qkv, start)
        outs.append(o.view(2, 2, n, 4, 64))
        done += n
    assert simsd.simsd_check_error(c.err) == 0
    return c, torch.cat(outs, 2)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_chunking_does_not_change_the_cache(dtype):
    """One chunk or many: the cached rows are the same bits, the attention
    outputs agree within the rounding of both."""
    a, oa = _fill([300], dtype)
    b, ob = _fill([8, 120, 1, 7, 164], dtype)
    assert a.prefix_len.tolist() == b.prefix_len.tolist() == [300, 300]
    rows = torch.arange(300)
    for s in range(2):
        page = a.block_table[s][rows.cuda() // 16].long()
        for x, y in ((a.k_cache, b.k_cache), (a.v_cache, b.v_cache)):
            assert torch.equal(x[:, page, :, rows.cuda() % 16], y[:, page, :, rows.cuda() % 16])
    # mask_block 8 with chunk ends inside a block: a token then misses the
    # rest of its block, so compare blocks that lie inside one chunk of both
    inside = [t for t in range(300) if (t // 8 * 8 + 8 <= 8) or (8 <= t // 8 * 8 and t // 8 * 8 + 8 <= 128)
              or (136 <= t // 8 * 8)]
    # rounding of P and O to bf16 on both sides: 4 u (A + |r|), |v| <= 3; fp32: 2^-15
    tol = 4 * 2.0 ** -8 * 3 if dtype == torch.bfloat16 else 2.0 ** -15
    assert (oa[:, :, inside].double() - ob[:, :, inside].double()).abs().max().item() <= tol


def test_drafts_from_a_truncated_distribution_keep_the_target():
    """Draft and target logits both truncated by simsd_sample: the emitted
    first token follows the target's truncated distribution (Eq. (2) with
    residual resampling), and no token outside it ever comes out."""
    g = torch.Generator().manual_seed(5)
    Bt, V, gamma = 20000, 24, 1
    t1, d1 = torch.randn(V, generator=g) * 1.5, torch.randn(V, generator=g) * 1.5
    plan = simsd.simsd_rope_plan_init("half", 64, 1.0e4)
    c = prompt.PromptCache(1, 1, 1, 1, 64, 16, 16, plan)
    f = lambda v, n: torch.full((n,), v, device="cuda")  # noqa: E731
    k = lambda v, n: torch.full((n,), v, dtype=torch.int32, device="cuda")  # noqa: E731
    draft, dlp = c.draw(d1.cuda().expand(Bt, gamma, V).contiguous(), torch.rand(Bt, gamma, generator=g).cuda(),
                        top_k=k(9, Bt), top_p=f(0.9, Bt))
    n = Bt * (gamma + 1)
    _, tlp = c.draw(t1.cuda().expand(Bt, gamma + 1, V).contiguous(), torch.rand(Bt, gamma + 1, generator=g).cuda(),
                    top_k=k(12, n), top_p=f(0.8, n))
    a = torch.empty(Bt, dtype=torch.int32, device="cuda")
    ot = torch.empty(Bt, gamma + 1, dtype=torch.int32, device="cuda")
    simsd.simsd_accept_sampled(tlp, dlp, draft, torch.rand(Bt, gamma, generator=g).cuda(),
                               torch.rand(Bt, generator=g).cuda(), a, ot, err_word=c.err)
    assert simsd.simsd_check_error(c.err) == 0
    _, idx, lp = ref.sample_row(t1.double().numpy(), 0.5, k=12, p=0.8)
    want = np.zeros(V)
    want[idx] = np.exp(lp)
    got = np.bincount(ot[:, 0].cpu().numpy(), minlength=V) / Bt
    assert (got[want == 0] == 0).all()
    # five standard deviations of a share
    assert np.all(np.abs(got - want) <= 5 * np.sqrt(want * (1 - want) / Bt) + 1e-12)


def test_one_tensor_off_the_gpu_is_refused():
    """Any tensor of a call left in host memory, and an error word of another
    type: refused before anything is launched."""
    T, Hq, Hkv, d, P = 4, 4, 2, 64, 16
    z = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    i = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    plan = simsd.simsd_rope_plan_init("half", 64, 1e4)
    calls = [
        (lambda **a: simsd.simsd_rope_rotate(plan, **a), dict(positions=i(T), q=z(T, Hq, d), q_out=z(T, Hq, d),
                                                              k=z(T, Hkv, d), k_out=z(T, Hkv, d))),
        (lambda **a: simsd.simsd_rope_append(plan, **a),
         dict(q=z(T, Hq, d), k=z(T, Hkv, d), v=z(T, Hkv, d), token_start=i(3), prefix_len=i(2), positions=i(T),
              q_out=z(T, Hq, d), k_cache=z(5, Hkv, P, d), v_cache=z(5, Hkv, P, d), block_table=i(2, 3), err_word=i(1))),
        (simsd.simsd_chunk_attention,
         dict(q=z(T, Hq, d), token_start=i(3), prefix_len=i(2), k_cache=z(5, Hkv, P, d), v_cache=z(5, Hkv, P, d),
              block_table=i(2, 3), out=z(T, Hq, d), lse=z(T, Hq), key_start=i(2), err_word=i(1),
              workspace=torch.zeros(1 << 20, dtype=torch.uint8, device="cuda"))),
        (simsd.simsd_sample,
         dict(logits=z(3, 7), u=z(3), token=i(3), temperature=z(3), top_k=i(3), top_p=z(3), min_p=z(3), kept=i(3),
              log_prob=z(3), log_probs=z(3, 7), err_word=i(1)))]
    for call, args in calls:
        call(**args)
        for name, t in args.items():
            with pytest.raises(ValueError):
                call(**{**args, name: t.cpu()})
        if "err_word" in args:
            with pytest.raises(ValueError):
                call(**{**args, "err_word": args["err_word"].to(torch.uint8)})
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_calls_in_a_cuda_graph(dtype):
    """Rotation, append, attention and sampling captured once and replayed on
    other inputs (lengths and offsets too): the bits of the calls made one by
    one.  Long enough a cache that the attention merges pieces."""
    T, Bt, Hq, Hkv, d, P, V, pages = 70, 3, 8, 2, 64, 64, 9001, 40
    code = simsd.SIMSD_F32 if dtype == torch.float32 else simsd.SIMSD_BF16
    plan = simsd.simsd_rope_plan_init("half", 64, 1.0e6, "linear", factor=2.0)
    i32 = dict(dtype=torch.int32, device="cuda")
    g = torch.Generator().manual_seed(8)
    table = torch.randperm(Bt * pages, generator=g).to(torch.int32).view(Bt, pages).cuda()
    nbytes = simsd.simsd_chunk_workspace_bytes(code, T, Bt, Hq, Hkv, d, pages, P)
    ws = torch.empty(max(16, nbytes), dtype=torch.uint8, device="cuda")
    qkv = torch.zeros(T, Hq + 2 * Hkv, d, dtype=dtype, device="cuda")
    start, n, pos = torch.zeros(Bt + 1, **i32), torch.zeros(Bt, **i32), torch.zeros(T, **i32)
    logits, u = torch.zeros(T, V, dtype=dtype, device="cuda"), torch.zeros(T, device="cuda")
    k0 = (torch.randn(Bt * pages, Hkv, P, d, generator=g) * 0.5).to(dtype).cuda()
    kc, vc = k0.clone(), k0.flip(0).contiguous()
    q, turned, out = (torch.zeros(T, Hq, d, dtype=dtype, device="cuda") for _ in range(3))
    lse, lps = torch.zeros(T, Hq, device="cuda"), torch.zeros(T, V, device="cuda")
    token, err = torch.zeros(T, **i32), torch.zeros(1, **i32)
    top_k = torch.full((T,), 300, **i32)

    def step():
        simsd.simsd_rope_append(plan, qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:], start, n, q, kc, vc, table,
                                err_word=err)
        simsd.simsd_chunk_attention(q, start, n, kc, vc, table, out, lse=lse, workspace=ws, err_word=err)
        simsd.simsd_rope_rotate(plan, pos, out, turned)
        simsd.simsd_sample(logits, u, token, top_k=top_k, log_probs=lps, err_word=err)

    def fill(seed, lengths, prefix):
        gg = torch.Generator().manual_seed(seed)
        for t, std in ((qkv, 1.0), (logits, 3.0)):
            t.copy_((torch.randn(t.shape, generator=gg) * std).to(dtype))
        u.copy_(torch.rand(T, generator=gg))
        pos.copy_(torch.randint(0, 9999, (T,), generator=gg, dtype=torch.int32))
        start.copy_(torch.tensor([0, lengths[0], lengths[0] + lengths[1], T], dtype=torch.int32))
        n.copy_(torch.tensor(prefix, dtype=torch.int32))
        kc.copy_(k0)
        for t in (q, turned, out, lse, lps, token):
            t.zero_()

    results = lambda: [t.clone() for t in (q, kc, out, lse, turned, token, lps)]  # noqa: E731
    fill(0, [1, 1], [2000, 0, 5])
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed, lengths, prefix in ((1, [1, 60], [2400, 7]), (2, [40, 0], [100, 2490]), (3, [1, 1], [0, 2000])):
        prefix = prefix + [1234]
        fill(seed, lengths, prefix)
        step()
        want = results()
        fill(seed, lengths, prefix)
        graph.replay()
        for a, b in zip(want, results()):
            assert torch.equal(a, b)
    assert simsd.simsd_check_error(err) == 0

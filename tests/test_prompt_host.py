"""Host side of the prompt calls, without a GPU: rotary plans against the
formulas, refusals of the C ABI before any CUDA work, and the binding's
checks of shapes and types."""
import ctypes
import math

import numpy as np
import pytest
import torch

from tests import _prompt as ref


@pytest.fixture(scope="module")
def simsd():
    from paper_2606_02544_gb300 import build, simsd
    build.build()
    simsd.load_library()
    return simsd


@pytest.mark.parametrize("rot", [2, 24, 64, 128])
@pytest.mark.parametrize("scaling", ["none", "linear", "ntk", "yarn"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_plan_frequencies(simsd, rot, scaling, layout):
    if scaling == "ntk" and rot == 2:
        pytest.skip("NTK scaling needs more than one pair")
    plan = simsd.simsd_rope_plan_init(layout, rot, 1.0e6, scaling, factor=4.0, context=8192)
    f, mag = ref.frequencies(rot, 1.0e6, scaling, 4.0, 8192)
    assert plan.rot_dim == rot and plan.layout == (layout == "interleaved")
    assert plan.magnitude == pytest.approx(mag, rel=1e-7)
    turns = np.array([plan.turn[i] for i in range(rot // 2)], dtype=np.float64)
    want = f / (2 * math.pi) * 2.0 ** 64
    # one unit of the plan's fixed point, and doubles on both sides: each power
    # is off by the rounding of its exponent times ln theta' (at most ln 1.6e7
    # = 17 units of 2^-53) and the few operations around it
    assert np.all(np.abs(turns - want) <= 1 + 2 * (17 + 4) * 2.0 ** -53 * want)
    assert all(plan.turn[i] == 0 for i in range(rot // 2, 64))


def test_plan_refusals(simsd):
    ok = dict(layout="half", rot_dim=64, theta=1e4)
    simsd.simsd_rope_plan_init(**ok)
    for bad in (dict(rot_dim=0), dict(rot_dim=63), dict(rot_dim=130), dict(theta=0.0), dict(theta=-1.0),
                dict(theta=float("inf")), dict(theta=float("nan")), dict(scaling="linear", factor=0.5),
                dict(scaling="linear", factor=float("nan")), dict(scaling="ntk", factor=2.0, rot_dim=2),
                dict(scaling="yarn", factor=2.0, context=0),
                dict(scaling="yarn", factor=2.0, context=100, beta_fast=1.0, beta_slow=1.0),
                dict(scaling="yarn", factor=2.0, context=100, beta_slow=-1.0)):
        with pytest.raises(simsd.SimsdError) as e:
            simsd.simsd_rope_plan_init(**{**ok, **bad})
        assert e.value.status == simsd.SIMSD_ERR_INVALID_ARG
    for bad in (dict(layout="quarter"), dict(scaling="cubic")):
        with pytest.raises(ValueError):
            simsd.simsd_rope_plan_init(**{**ok, **bad})
    assert simsd.load_library().simsd_rope_plan_init(None, 0, 64, 1e4, 0, 1.0, 0, 32.0, 1.0) == 1


def test_c_refusals_before_any_cuda_work(simsd):
    lib = simsd.load_library()
    one, odd = ctypes.c_void_p(16), ctypes.c_void_p(24)
    plan = simsd.simsd_rope_plan_init("half", 64, 1e4)
    pl = ctypes.addressof(plan)

    def append(dtype=1, plan=pl, q=one, qs=512, k=one, ks=128, v=one, vs=128, ts=one, n=one, T=4, Bt=2, Hq=8, Hkv=2,
               d=64, qo=one, kc=one, vc=one, pages=9, bt=one, mp=3, P=16):
        return lib.simsd_rope_append(dtype, plan, q, qs, k, ks, v, vs, ts, n, None, T, Bt, Hq, Hkv, d, qo, kc, vc,
                                     pages, bt, mp, P, None, None)

    assert append(dtype=7) == 2
    for bad in (dict(plan=None), dict(q=None), dict(k=None), dict(v=None), dict(ts=None), dict(n=None), dict(bt=None),
                dict(kc=None), dict(vc=None), dict(qo=None), dict(q=odd), dict(qo=odd), dict(kc=odd), dict(qs=511),
                dict(ks=100), dict(qs=516), dict(d=32), dict(d=63), dict(T=-1), dict(Bt=-1), dict(Hq=0), dict(Hkv=0),
                dict(P=0), dict(mp=-1)):
        assert append(**bad) == 1, bad
    assert append(T=0) == 0 and append(Bt=0) == 0
    broken = simsd.RopePlan.from_buffer_copy(plan)
    broken.reserved = 1
    assert append(plan=ctypes.addressof(broken)) == 1
    broken = simsd.RopePlan.from_buffer_copy(plan)
    broken.magnitude = float("nan")
    assert append(plan=ctypes.addressof(broken)) == 1

    def rotate(dtype=1, pos=one, q=one, qs=512, qo=one, qos=512, Hq=8, k=one, ks=128, ko=one, kos=128, Hkv=2, T=4,
               d=64):
        return lib.simsd_rope_rotate(dtype, pl, pos, q, qs, qo, qos, Hq, k, ks, ko, kos, Hkv, T, d, None)

    for bad in (dict(pos=None), dict(q=None), dict(qo=odd), dict(qos=100), dict(k=None), dict(ko=None), dict(Hkv=0),
                dict(Hq=0), dict(T=-1), dict(d=60)):
        assert rotate(**bad) == 1, bad
    assert rotate(dtype=5) == 2 and rotate(T=0) == 0

    def attend(dtype=1, q=one, qs=512, ts=one, n=one, kc=one, vc=one, pages=9, bt=one, mp=3, P=16, T=4, Bt=2, Hq=8,
               Hkv=2, d=64, block=1, window=0, scale=0.0, out=one, ws=None, wsb=0):
        return lib.simsd_chunk_attention(dtype, q, qs, ts, n, None, kc, vc, pages, bt, mp, P, T, Bt, Hq, Hkv, d,
                                         block, window, scale, out, None, ws, wsb, None, None)

    for bad in (dict(q=None), dict(ts=None), dict(n=None), dict(kc=None), dict(vc=None), dict(bt=None), dict(out=None),
                dict(q=odd), dict(out=odd), dict(qs=100), dict(Hq=7), dict(Hkv=0), dict(block=-1), dict(window=-1),
                dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(T=-1), dict(pages=0),
                dict(mp=0)):
        assert attend(**bad) == 1, bad
    for bad in (dict(dtype=9), dict(P=12), dict(P=4), dict(d=96), dict(mp=1 << 27, P=64)):
        assert attend(**bad) == 2, bad
    assert attend(T=0) == 0 and attend(Bt=0) == 0

    def sample(dtype=0, x=one, stride=100, R=2, V=100, u=one, token=one, probs=None):
        return lib.simsd_sample(dtype, x, stride, R, V, u, None, None, None, None, token, None, None, probs, None,
                                None)

    for bad in (dict(x=None), dict(u=None), dict(token=None), dict(x=odd), dict(probs=odd), dict(stride=99), dict(V=0),
                dict(V=(1 << 24) + 1, stride=1 << 25), dict(R=-1)):
        assert sample(**bad) == 1, bad
    assert sample(dtype=3) == 2 and sample(R=0) == 0


def test_binding_refusals(simsd):
    """Wrong shapes, types and layouts raise before the library is called."""
    T, Hq, Hkv, d, P = 4, 4, 2, 64, 16
    q = torch.zeros(T, Hq, d)
    k = torch.zeros(T, Hkv, d)
    kc = torch.zeros(5, Hkv, P, d)
    bt = torch.zeros(2, 3, dtype=torch.int32)
    ts = torch.zeros(3, dtype=torch.int32)
    n = torch.zeros(2, dtype=torch.int32)
    plan = simsd.simsd_rope_plan_init("half", 64, 1e4)
    good = dict(q=q, k=k, v=k, token_start=ts, prefix_len=n, q_out=q, k_cache=kc, v_cache=kc, block_table=bt)
    for bad in (dict(k=k.double()), dict(v=k[:, :1]), dict(q_out=q.bfloat16()), dict(q_out=q[:3]),
                dict(token_start=ts[:2]), dict(token_start=ts.long()), dict(k_cache=kc.transpose(0, 1)),
                dict(v_cache=kc[:4]), dict(block_table=bt.long()), dict(block_table=bt.t()),
                dict(positions=torch.zeros(3, dtype=torch.int32)), dict(q=q.transpose(1, 2).contiguous().transpose(1, 2))):
        with pytest.raises((ValueError, TypeError)):
            simsd.simsd_rope_append(plan, **{**good, **bad})
    good = dict(q=q, token_start=ts, prefix_len=n, k_cache=kc, v_cache=kc, block_table=bt, out=q)
    for bad in (dict(out=q[:2]), dict(lse=torch.zeros(T, Hq, dtype=torch.float64)), dict(lse=torch.zeros(T, Hq + 1)),
                dict(key_start=n.long()), dict(key_start=ts), dict(prefix_len=n.float()), dict(k_cache=kc.bfloat16())):
        with pytest.raises((ValueError, TypeError)):
            simsd.simsd_chunk_attention(**{**good, **bad})
    x, u, tok = torch.zeros(3, 7), torch.zeros(3), torch.zeros(3, dtype=torch.int32)
    good = dict(logits=x, u=u, token=tok)
    for bad in (dict(u=u.double()), dict(u=u[:2]), dict(token=tok.long()), dict(top_k=u), dict(top_p=tok),
                dict(log_probs=torch.zeros(3, 8)), dict(logits=x.t()), dict(logits=x.half())):
        with pytest.raises((ValueError, TypeError)):
            simsd.simsd_sample(**{**good, **bad})
    with pytest.raises(ValueError):
        simsd.simsd_rope_rotate(plan, tok, q, q)
    with pytest.raises(ValueError):
        simsd.simsd_rope_rotate(plan, torch.zeros(T, dtype=torch.int32), q, q, k=k)


def test_reference_attention_gradients_of_lse():
    """The plain form against differences: d lse / d (scale q.k_j) is the
    probability with which row j enters the output."""
    r = np.random.default_rng(0)
    q, k, v = r.normal(size=(1, 1, 8)), r.normal(size=(5, 1, 8)), r.normal(size=(5, 1, 8))
    out, lse, _ = ref.attention(q, k, v, 4, 1, 0.3)
    p = np.array([(ref.attention(q, np.where(np.arange(5)[:, None, None] == j, k + 1e-6 * q, k), v, 4, 1, 0.3)[1] - lse)
                  [0, 0] / (1e-6 * 0.3 * (q ** 2).sum()) for j in range(5)])
    assert p.sum() == pytest.approx(1, abs=1e-5)
    assert np.allclose(p @ v[:, 0], out[0, 0], atol=1e-5)


def test_reference_sampling_shares():
    """The plain form over a grid of random numbers draws each kept token in
    its share."""
    x = np.array([0.0, 2.0, 1.0, 2.0, -np.inf, 0.5])
    n = 20000
    got = np.bincount([ref.sample_row(x, (i + 0.5) / n, T=0.7, k=4, p=0.95)[0] for i in range(n)], minlength=6) / n
    tok, idx, lp = ref.sample_row(x, 0.5, T=0.7, k=4, p=0.95)
    want = np.zeros(6)
    want[idx] = np.exp(lp)
    assert np.allclose(got, want, atol=2.0 / n)
    assert list(idx) == [1, 3, 2]  # the tie goes to the lower index; top_p ends before 0.5


def test_append_refuses_rows_past_32_bits(simsd):
    """A sequence whose block table reaches past 2^31 rows: its row numbers
    are 32-bit on the device.  (Refused before any CUDA work: with T = 0 a
    call that is not refused returns at once.)"""
    lib = simsd.load_library()
    plan = simsd.simsd_rope_plan_init("half", 64, 1e4)
    one = ctypes.c_void_p(16)

    def append(max_pages, page_size):
        return lib.simsd_rope_append(1, ctypes.addressof(plan), one, 512, one, 128, one, 128, one, one, None, 0, 2, 8, 2,
                                     64, one, one, one, 9, one, max_pages, page_size, None, None)

    for max_pages, page_size in ((1 << 25, 64), (1 << 27, 64), ((1 << 31) - 1, (1 << 31) - 1), (1 << 21, 1024)):
        assert append(max_pages, page_size) == simsd.SIMSD_ERR_UNSUPPORTED
    assert append((1 << 25) - 4, 64) == 0 and append(1, 0x7fffff00) == 0


def test_rope_refuses_token_numbers_past_32_bits(simsd):
    """A block of tokens at the end of 2^31 - 1 would pass 32 bits."""
    lib = simsd.load_library()
    plan = simsd.simsd_rope_plan_init("half", 64, 1e4)
    one, pl = ctypes.c_void_p(16), ctypes.addressof(plan)
    for T in (0x7fffff01, 0x7fffffff):
        assert lib.simsd_rope_rotate(1, pl, one, one, 64, one, 64, 1, None, 0, None, 0, 0, T, 64,
                                     None) == simsd.SIMSD_ERR_UNSUPPORTED
        assert lib.simsd_rope_append(1, pl, one, 64, one, 64, one, 64, one, one, None, T, 1, 1, 1, 64, one, one, one, 9,
                                     one, 9, 16, None, None) == simsd.SIMSD_ERR_UNSUPPORTED


def test_tensors_off_the_gpu_are_refused(simsd):
    """Pointers to host memory never reach the library."""
    T, Hq, Hkv, d, P = 4, 4, 2, 64, 16
    q, k, kc = torch.zeros(T, Hq, d), torch.zeros(T, Hkv, d), torch.zeros(5, Hkv, P, d)
    i32 = dict(dtype=torch.int32)
    ts, n, bt, pos = torch.zeros(3, **i32), torch.zeros(2, **i32), torch.zeros(2, 3, **i32), torch.zeros(T, **i32)
    plan = simsd.simsd_rope_plan_init("half", 64, 1e4)
    with pytest.raises(ValueError, match="CUDA device"):
        simsd.simsd_rope_rotate(plan, pos, q, q, k, k)
    with pytest.raises(ValueError, match="CUDA device"):
        simsd.simsd_rope_append(plan, q, k, k, ts, n, q, kc, kc, bt)
    with pytest.raises(ValueError, match="CUDA device"):
        simsd.simsd_chunk_attention(q, ts, n, kc, kc, bt, q)
    with pytest.raises(ValueError, match="CUDA device"):
        simsd.simsd_sample(torch.zeros(3, 7), torch.zeros(3), torch.zeros(3, **i32))

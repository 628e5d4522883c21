"""Refusals of the calls for long caches, without a GPU: argument errors are
found on the host before anything is launched, and the Python binding looks
at shapes, types and devices."""
import ctypes

import pytest
import torch

from paper_2606_02544_gb300 import build, simsd
from tests import _longcache as ref

BAD, UNSUPPORTED = simsd.SIMSD_ERR_INVALID_ARG, simsd.SIMSD_ERR_UNSUPPORTED
one = ctypes.c_void_p(256)
odd = ctypes.c_void_p(260)
F = ctypes.c_float


@pytest.fixture(scope="module")
def lib():
    build.build()
    return simsd.load_library()


def q4(**kw):
    v = dict(k_codes=256, k_scales=256, v_codes=256, v_scales=256, k_unit=1.0, v_unit=1.0) | kw
    c = simsd._Q4Cache(*v.values())
    return ctypes.byref(c), c


def test_numbers_of_the_plain_form():
    assert ref.SCALES[126] == 448 and ref.SCALES[1] == 2.0 ** -9 and ref.SCALES[8] == 2.0 ** -6
    assert (ref.SCALES[1:] > ref.SCALES[:-1]).all()


@pytest.mark.parametrize("change,status", [
    (dict(dtype=2), UNSUPPORTED), (dict(T=-1), BAD), (dict(Hkv=3), BAD), (dict(d=96), UNSUPPORTED),
    (dict(P=24), UNSUPPORTED), (dict(P=4), UNSUPPORTED), (dict(block=-1), BAD), (dict(window=-1), BAD),
    (dict(sinks=-1), BAD), (dict(scale=-1.0), BAD), (dict(scale=float("nan")), BAD), (dict(q=None), BAD),
    (dict(q=odd), BAD), (dict(qs=8 * 128 - 8), BAD), (dict(qs=8 * 128 + 1), BAD), (dict(start=None), BAD),
    (dict(out=odd), BAD), (dict(out=None), BAD), (dict(table=None), BAD), (dict(pages=0), BAD),
    (dict(max_pages=1 << 26), UNSUPPORTED), (dict(T=1 << 28, Hq=8), UNSUPPORTED)])
@pytest.mark.parametrize("four", [False, True])
def test_attention_refusals(lib, four, change, status):
    a = dict(dtype=1, q=one, qs=8 * 128, start=one, prefix=one, pages=4, table=one, max_pages=4, P=64, T=3, Bt=2,
             Hq=8, Hkv=2, d=128, block=1, window=0, sinks=0, scale=0.0, out=one) | change
    tail = (a["pages"], a["table"], a["max_pages"], a["P"], a["T"], a["Bt"], a["Hq"], a["Hkv"], a["d"], a["block"],
            a["window"], a["sinks"], F(a["scale"]), a["out"], None, one, 1 << 20, None, None)
    head = (a["dtype"], a["q"], a["qs"], a["start"], a["prefix"], None)
    if four:
        rc = lib.simsd_chunk_attention_q4(*head, q4()[0], *tail)
    else:
        rc = lib.simsd_chunk_attention_sinks(*head, one, one, *tail)
    assert rc == status


@pytest.mark.parametrize("change", [dict(k_codes=0), dict(v_scales=0), dict(k_scales=264), dict(v_codes=4),
                                    dict(k_unit=0.0), dict(v_unit=-1.0), dict(k_unit=float("inf")),
                                    dict(v_unit=float("nan")), dict(k_unit=2.0 ** -65), dict(v_unit=2.0 ** 65)])
def test_cache_refusals(lib, change):
    c, _ = q4(**change)
    plan = simsd.simsd_rope_plan_init("half", 128, 1e4)
    assert lib.simsd_chunk_attention_q4(1, one, 1024, one, one, None, c, 4, one, 4, 64, 3, 2, 8, 2, 128, 1, 0, 0,
                                        F(0.0), one, None, one, 1 << 20, None, None) == BAD
    assert lib.simsd_rope_append_q4(1, ctypes.byref(plan), one, 1024, one, 256, one, 256, one, one, None, 3, 2, 8, 2,
                                    128, one, c, 4, one, 4, 64, None, None) == BAD
    assert lib.simsd_q4_expand(1, c, 4, one, 4, 64, one, one, 2, 2, 128, one, one, None, None) == BAD
    assert lib.simsd_q4_expand(1, None, 4, one, 4, 64, one, one, 2, 2, 128, one, one, None, None) == BAD


@pytest.mark.parametrize("change,status", [
    (dict(dtype=7), UNSUPPORTED), (dict(T=-1), BAD), (dict(d=32), UNSUPPORTED), (dict(P=12), UNSUPPORTED),
    (dict(q=odd), BAD), (dict(ks=2 * 128 - 8), BAD), (dict(out=None), BAD), (dict(start=None), BAD),
    (dict(plan=None), BAD), (dict(max_pages=1 << 26), UNSUPPORTED), (dict(T=0x7fffffff), UNSUPPORTED)])
def test_append_refusals(lib, change, status):
    plan = simsd.simsd_rope_plan_init("half", 64, 1e4)
    a = dict(dtype=1, plan=ctypes.byref(plan), q=one, ks=256, start=one, T=3, d=128, out=one, max_pages=4, P=64) | change
    assert lib.simsd_rope_append_q4(a["dtype"], a["plan"], a["q"], 1024, one, a["ks"], one, 256, a["start"], one,
                                    None, a["T"], 2, 8, 2, a["d"], a["out"], q4()[0], 4, one, a["max_pages"], a["P"],
                                    None, None) == status


def test_rotated_part_larger_than_the_head(lib):
    plan = simsd.simsd_rope_plan_init("half", 128, 1e4)
    assert lib.simsd_rope_append_q4(1, ctypes.byref(plan), one, 512, one, 128, one, 128, one, one, None, 3, 2, 8, 2,
                                    64, one, q4()[0], 4, one, 4, 64, None, None) == BAD


@pytest.mark.parametrize("change,status", [
    (dict(dtype=3), UNSUPPORTED), (dict(Bt=-1), BAD), (dict(d=48), UNSUPPORTED), (dict(P=20), UNSUPPORTED),
    (dict(first=None), BAD), (dict(k=odd), BAD), (dict(v=None), BAD), (dict(Hkv=1 << 20), UNSUPPORTED)])
def test_expand_refusals(lib, change, status):
    a = dict(dtype=1, Bt=2, d=128, P=64, first=one, k=one, v=one, Hkv=2) | change
    assert lib.simsd_q4_expand(a["dtype"], q4()[0], 4, one, 4, a["P"], a["first"], one, a["Bt"], a["Hkv"], a["d"],
                               a["k"], a["v"], None, None) == status


def arrays(*changes):
    out = []
    for c in changes or ({},):
        v = dict(base=256, page_bytes=64, layer_bytes=64 * 10, layers=2) | c
        out.append(simsd._PageArray(*v.values()))
    return (simsd._PageArray * len(out))(*out), len(out)


@pytest.mark.parametrize("change", [dict(base=0), dict(base=264), dict(page_bytes=0), dict(page_bytes=24),
                                    dict(layers=0), dict(layer_bytes=64 * 9), dict(layer_bytes=648)])
def test_array_refusals(lib, change):
    for a, n in (arrays(change), arrays({}, change)):
        assert lib.simsd_pages_fork(a, n, one, one, 1, one, one, one, 10, 4, 4, 8, one, 1 << 20, None, None) == BAD
        assert lib.simsd_pages_compact(a, n, one, one, 10, 4, 4, None, one, 1 << 20, None, None) == BAD


def test_page_refusals(lib):
    a, n = arrays()
    fork = lambda **k: lib.simsd_pages_fork(*(dict(  # noqa: E731
        a=a, na=n, src=one, dst=one, n=1, lens=one, table=one, refs=one, pages=10, Bt=4, mp=4, P=8, ws=one,
        bytes=1 << 20, err=None, stream=None) | k).values())
    for bad in (dict(na=9), dict(na=-1), dict(a=None), dict(src=None), dict(dst=None), dict(n=-1), dict(lens=None),
                dict(table=None), dict(refs=None), dict(refs=odd), dict(pages=-1), dict(P=0), dict(ws=None),
                dict(ws=odd), dict(bytes=16)):
        assert fork(**bad) == BAD, bad
    assert fork(Bt=65537) == UNSUPPORTED and fork(mp=1 << 29) == UNSUPPORTED
    assert fork(n=0) == 0 and fork(Bt=0) == 0
    assert lib.simsd_pages_extend(None, one, one, one, 10, 4, 4, 8, None, None) == BAD
    assert lib.simsd_pages_extend(one, one, None, one, 10, 4, 4, 8, None, None) == BAD
    assert lib.simsd_pages_extend(one, one, one, one, 10, 4, 4, -8, None, None) == BAD
    assert lib.simsd_pages_extend(one, one, one, one, 10, 0, 4, 8, None, None) == 0
    assert lib.simsd_pages_release(None, one, one, 3, one, one, 10, 4, 4, 8, None, None) == BAD
    assert lib.simsd_pages_release(one, None, one, 3, one, one, 10, 4, 4, 8, None, None) == BAD
    assert lib.simsd_pages_release(one, one, one, -1, one, one, 10, 4, 4, 8, None, None) == BAD
    assert lib.simsd_pages_release(one, one, one, 0, one, one, 10, 4, 4, 8, None, None) == 0
    need = lib.simsd_pages_workspace_bytes(10, 0)
    assert lib.simsd_pages_compact(a, n, one, one, 10, 4, 4, None, one, need - 1, None, None) == BAD
    assert lib.simsd_pages_compact(a, n, one, odd, 10, 4, 4, None, one, need, None, None) == BAD
    assert lib.simsd_pages_workspace_bytes(-1, 0) == 0


def test_binding_refuses_wrong_tensors():
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8)  # noqa: E731
    with pytest.raises(ValueError):  # scales of another width
        simsd.Q4Cache(u8(3, 2, 8, 64), u8(3, 2, 8, 4), u8(3, 2, 8, 64), u8(3, 2, 8, 8))
    with pytest.raises(ValueError):  # not on a GPU
        simsd.Q4Cache(u8(3, 2, 8, 64), u8(3, 2, 8, 8), u8(3, 2, 8, 64), u8(3, 2, 8, 8))
    for tensors in ([u8(3, 2, 8)], [u8(3, 2, 8, 64)] * 9, [u8(3, 2, 8, 64), u8(4, 2, 8, 64)],
                    [u8(3, 2, 8, 64)[..., :32]], [u8(3, 2, 8, 64)]):
        with pytest.raises(ValueError):
            simsd.PageSet(tensors)
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError):  # host memory
        simsd.simsd_pages_extend(i(2), i(2), i(2, 4), i(8), 4)
    with pytest.raises(ValueError):
        simsd.simsd_pages_release(i(2, 4).long(), i(8), i(2), i(2), 4)
    with pytest.raises(ValueError):
        q = torch.zeros(2, 4, 64)
        simsd.simsd_chunk_attention_sinks(q, i(2), i(1), torch.zeros(3, 2, 8, 64), torch.zeros(3, 2, 8, 64), i(1, 2),
                                          torch.zeros(2, 4, 64), 8, 1)


@pytest.mark.parametrize("mp", [4, 0])
def test_counts_are_looked_at_whatever_the_table(lib, mp):
    """A table of no columns does not excuse counts that are null or not on a
    16-byte boundary: they are read all the same."""
    a, n = arrays()
    for refs in (None, odd):
        assert lib.simsd_pages_extend(one, one, one, refs, 10, 4, mp, 8, None, None) == BAD
        assert lib.simsd_pages_release(one, one, one, 3, one, refs, 10, 4, mp, 8, None, None) == BAD
        assert lib.simsd_pages_fork(a, n, one, one, 1, one, one, refs, 10, 4, mp, 8, one, 1 << 20, None, None) == BAD
        assert lib.simsd_pages_compact(a, n, one, refs, 10, 4, mp, None, one, 1 << 20, None, None) == BAD
    assert lib.simsd_pages_extend(one, one, one, one, 10, 0, mp, 8, None, None) == 0


def test_granted_is_a_place_of_its_own(lib):
    tail = (10, 4, 4, 8)
    assert lib.simsd_pages_extend_granted(one, one, one, one, *tail, None, None, None) == BAD
    assert lib.simsd_pages_extend_granted(one, one, one, one, *tail, one, None, None) == BAD
    assert lib.simsd_pages_extend_granted(one, one, None, one, *tail, ctypes.c_void_p(512), None, None) == BAD
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError):
        simsd.simsd_pages_extend(i(2), i(2), i(2, 4), i(8), 4, granted=i(3))


def test_tables_whose_wanted_pages_pass_32_bits_are_refused(lib):
    """65536 sequences of 32768 entries each may want 2^31 pages, which a count
    of 32 bits has as a negative number: none were handed out, nor an error set."""
    assert lib.simsd_pages_extend(one, one, one, one, 1 << 20, 65536, 1 << 15, 8, None, None) == UNSUPPORTED
    assert lib.simsd_pages_extend_granted(one, one, one, one, 1 << 20, 65535, 1 << 16, 8, ctypes.c_void_p(512), None,
                                          None) == UNSUPPORTED

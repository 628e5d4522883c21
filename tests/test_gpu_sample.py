"""Sampling with temperature, top-k, top-p and min-p from given random numbers
on the GPU, against the plain 64-bit form."""
import numpy as np
import pytest
import torch

from paper_2606_02544_gb300 import simsd
from tests import _prompt as ref

pytestmark = pytest.mark.gpu


def run(x, u, T=None, k=None, p=None, mp=None, probs=True):
    R, V = x.shape
    dev = dict(device="cuda")
    f = lambda v: None if v is None else torch.as_tensor(np.asarray(v, dtype=np.float32), **dev)  # noqa: E731
    token = torch.full((R,), -9, dtype=torch.int32, **dev)
    kept = torch.full((R,), -9, dtype=torch.int32, **dev)
    lp = torch.full((R,), float("nan"), **dev)
    lps = torch.full((R, V), float("nan"), **dev) if probs else None
    err = torch.zeros(1, dtype=torch.int32, **dev)
    simsd.simsd_sample(x, f(u), token, temperature=f(T),
                       top_k=None if k is None else torch.as_tensor(np.asarray(k, dtype=np.int32), **dev), top_p=f(p),
                       min_p=f(mp), kept=kept, log_prob=lp, log_probs=lps, err_word=err)
    word = simsd.simsd_check_error(err)
    return token.cpu().numpy(), kept.cpu().numpy(), lp.cpu().numpy(), lps.cpu().numpy() if probs else None, word


def check(x, seed, T=1.0, k=0, p=1.0, mp=0.0, probs=True):
    """Every row with its own random number (and, as given, parameters)."""
    R, V = x.shape
    r = np.random.default_rng(seed)
    full = lambda v: np.broadcast_to(np.asarray(v, dtype=np.float64), (R,)).astype(np.float32).astype(np.float64).copy()  # noqa: E731
    T, p, mp = full(T), full(p), full(mp)
    k = np.broadcast_to(np.asarray(k), (R,)).copy()
    u = r.random(R)
    rows = x.double().cpu().numpy()
    for i in range(R):
        u[i], p[i], mp[i] = ref.settle(rows[i], u[i], T[i], k[i], p[i], mp[i])
    u, p, mp = (v.astype(np.float32) for v in (u, p, mp))
    token, kept, lp, lps, word = run(x, u, T, k, p, mp, probs)
    assert word == 0
    for i in range(R):
        t, idx, logp = ref.sample_row(rows[i], float(u[i]), T[i], k[i], float(p[i]), float(mp[i]))
        assert token[i] == t, i
        assert kept[i] == len(idx), i
        want = logp[list(idx).index(t)]
        # fp32: z = (x - m) / T correctly rounded, the logarithm of the sum to 2^-22 of a few tens
        tol = 2.0 ** -20 * (1 + abs(want))
        assert abs(lp[i] - want) <= tol, i
        if probs:
            dist = np.full(V, -np.inf)
            dist[idx] = logp
            assert np.array_equal(np.isfinite(lps[i]), np.isfinite(dist)), i
            ok = np.isfinite(dist)
            assert np.all(np.abs(lps[i][ok] - dist[ok]) <= 2.0 ** -20 * (1 + np.abs(dist[ok]))), i


def logits(R, V, spread, seed, dtype=torch.float32, banned=0.01):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(R, V, generator=g) * spread
    x.masked_fill_(torch.rand(V, generator=g) < banned, float("-inf"))
    x[:, seed % V] = 0.5  # a row with at least one logit
    return x.to(dtype).cuda()


LIMITS = [dict(), dict(k=1), dict(k=7), dict(k=100), dict(p=0.9), dict(p=0.999), dict(p=0.0), dict(mp=0.05),
          dict(k=40, p=0.8), dict(k=90, p=0.95, mp=0.01), dict(T=0.0), dict(T=0.0, k=5, p=0.5)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1, 2, 33, 1000, 5003])
@pytest.mark.parametrize("limits", range(len(LIMITS)))
def test_limits(dtype, V, limits):
    check(logits(6, V, 2.0, 3 * V + limits, dtype), V, **{"T": 0.8, **LIMITS[limits]})


@pytest.mark.parametrize("V,spread,limits", [
    (40001, 2.0, dict(p=0.9)), (40001, 1.0, dict(p=0.99)), (40001, 4.0, dict(p=0.95)), (40001, 2.0, dict(k=50, p=0.95)),
    (40001, 0.05, dict(p=0.9)),           # almost flat: bins of the histogram hold more than the list
    (40001, 0.02, dict(k=20000)), (40001, 1.0, dict(k=9000, p=0.9)), (151936, 2.0, dict(k=1000)),
    (151936, 3.0, dict(p=0.9)), (300007, 2.0, dict(p=0.5)), (151936, 2.0, dict()), (151936, 2.0, dict(mp=0.02))])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_large_vocabularies(V, spread, limits, dtype):
    check(logits(3, V, spread, V % 1000 + 1, dtype), V, **{"T": 0.9, **limits}, probs=False)


def test_many_rows_and_row_stride():
    """More rows than clusters of several CTAs are made for; rows that are not
    16-byte aligned."""
    wide = logits(700, 1201, 2.0, 5)
    check(wide[:, :1199], 1, k=30, p=0.9)


def test_a_temperature_of_every_size():
    x = logits(8, 3001, 2.0, 8)
    check(x, 2, T=[0.0, 1e-3, 0.1, 0.5, 1.0, 3.0, 50.0, 1e4], p=0.9)
    # so low that 1 / T overflows: only the first token (and its equals) have weight
    token, kept, lp, _, word = run(x, [0.5] * 8, T=[1e-42] * 8)
    assert word == 0 and np.array_equal(token, x.argmax(1).cpu().numpy()) and np.all(lp == 0)


def test_ties_go_to_the_lowest_index():
    x = torch.zeros(4, 50, device="cuda")
    x[:, 10:20] = 3.0
    x[1] = x[1].flip(0)
    token, kept, lp, lps, word = run(x, [0.99, 0.99, 0.0, 0.5], k=[4, 4, 15, 1])
    assert word == 0 and list(kept) == [4, 4, 15, 1]
    assert list(np.flatnonzero(np.isfinite(lps[0]))) == [10, 11, 12, 13]
    assert list(np.flatnonzero(np.isfinite(lps[1]))) == [30, 31, 32, 33]
    assert list(np.flatnonzero(np.isfinite(lps[2]))) == list(range(5)) + list(range(10, 20))
    assert list(token) == [13, 33, 0, 10]
    # top_p among equals: half of fifty equal tokens and no more
    y = torch.full((2, 50), -2.5, device="cuda")
    _, kept, _, lps, _ = run(y, [0.1, 0.9], p=[0.49, 0.5 + 1e-3])
    assert list(kept) == [25, 26]
    assert list(np.flatnonzero(np.isfinite(lps[0]))) == list(range(25))


@pytest.mark.parametrize("V", [70000, 1 << 20])
def test_ties_beyond_the_list(V):
    """More equal tokens than the list holds: found by index."""
    x = torch.zeros(2, V, device="cuda")
    x[:, V // 2] = 1.0
    token, kept, _, lps, word = run(x, [0.0, 0.999], k=[20001, 20001])
    assert word == 0 and list(kept) == [20001, 20001]
    assert np.isfinite(lps[0][:20000]).all() and not np.isfinite(lps[0][20000:V // 2]).any()
    assert token[0] == 0
    if V // 2 > 20000:
        w = np.where(np.arange(V) == V // 2, np.e, 1.0)[np.isfinite(lps[1])]
        at = np.flatnonzero(np.isfinite(lps[1]))
        assert token[1] == at[np.flatnonzero(np.cumsum(w) > np.float32(0.999) * w.sum())[0]]


def test_infinite_and_nan_logits():
    V = 300
    x = torch.randn(5, V, device="cuda")
    x[0, 7] = float("nan")                      # never drawn
    x[1, 3] = x[1, 200] = float("inf")          # share the weight
    x[2] = float("-inf")
    x[2, 250] = -1e30                           # the only one
    x[3] = float("-inf")                        # none: an error
    x[4, ::2] = torch.finfo(torch.float32).min  # masks of the type's lowest value
    token, kept, lp, lps, word = run(x, [0.9] * 5)
    assert word == simsd.EW_SAMPLE
    assert kept[0] == V - 1 and np.isneginf(lps[0, 7])
    assert token[1] == 200 and lp[1] == pytest.approx(-np.log(2), abs=1e-6)
    assert token[2] == 250 and kept[2] == 1 and lp[2] == 0
    assert token[3] == -1 and kept[3] == 0 and np.isneginf(lp[3]) and np.isneginf(lps[3]).all()
    assert token[4] % 2 == 1
    assert np.isfinite(lps[[0, 4]].max(1)).all()


def test_parameters_out_of_range():
    x = logits(8, 500, 1.0, 1)
    ok = run(x, [0.5] * 8)[0]
    nan, inf = float("nan"), float("inf")
    token, kept, lp, lps, word = run(x, [0.5, 1.0, -0.1, nan, 0.5, 0.5, 0.5, 0.5], T=[1, 1, 1, 1, -1.0, inf, nan, 1])
    assert word == simsd.EW_SAMPLE
    assert list(token[1:7]) == [-1] * 6 and list(kept[1:7]) == [0] * 6
    assert token[0] == ok[0] and token[7] == ok[7]
    token, _, _, _, word = run(x, [0.5] * 8, p=[nan] + [1.5] * 7, mp=[0.0, nan] + [0.0] * 6, k=[-3] * 8)
    assert word == simsd.EW_SAMPLE and list(token[:2]) == [-1, -1] and np.array_equal(token[2:], ok[2:])


def test_same_tokens_every_time():
    x = logits(20, 40000, 1.0, 2)
    u = np.random.default_rng(0).random(20)
    a, b = run(x, u, p=[0.9] * 20), run(x, u, p=[0.9] * 20)
    for s, t in zip(a[:4], b[:4]):
        assert np.array_equal(s, t)


def test_shares_over_a_grid_of_random_numbers():
    """One row under 20000 random numbers: every kept token in its share."""
    n, V = 20000, 200
    x = logits(1, V, 1.5, 4)
    u = (np.arange(n) + 0.5) / n
    token, kept, _, lps, _ = run(x.expand(n, V).contiguous(), u, k=[60] * n, p=[0.9] * n)
    got = np.bincount(token, minlength=V) / n
    assert np.allclose(got, np.exp(lps[0]), atol=2.0 / n)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("limits", [dict(p=0.9), dict(p=0.999), dict(k=30, p=0.95), dict(p=0.99, mp=0.01)])
def test_a_few_tokens_far_above_all_others(dtype, limits):
    """A certain next token: the sample that lays the histogram's bins need
    not hold it, whether it lies inside them or above them all."""
    x = logits(6, 40001, 2.0, 21, dtype)
    x[0, 77] = 19.0
    x[1, 30000] = x[1, 30001] = 25.0
    x[2, 4] = 60.0
    x[3, 40000], x[3, 39] = 400.0, 399.0
    x[4, 5000:5003] = 1e4
    check(x, 22, T=0.8, probs=False, **limits)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("hidden", [float("-inf"), -1e30, -1e4])
@pytest.mark.parametrize("limits", [dict(p=0.9), dict(k=3), dict(k=500, p=0.9), dict(p=0.95, mp=0.05)])
def test_all_but_a_few_tokens_masked(dtype, hidden, limits):
    """As under a grammar: none, one or some of the sampled tokens are open."""
    x = logits(5, 40001, 2.0, 23, torch.float32, banned=0.0)
    r = np.random.default_rng(24)
    for i, n in enumerate([1, 3, 40, 700, 9000]):
        open_ = torch.as_tensor(r.permutation(40001)[:n]).cuda()
        keep = x[i, open_].clone()
        x[i] = hidden
        x[i, open_] = keep
    check(x.to(dtype), 25, T=0.9, probs=False, **limits)


@pytest.mark.parametrize("V,spread,limits", [
    (40001, 1.0, dict(k=600)), (40001, 1.0, dict(k=1100, p=0.9)), (40001, 2.0, dict(k=2500, p=0.97, mp=0.001)),
    (40001, 1.0, dict(k=4096, p=0.9)), (40001, 1.0, dict(k=4097)), (5000, 0.5, dict(k=4900, p=0.99)),
    (40001, 0.5, dict(p=0.99, mp=0.4)),    # min_p cuts above what top_p leaves open
    (40001, 0.5, dict(k=30000, mp=0.3)), (40001, 2.0, dict(p=0.9999)), (40001, 2.0, dict(T=200.0, p=0.8)),
    (40001, 2.0, dict(T=0.01, p=0.9))])
def test_lists_of_every_length(V, spread, limits):
    check(logits(4, V, spread, 26), 27, **{"T": 1.0, **limits}, probs=False)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [5000, 40001])
@pytest.mark.parametrize("limits", [dict(k=50, p=0.9), dict(k=50, p=0.9, mp=0.3), dict(k=20000, p=0.5), dict(p=0.999)])
def test_fewer_open_tokens_than_top_k(dtype, V, limits):
    """Masked tokens fill top_k but have no weight; top_p cuts among the open
    ones.  One row has a weight just above and one just below nothing."""
    r = np.random.default_rng(31)
    x = torch.full((6, V), -1e30)
    for i, n in enumerate([1, 2, 10, 10, 49, 50]):
        x[i, torch.as_tensor(r.permutation(V)[:n])] = torch.randn(n, generator=torch.Generator().manual_seed(i))
    x[2, 11] = float(x[2].max()) - 20.0
    x[3, 11] = float(x[3].max()) - 60.0
    check(x.to(dtype).cuda(), 32, T=0.9, probs=False, **limits)


def test_equal_logits():
    """All of a row on one value: kept by index."""
    V = 151936
    x = torch.full((3, V), 0.25, device="cuda", dtype=torch.bfloat16)
    token, kept, lp, _, word = run(x, [0.0, 0.5, 0.999], p=[0.5 + 0.25 / V] * 3, probs=False)
    # float32 cannot hold the place between two tokens: within its rounding of half the vocabulary
    assert word == 0 and np.all(np.abs(kept - V / 2) <= 1 + V * 2.0 ** -24)
    assert token[0] == 0 and abs(token[1] - V / 4) <= 2 and np.allclose(lp, -np.log(kept), atol=1e-5)
    token, kept, _, _, _ = run(x, [0.0, 0.5, 0.999], k=[1, 70, V - 1], probs=False)
    assert list(kept) == [1, 70, V - 1] and token[0] == 0 and token[1] == 35


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,limits", [(1066, dict(k=79, p=0.95)), (1066, dict(p=0.9, mp=0.05)), (9000, dict(k=3000, p=0.99)),
                                      (9000, dict(p=0.999)), (9000, dict(T=50.0, p=0.7)), (9000, dict(k=7000))])
def test_many_short_rows(dtype, V, limits):
    """More short rows than two to a SM: smaller blocks, longer runs of the sort."""
    check(logits(400, V, 1.5, V, dtype), 33, **{"T": 0.9, **limits}, probs=V < 2000)


def between(x, us, T=1.0, k=0, mp=0.0):
    """For each u the first and the last token that it may fall on, and the
    number kept: cumulative weights in whole numbers of 2^-120 (a sum in
    doubles loses 2^-53 beside 1 with every token), all weights but the
    largest, which is exactly 1, within 2^-20 of themselves.  That covers the
    kernel's: z is exact in these tests, expf good to 2^-22, a sum of 16
    weights to 16 2^-24 / 2."""
    _, idx, _ = ref.sample_row(x, 0.5, T, k, 1.0, mp)
    by = np.sort(idx)
    w = np.exp((x[by] - x[by].max()) / T)
    top = x[by] == x[by].max()
    at = []
    for f in ((1 << 20) - 1, (1 << 20) + 1):
        c = np.cumsum(np.array([(1 << 120) if t else (int(v * 2.0 ** 100) << 20) * f >> 20 for v, t in zip(w, top)],
                               dtype=object))
        j = [int(np.searchsorted(c, int(float(u) * 2.0 ** 149) * c[-1] >> 149, side="right")) for u in us]
        at.append([int(by[min(i, len(by) - 1)]) for i in j])
    return np.minimum(*at), np.maximum(*at), len(idx)


ENDS = [0.0, 1e-45, 2.0 ** -24, 3 * 2.0 ** -24, 0.5, 1 - 2.0 ** -23, 1 - 2.0 ** -24]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,rows", [(4096, 7), (1201, 400), (151936, 7)])
@pytest.mark.parametrize("limits", [dict(), dict(k=1000), dict(k=100000), dict(mp=1e-30), dict(p=1 - 2.0 ** -24)])
def test_random_numbers_at_the_ends(dtype, V, rows, limits):
    """One token far above equal others, which together hold what the first
    or the last 2^-24 of the random numbers fall on: a token is drawn from
    them, by index, however small one of them is against the largest."""
    for gap in (26.5, 27.5, 28.5, 29.5, 31.0):
        for at in (0, V // 3, V - 1):
            x = torch.zeros(rows, V)
            x[:, at] = gap
            u = np.resize(np.asarray(ENDS, dtype=np.float32), rows)
            full = lambda v: None if v is None else [v] * rows  # noqa: E731
            token, kept, lp, _, word = run(x.to(dtype).cuda(), u, k=full(limits.get("k")), p=full(limits.get("p")),
                                           mp=full(limits.get("mp")), probs=False)
            assert word == 0
            assert (token >= 0).all() and np.array_equal(token, np.resize(token[:7], rows))
            if "p" in limits:  # (where that cuts hangs on the last bits of the sum)
                assert (kept >= 1).all() and np.isfinite(lp).all()
                continue
            row = x[0].to(dtype).double().numpy()
            lo, hi, n = between(row, u[:7], k=limits.get("k", 0), mp=limits.get("mp", 0.0))
            assert (lo <= token[:7]).all() and (token[:7] <= hi).all(), (gap, at)
            assert (kept == n).all()
            want = row[token[:7]] - gap - np.log1p((n - 1) * np.exp(-gap))
            assert (np.abs(lp[:7] - want) <= 2.0 ** -20 * (1 + np.abs(want))).all()


@pytest.mark.parametrize("V,rows", [(5003, 7), (1201, 400), (40001, 7)])
@pytest.mark.parametrize("limits", [dict(), dict(k=1), dict(k=900), dict(p=0.9), dict(mp=0.01), dict(T=0.0)])
def test_the_ends_of_ordinary_rows(V, rows, limits):
    """Zero (of either sign) falls on the first kept token, the largest number
    on a kept one; a weight that fp32 holds is a weight."""
    x = logits(rows, V, 2.0, 41)
    x[:, 0] = x.amax(1) - 90.0  # e^-90: below any sum's last bit, above zero
    full = lambda v: None if v is None else [v] * rows  # noqa: E731
    args = dict(T=full(limits.get("T")), k=full(limits.get("k")), p=full(limits.get("p")), mp=full(limits.get("mp")))
    rows64 = x[:7].double().cpu().numpy()
    for u in (0.0, -0.0, 1 - 2.0 ** -24):
        token, kept, lp, _, word = run(x, [u] * rows, probs=False, **args)
        assert word == 0
        for i in range(7):
            if limits.get("p"):
                continue  # (its cut hangs on the last bits of the sum)
            _, idx, _ = ref.sample_row(rows64[i], 0.5, limits.get("T", 1.0), limits.get("k", 0), 1.0,
                                       limits.get("mp", 0.0))
            assert token[i] == idx.min() if u == 0 else token[i] in idx
        assert (token >= 0).all() and np.isfinite(lp).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,rows", [(1201, 400), (9000, 4), (40001, 4)])
@pytest.mark.parametrize("T", [1e-10, 0.3, 1.0])
@pytest.mark.parametrize("limits", [dict(), dict(k=50), dict(k=700), dict(p=0.9), dict(k=700, p=0.9), dict(mp=0.01)])
def test_masks_of_the_lowest_value(dtype, V, rows, T, limits):
    """Finite masks so low that their distance over the temperature is past
    the largest number: no weight, and no NaN."""
    r = np.random.default_rng(51)
    low = torch.finfo(dtype).min
    x = torch.full((rows, V), low)
    for i in range(rows):
        n = [1, 40, 300, 900][i % 4]
        x[i, torch.as_tensor(r.permutation(V)[:n])] = torch.randn(n, generator=torch.Generator().manual_seed(i)) * 2
    x = x.to(dtype)
    x[1, 5] = -1e30
    rows64 = x.double().numpy()
    u, p, mp = (np.empty(rows) for _ in range(3))
    lim = dict(k=limits.get("k", 0), p=limits.get("p", 1.0), min_p=limits.get("mp", 0.0))
    T32 = float(np.float32(T))
    for i in range(rows):
        u[i], p[i], mp[i] = ref.settle(rows64[i], r.random(), T32, **lim)
    u, p, mp = (v.astype(np.float32) for v in (u, p, mp))
    token, kept, lp, lps, word = run(x.cuda(), u, [T] * rows, [lim["k"]] * rows, p, mp)
    assert word == 0 and not np.isnan(lps).any() and not np.isnan(lp).any()
    for i in range(rows):
        t, idx, logp = ref.sample_row(rows64[i], float(u[i]), T32, lim["k"], float(p[i]), float(mp[i]))
        assert token[i] == t and kept[i] == len(idx), i
        dist = np.full(V, -np.inf)
        with np.errstate(over="ignore"):
            dist[idx] = logp.astype(np.float32)  # (-inf where it is below fp32's range)
        ok = np.isfinite(dist)
        assert np.array_equal(np.isfinite(lps[i]), ok), i
        assert np.all(np.abs(lps[i][ok] - dist[ok]) <= 2.0 ** -20 * (1 + np.abs(dist[ok]))), i


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,rows", [(9001, 3), (40001, 3), (151936, 3), (40001, 60)])
@pytest.mark.parametrize("limits", [dict(), dict(p=0.9), dict(k=1000, p=0.98, mp=0.001)])
def test_distributions_of_rows_on_several_ctas(dtype, V, rows, limits):
    """Two, four and eight CTAs a row: the values of the distribution."""
    check(logits(rows, V, 2.5, 61, dtype), 62, **{"T": 0.8, **limits})


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,rows", [(9000, 400), (32003, 310), (32769, 310), (32003, 20)])
@pytest.mark.parametrize("limits", [dict(k=4500, p=0.9), dict(k=8000, p=0.99, mp=1e-4), dict(k=4097, p=0.5)])
def test_top_p_of_more_tokens_than_the_list_holds(dtype, V, rows, limits):
    """top_k beyond the list, then top_p of their sum, found by the search
    over the row: in blocks of 256 and of 512 threads and in clusters."""
    check(logits(rows, V, 2.0, 71, dtype), 72, **{"T": 0.7, **limits}, probs=False)

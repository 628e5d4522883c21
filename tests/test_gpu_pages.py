"""Pages of a cache on the GPU (fork, extend, release, compact) against their
definitions on lists; contents, tables and counts have to be equal."""
import numpy as np
import pytest
import torch

from paper_2606_02544_gb300 import simsd
from tests._longcache import Pool

pytestmark = pytest.mark.gpu
END = 2 ** 31 - 1


class Device:
    """A Pool beside the same on the GPU: page p of array a, layer l holds
    data[p] + 1000 a + 100 l in every place."""

    def __init__(self, ref, layers=2, shape=(2, 8, 16), pairs=64, dtype=torch.float32, arrays=2):
        self.ref = ref
        i32 = dict(dtype=torch.int32, device="cuda")
        self.table, self.refs, self.lens = (torch.tensor(x, **i32) for x in (ref.table, ref.refs, ref.lens))
        self.caches = []
        for a in range(arrays):
            x = torch.tensor(ref.data, device="cuda")[None, :, None, None, None] + 1000 * a
            x = x + 100 * torch.arange(layers, device="cuda")[:, None, None, None, None]
            self.caches.append(x.expand(layers, len(ref.data), *shape).to(dtype).contiguous())
        self.pages = simsd.PageSet(self.caches)
        self.ws = torch.full((simsd.simsd_pages_workspace_bytes(len(ref.refs), pairs),), 255, dtype=torch.uint8,
                             device="cuda")
        self.err = torch.zeros(1, **i32)
        self.live = torch.zeros(1, **i32)
        self.i32 = i32

    def t(self, x):
        return torch.tensor(np.asarray(x), **self.i32)

    def extend(self, add):
        simsd.simsd_pages_extend(self.lens, self.t(add), self.table, self.refs, self.ref.P, err_word=self.err)

    def release(self, seq, first, last):
        simsd.simsd_pages_release(self.table, self.refs, self.t(first), self.t(last), self.ref.P,
                                  seq=None if seq is None else self.t(seq), err_word=self.err)

    def fork(self, src, dst):
        simsd.simsd_pages_fork(self.pages, self.t(src), self.t(dst), self.lens, self.table, self.refs, self.ref.P,
                               workspace=self.ws, err_word=self.err)

    def compact(self):
        simsd.simsd_pages_compact(self.pages, self.table, self.refs, self.live, workspace=self.ws, err_word=self.err)
        return int(self.live)

    def grow(self, add):
        """Rows are written: lengths advance on both sides, and the pages of
        the new rows get contents of their own."""
        r = self.ref
        for b, n in enumerate(add):
            for k in range(r.lens[b] // r.P, -(-(r.lens[b] + n) // r.P) if n else 0):
                p = r.table[b, k]
                r.data[p] = 3 * r.data[p] % 10007 + 1
                for a, x in enumerate(self.caches):
                    for l in range(x.shape[0]):
                        x[l, p] = float(r.data[p] + 1000 * a + 100 * l)
            r.lens[b] += n
        self.lens.copy_(self.t(r.lens))

    def same(self, contents=True):
        r = self.ref
        assert np.array_equal(self.table.cpu().numpy(), r.table)
        assert np.array_equal(self.refs.cpu().numpy(), r.refs)
        assert np.array_equal(self.lens.cpu().numpy(), r.lens)
        held = torch.as_tensor(np.flatnonzero(r.refs > 0)).cuda()
        if not contents or not len(held):
            return
        data = torch.as_tensor(r.data).cuda()[held]
        for a, x in enumerate(self.caches):
            for l in range(x.shape[0]):
                want = (data + 1000 * a + 100 * l).to(x.dtype)[:, None, None, None].expand_as(x[l, held])
                assert torch.equal(x[l, held], want), (a, l)

    def word(self):
        w = simsd.simsd_check_error(self.err)
        self.err.zero_()
        return w


@pytest.mark.parametrize("seed,Bt,max_pages,num_pages,P,shape", [
    (0, 6, 9, 40, 4, (2, 4, 16)), (1, 40, 30, 700, 16, (1, 16, 4)), (2, 3, 5, 11, 1, (1, 1, 4)),
    (3, 300, 12, 2500, 8, (1, 8, 4)), (4, 2, 40, 61, 7, (3, 7, 12)), (5, 70, 6, 20011, 64, (1, 64, 4))])
def test_random_lives(seed, Bt, max_pages, num_pages, P, shape):
    """Sequences of calls as a serving loop makes them; after each everything
    is as the definitions have it."""
    rng = np.random.RandomState(seed)
    ref = Pool(Bt, max_pages, num_pages, P)
    if num_pages > 20000:  # pages far behind the first step of the search
        ref.refs[:17000] = 1
    dev = Device(ref, shape=shape, pairs=Bt)
    for _ in range(12):
        what = rng.randint(5)
        if what <= 1:
            room = max_pages * P - ref.lens
            add = np.minimum(room, rng.randint(0, 3 * P + 1, Bt)) * (rng.rand(Bt) < 0.6)
            # rows are not written into pages that a cut has left shared
            for b in range(Bt):
                ks = range(ref.lens[b] // P, -(-(ref.lens[b] + add[b]) // P) if add[b] else 0)
                if any(ref.table[b, k] >= 0 and ref.refs[ref.table[b, k]] > 1 for k in ks):
                    add[b] = 0
            ok = ref.extend(add)
            dev.extend(add)
            assert dev.word() == (0 if ok else simsd.EW_POOL)
            if ok:
                dev.grow(add)
        elif what == 2:
            seq = rng.permutation(Bt)[:rng.randint(1, Bt + 1)]
            first = rng.randint(0, 2 * P, len(seq)) * (rng.rand(len(seq)) < 0.5)
            last = np.where(rng.rand(len(seq)) < 0.5, END, rng.randint(0, max_pages * P + 1, len(seq)))
            ref.release(seq, first, last)
            dev.release(seq, first, last)
            for b, l in zip(seq, last):  # (rows whose pages are gone are not continued)
                if l == END:
                    ref.lens[b] = 0
                    ref.release([b], [0], [END])
                    dev.release([b], [0], [END])
            dev.lens.copy_(dev.t(ref.lens))
            assert dev.word() == 0
        elif what == 3:
            order = rng.permutation(Bt)
            n = rng.randint(1, max(2, Bt // 2))
            dst, src = order[:n], order[rng.randint(n, Bt, n)]
            ok = ref.fork(src, dst)
            dev.fork(src, dst)
            assert dev.word() == (0 if ok else simsd.EW_POOL)
        elif num_pages < 20000:
            assert dev.compact() == ref.compact()
            assert dev.word() == 0
        dev.same()


def test_many_pages_at_once():
    """More requests than a round of the search hands out, in one sequence and
    over many."""
    for Bt, max_pages, num_pages in ((1, 9001, 12000), (9000, 2, 30000)):
        ref = Pool(Bt, max_pages, num_pages, 2)
        ref.refs[::3] = 1
        dev = Device(ref, layers=1, shape=(1, 1, 4), arrays=1)
        add = np.full(Bt, 2 * max_pages - 1)
        if Bt > 1:
            add[::2] = 1
        if (ref.refs == 0).sum() < (add + 1).sum() // 2:
            add[0] -= 2 * 2000
        assert ref.extend(add)
        dev.extend(add)
        assert dev.word() == 0
        dev.same(contents=False)


def test_many_forks_at_once():
    ref = Pool(6001, 3, 20000, 4)
    dev = Device(ref, layers=1, shape=(1, 1, 4), pairs=6000, arrays=1)
    add = np.zeros(6001, dtype=int)
    add[0] = 6
    ref.extend(add), dev.extend(add), dev.grow(add)
    src, dst = np.zeros(6000, dtype=int), np.arange(1, 6001)
    assert ref.fork(src, dst)
    dev.fork(src, dst)
    assert dev.word() == 0
    dev.same()


def test_too_few_pages_change_nothing():
    ref = Pool(4, 4, 5, 8)
    dev = Device(ref)
    add = np.array([9, 0, 8, 0])
    assert ref.extend(add)
    dev.extend(add), dev.grow(add)
    for add in ([0, 17, 0, 0], [0, 8, 8, 8]):
        assert not ref.extend(np.array(add))
        dev.extend(add)
        assert dev.word() == simsd.EW_POOL
        dev.same()
    dev.grow(np.array([0, 0, 1, 0]) * 0)
    assert ref.fork([0, 2], [1, 3])  # one partial page, one whole one
    dev.fork([0, 2], [1, 3])
    assert dev.word() == 0
    dev.same()
    ref.release([1], [0], [END]), dev.release([1], [0], [END])
    add = np.array([0, 0, 9, 0])
    assert ref.extend(add)
    dev.extend(add)
    dev.grow(np.array([0, 0, 9, 0]))
    assert not ref.fork([0], [1])
    dev.fork([0], [1])
    assert dev.word() == simsd.EW_POOL
    dev.same()


def test_refused_pairs_and_lengths():
    ref = Pool(8, 3, 20, 4)
    dev = Device(ref)
    add = np.array([6, 7, 0, 0, 0, 3, 0, 0])
    ref.extend(add), dev.extend(add), dev.grow(add)
    # 2 is named twice, 1 is a source, 8 and -1 do not exist, 0 -> 3 stands
    src, dst = [0, 0, 0, 0, 8, 0, 1], [2, 2, 1, 8, 4, 3, 4]
    dst2 = [2, 2, 1, 8, -1, 3, 4]
    pairs = [(s, d) for s, d in zip(src, dst2)]
    assert ref.fork([s for s, _ in pairs], [d for _, d in pairs])
    dev.fork(src, dst2)
    assert dev.word() == simsd.EW_SEQ
    dev.same()
    # lengths outside the table
    dev.lens[6] = 13
    ref.lens[6] = 13
    dev.fork([6], [7])
    assert dev.word() == simsd.EW_PREFIX_LEN
    dev.extend(np.array([0, 0, 0, 0, 0, 0, 1, 0]))
    assert dev.word() == simsd.EW_PREFIX_LEN
    dev.extend(np.array([0, 0, 0, 0, 0, -1, 0, 2]))
    assert dev.word() == simsd.EW_PREFIX_LEN
    ref.extend(np.array([0, 0, 0, 0, 0, 0, 0, 2]))
    dev.same()
    dev.release([9], [0], [END])
    assert dev.word() == simsd.EW_SEQ
    # an entry that is no page, and a count that is too low
    dev.table[0, 0] = 20
    dev.release([0], [0], [4])
    assert dev.word() == simsd.EW_PAGE and int(dev.table[0, 0]) == -1
    dev.table[0, 0] = 19
    dev.release([0], [0], [4])
    assert dev.word() == simsd.EW_PAGE and int(dev.refs[19]) == 0


def test_shared_page_is_not_extended_into():
    """A sequence cut back into a page that a fork shares."""
    ref = Pool(3, 4, 20, 4)
    dev = Device(ref)
    add = np.array([8, 0, 5])
    ref.extend(add), dev.extend(add), dev.grow(add)
    ref.fork([0], [1]), dev.fork([0], [1])
    dev.same()
    dev.lens[1] = 6
    dev.extend([0, 5, 4])
    assert dev.word() == simsd.EW_SHARED
    ref.lens[1] = 6
    ref.extend(np.array([0, 0, 4]))
    dev.same()


def test_released_twice_and_empty_calls():
    ref = Pool(3, 4, 20, 4)
    dev = Device(ref)
    add = np.array([8, 16, 5])
    ref.extend(add), dev.extend(add), dev.grow(add)
    ref.release([1], [3], [13])
    dev.release([1, 1, 1], [3, 4, 3], [13, 12, 13])
    dev.release(None, [0, 0, 5], [0, 3, 2])
    dev.release([], [], [])
    dev.fork([], [])
    dev.extend([0, 0, 0])
    assert dev.word() == 0
    dev.same()
    assert dev.compact() == ref.compact()
    dev.same()
    assert dev.compact() == ref.compact()  # (nothing moves)
    dev.same()


@pytest.mark.parametrize("dtype,shape", [(torch.uint8, (2, 16, 8)), (torch.bfloat16, (8, 64, 128)),
                                         (torch.float32, (1, 1, 4))])
def test_contents_of_every_kind(dtype, shape):
    """Pages of one vector to several turns of a block, one layer and many."""
    g = torch.Generator(device="cuda").manual_seed(3)
    for layers in (1, 5):
        caches = [torch.randint(0, 256, (layers, 30, *shape[:2], w * torch.tensor([], dtype=dtype).element_size()),
                                dtype=torch.uint8, device="cuda", generator=g) for w in (shape[2], 2 * shape[2])]
        caches = [x if layers > 1 else x[0] for x in caches]
        before = [x.clone() for x in caches]
        i32 = dict(dtype=torch.int32, device="cuda")
        table = torch.tensor([[29, 4, -1], [17, 21, 3]], **i32)
        refs = torch.zeros(30, **i32)
        refs[table[table >= 0].long()] = 1
        err, live = torch.zeros(1, **i32), torch.zeros(1, **i32)
        pages = simsd.PageSet(caches)
        ws = torch.empty(simsd.simsd_pages_workspace_bytes(30, 1), dtype=torch.uint8, device="cuda")
        simsd.simsd_pages_compact(pages, table, refs, live, workspace=ws, err_word=err)
        assert table.tolist() == [[2, 4, -1], [0, 1, 3]] and int(live) == 5
        for x, y in zip(caches, before):
            at = (slice(None),) if layers > 1 else ()
            for p, q in ((2, 29), (4, 4), (0, 17), (1, 21), (3, 3)):
                assert torch.equal(x[(*at, p)], y[(*at, q)])
        lens = torch.tensor([5, 12], **i32)
        table = torch.cat([table, torch.full((1, 3), -1, **i32)])
        lens = torch.cat([lens, torch.zeros(1, **i32)])
        simsd.simsd_pages_fork(pages, torch.tensor([0], **i32), torch.tensor([2], **i32), lens, table, refs, 4,
                               workspace=ws, err_word=err)
        assert table[2].tolist() == [2, 5, -1] and lens.tolist() == [5, 12, 5] and simsd.simsd_check_error(err) == 0
        for x, y in zip(caches, before):
            assert torch.equal(x[:, 5] if layers > 1 else x[5], y[:, 4] if layers > 1 else y[4])


def test_replayed_graph():
    """All four calls captured once and replayed on other lengths and pairs."""
    ref = Pool(6, 8, 60, 4)
    dev = Device(ref, pairs=2)
    add, src, dst = dev.t(np.zeros(6, int)), dev.t([0, 0]), dev.t([1, 2])
    first, last, seq = dev.t([0]), dev.t([0]), dev.t([5])

    def calls():
        simsd.simsd_pages_release(dev.table, dev.refs, first, last, 4, seq=seq, err_word=dev.err)
        simsd.simsd_pages_fork(dev.pages, src, dst, dev.lens, dev.table, dev.refs, 4, workspace=dev.ws,
                               err_word=dev.err)
        simsd.simsd_pages_extend(dev.lens, add, dev.table, dev.refs, 4, err_word=dev.err)
        simsd.simsd_pages_compact(dev.pages, dev.table, dev.refs, dev.live, workspace=dev.ws, err_word=dev.err)

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        for _ in range(2):
            calls()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            calls()
    torch.cuda.synchronize()
    start = np.array([7, 0, 0, 9, 0, 14])
    ref.extend(start)
    dev.extend(start)
    dev.grow(start)
    for n, (a, sr, ds, f, l, q) in enumerate([([3, 1, 0, 9, 0, 0], [0, 3], [1, 2], 4, 12, 5),
                                              ([0, 0, 8, 0, 5, 0], [3, 1], [4, 0], 0, END, 5)]):
        for x, v in ((add, a), (src, sr), (dst, ds), (first, [f]), (last, [l]), (seq, [q])):
            x.copy_(dev.t(v))
        graph.replay()
        ref.release([q], [f], [l])
        assert ref.fork(sr, ds) and ref.extend(np.array(a))
        assert ref.compact() == int(dev.live) and dev.word() == 0
        held = ref.refs > 0
        for b in range(6):  # (pages that extend handed out hold what was there)
            for k in range(-(-ref.lens[b] // 4), 8):
                if ref.table[b, k] >= 0:
                    held[ref.table[b, k]] = False
        dev.same(contents=False)
        got = dev.caches[1][1, :, 0, 0, 0].cpu().numpy()
        assert np.array_equal(got[held], (ref.data + 1100)[held])


@pytest.mark.parametrize("num_pages,live", [(40003, 0.5), (16384, 0.7), (16385, 0.02), (33000, 1.0), (33000, 0.0)])
def test_large_pools_are_made_dense(num_pages, live):
    """More pages than a step of the search, more moves than its list."""
    rng = np.random.RandomState(num_pages)
    ref = Pool(50, 900, num_pages, 1)
    used = rng.permutation(num_pages)[:min(45000, int(live * num_pages))]
    ref.refs[used] = 1
    for b in range(50):  # (some pages are in no table)
        row = used[b::50][:899]
        ref.table[b, 1:1 + len(row)] = row
    dev = Device(ref, layers=1, shape=(1, 1, 4), arrays=1)
    assert dev.compact() == ref.compact()
    assert dev.word() == 0
    dev.same()
    assert (ref.refs[:int((ref.refs > 0).sum())] > 0).all()


def test_pools_past_four_gigabytes():
    """Pages whose contents lie past 2^32 bytes: forked and moved from there."""
    n, i32 = 4200, dict(dtype=torch.int32, device="cuda")
    cache = torch.zeros(1, n, 8, 64, 2048, dtype=torch.uint8, device="cuda")  # 1 MB a page
    cache[0, n - 1] = 7
    cache[0, n - 2, :, :, ::3] = 9
    table = torch.tensor([[n - 1, n - 2], [-1, -1]], **i32)
    refs, lens = torch.zeros(n, **i32), torch.tensor([100, 0], **i32)
    refs[n - 2:] = 1
    pages, err, live = simsd.PageSet([cache]), torch.zeros(1, **i32), torch.zeros(1, **i32)
    ws = torch.empty(simsd.simsd_pages_workspace_bytes(n, 1), dtype=torch.uint8, device="cuda")
    simsd.simsd_pages_fork(pages, torch.tensor([0], **i32), torch.tensor([1], **i32), lens, table, refs, 64,
                           workspace=ws, err_word=err)
    assert table.tolist() == [[n - 1, n - 2], [n - 1, 0]] and torch.equal(cache[0, 0], cache[0, n - 2])
    simsd.simsd_pages_compact(pages, table, refs, live, workspace=ws, err_word=err)
    assert table.tolist() == [[2, 1], [2, 0]] and int(live) == 3 and refs[:3].tolist() == [1, 1, 2]
    assert bool((cache[0, 2] == 7).all()) and torch.equal(cache[0, 1], cache[0, 0])
    assert simsd.simsd_check_error(err) == 0


@pytest.mark.parametrize("Bt,free", [(24, 400), (24, 3), (1500, 20000), (1500, 700)])
def test_extend_says_which_sequences_may_go_on(Bt, free):
    """Lengths of sequences that have their pages, -1 for those that were
    refused, and with too few free pages for all that want one."""
    P, max_pages = 4, 40
    i32 = dict(dtype=torch.int32, device="cuda")
    rng = np.random.RandomState(Bt + free)
    used = Bt * 3
    table = np.full((Bt, max_pages), -1)
    table[:, :3] = rng.permutation(used).reshape(Bt, 3)
    refs = np.zeros(used + free, dtype=int)
    refs[:used] = 1
    lens, add = np.full(Bt, 10), rng.choice([0, 2, 3, 7, 50, 130], Bt)
    kind = np.arange(Bt) % 8
    table[kind == 1, 2] = table[0, 2]  # shared (with sequence 0 too)
    refs[:used] = np.bincount(table[:, :3].ravel(), minlength=used)
    lens[kind == 2] = -3
    add[kind == 3] = 151  # past the table
    table[kind == 4, 2] = used + free + 7
    add[kind == 5] = -1
    wants = np.array([sum(table[b, k] == -1 for k in range(lens[b] // P, -(-(lens[b] + add[b]) // P)))
                      if add[b] > 0 and lens[b] >= 0 and lens[b] + add[b] <= max_pages * P else 0 for b in range(Bt)])
    wrong = (kind == 2) | (kind == 3) | (kind == 5) | ((kind == 4) & (add > 0)) | ((kind == 1) & (add > 0))
    wrong[0] = add[0] > 0
    wants[wrong] = 0
    short = wants.sum() > free
    assert short == (free in (3, 700))
    t = lambda x: torch.tensor(np.asarray(x), **i32)  # noqa: E731
    got, err, tab, cnt = torch.full((Bt,), 77, **i32), torch.zeros(1, **i32), t(table), t(refs)
    plain = [t(table), t(refs), torch.zeros(1, **i32)]
    simsd.simsd_pages_extend(t(lens), t(add), tab, cnt, P, err_word=err, granted=got)
    simsd.simsd_pages_extend(t(lens), t(add), plain[0], plain[1], P, err_word=plain[2])
    assert all(torch.equal(a, b) for a, b in zip((tab, cnt, err), plain))
    no = wrong | ((wants > 0) if short else False)
    assert np.array_equal(got.cpu().numpy(), np.where(no, -1, lens))
    word = simsd.simsd_check_error(err)
    assert bool(word & simsd.EW_POOL) == short and word & simsd.EW_PREFIX_LEN and torch.equal(tab, t(table)) == short

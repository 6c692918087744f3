"""The books of a cache's pages, and the copies behind them, against the same place by place on the host: everything has to be equal."""
import numpy as np
import pytest

import pages_ref as P

pytestmark = pytest.mark.gpu

# pages, sequences, places, tokens of a page: nothing, single ones, around a block's and a wave's counts, several chunks of pages, many sequences
SIZES = [(0, 0, 0, 16), (0, 3, 4, 16), (5, 0, 7, 16), (5, 2, 0, 32), (1, 1, 1, 16), (3, 1, 9, 64), (40, 3, 8, 16), (70, 5, 65, 32), (4095, 30, 64, 64), (4097, 7, 300, 16), (9000, 70, 63, 128),
         (20000, 257, 33, 16), (70000, 64, 500, 48), (300, 1100, 3, 16),
         (4000, 60, 100, 16), (8192, 1024, 5, 16), (8192, 16, 256, 16), (50, 300, 20, 16), (8193, 200, 40, 32)]


@pytest.fixture(scope="module")
def B():
    from paper_2401_10652_amd import binding
    binding.lib()
    return binding


def ints(x):
    import torch
    return torch.from_numpy(np.asarray(x, np.int64).astype(np.int32)).cuda()


class Device:
    """The books on the device, and others behind them that hold nonsense; same: which of the arrays are the same for both."""

    def __init__(self, B, books, places, same=()):
        import torch
        batch = len(books.table)
        self.uses, self.table = ints(books.uses), ints(books.table).view(batch, places)
        self.uses_out = self.uses if "uses" in same else torch.full_like(self.uses, 77)
        self.table_out = self.table if "table" in same else torch.full_like(self.table, 88)
        self.before, self.same = (self.uses.clone(), self.table.clone()), same
        self.books, self.out = B.page_books(self.uses, self.table, books.page), B.page_books(self.uses_out, self.table_out, books.page)
        need = B.ac_pages_workspace_bytes(self.books)
        self.room = torch.full((need + 64,), 0xa5, dtype=torch.uint8, device="cuda")
        self.workspace = self.room[:need]
        self.count = torch.full((1,), -5, dtype=torch.int32, device="cuda")

    def check(self, books, count):
        assert self.uses_out.tolist() == books.uses and self.table_out.tolist() == books.table and self.count.item() == count
        assert (self.room[self.workspace.numel():] == 0xa5).all()
        for name, now, before in zip(("uses", "table"), (self.uses, self.table), self.before):
            assert name in self.same or (now == before).all()


def layers(B, rng, pages, page, shapes, gap=0):
    """Caches of random codes; (kv_caches, host arrays of each, device tensors)."""
    import torch
    descs, hosts, down = [], [], []
    for heads, d in shapes:
        host = [rng.integers(0, 256, s).astype(np.uint8) for s in ((pages, heads, page, d), (pages, heads, page // 16, d, 16))]
        host += [rng.standard_normal((pages, heads, page // 16)).astype(np.float32) for _ in range(2)]
        dev = []
        for x in host:
            flat = torch.from_numpy(x.reshape(pages, int(np.prod(x.shape[1:])))).cuda()
            spread = torch.zeros((pages, flat.shape[1] + gap), dtype=flat.dtype, device="cuda")
            spread[:, :flat.shape[1]] = flat
            dev.append(spread[:, :flat.shape[1]].unflatten(1, x.shape[1:]))
        descs.append(B.kv_cache(*dev))
        hosts.append(host)
        down.append(dev)
    return B.kv_caches(descs), hosts, down


def check_layers(hosts, devs, moves):
    for host, dev in zip(hosts, devs):
        for want, got in zip(P.copied(host, moves), dev):
            assert np.array_equal(want, got.cpu().numpy())


@pytest.mark.parametrize("same", [(), ("uses",), ("table",), ("uses", "table")])
@pytest.mark.parametrize("pages,batch,places,page", SIZES)
def test_update(B, pages, batch, places, page, same):
    rng = np.random.default_rng(pages * 7 + batch)
    books = P.random_books(rng, pages, batch, places, page)
    tokens = places * page
    ends = lambda: np.sort(rng.integers(-40, tokens + 200, (2, batch)), 0)  # noqa: E731
    drop, take = ends(), ends()
    if batch > 2:
        drop[:, 0], drop[:, 1], take[:, 1] = (5, 5), (0, (1 << 31) - 1), (-(1 << 31), (1 << 31) - 1)       # nothing; the whole sequence; the whole of another
        take[:, 2] = (50, 20)
    for d, t in ((drop, take), (drop, None), (None, take), (None, None)):
        dev = Device(B, books, places, same)
        after = P.Books(books.uses, books.table, page)
        short = after.update(d, t)
        B.ac_op_pages_update(dev.books, dev.out, dev.workspace, None if d is None else tuple(ints(x) for x in d), None if t is None else tuple(ints(x) for x in t), dev.count)
        dev.check(after, short)


@pytest.mark.parametrize("pages,batch,places,page", [(700, 64, 16, 16), (600, 41, 25, 32), (900, 64, 32, 16), (1500, 3, 683, 16), (2000, 17, 241, 16)])
def test_tables_that_fill_their_threads(B, pages, batch, places, page):
    """Up to 1024, 2048 and 4096 places, and one more: a thread has one, two or four, or several launches go through them."""
    for same in ((), ("uses", "table")):
        test_update(B, pages, batch, places, page, same)
        test_compact(B, pages, batch, places, page, same)
    test_fork(B, pages, batch, places, page, ())


def test_update_runs_dry_and_frees_what_it_takes(B):
    """One page for many places; pages that this very call frees are taken; no one counts what is missing."""
    books = P.Books([1, 1, 0, 1], [[0, 1, -1, -1], [3, -1, -1, -1]], 16)
    dev = Device(B, books, 4, ("uses", "table"))
    drop, take = ([0, 0], [16, 0]), ([16, 0], [64, 64])
    short = books.update(drop, take)
    assert short == 3 and books.table == [[-1, 1, 0, 2], [3, -1, -1, -1]]
    B.ac_op_pages_update(dev.books, dev.out, dev.workspace, tuple(ints(x) for x in drop), tuple(ints(x) for x in take), dev.count)
    dev.check(books, short)
    B.ac_op_pages_update(dev.books, dev.out, dev.workspace, tuple(ints(x) for x in drop), tuple(ints(x) for x in take))
    books.update(drop, take)
    dev.check(books, 3)


@pytest.mark.parametrize("same", [(), ("uses",)])
@pytest.mark.parametrize("pages,batch,places,page", SIZES)
def test_fork(B, pages, batch, places, page, same):
    import torch
    rng = np.random.default_rng(pages * 5 + batch)
    shapes = [(2, 32), (1, 64)] if pages < 1000 else [(1, 32)]
    for fill in (0.3, 0.9):
        books = P.random_books(rng, pages, batch, places, page, fill)
        if batch > 3:
            books.length[:4] = [0, page * (places // 2), -3, places * page + 100]
        caches, hosts, devs = layers(B, rng, pages, page, shapes, gap=16)
        parent = rng.integers(-1, batch + 1, batch) if batch else np.zeros(0)
        parent[:batch // 3] = parent[-1] if batch else 0                     # many of one
        dev = Device(B, books, places, same)
        length, length_out = ints(books.length), torch.full((batch,), -9, dtype=torch.int32, device="cuda")
        short, moves = books.fork([int(p) for p in parent])
        B.ac_op_cache_fork(caches, dev.books, dev.out, ints(parent), length, length_out, dev.workspace, dev.count)
        dev.check(books, short)
        assert length_out.tolist() == books.length
        check_layers(hosts, devs, moves)


def test_fork_of_beams_again_and_again(B):
    """A search's steps: the books turn between two places, the last pages' copies come from those that beams without children give up; nothing is lost or kept."""
    import torch
    rng = np.random.default_rng(3)
    prompts, beams, page, places = 3, 4, 16, 12
    batch = prompts * beams
    table, at = np.full((batch, places), -1, np.int64), 0
    length = np.repeat([40, 16, 5], beams)
    for b in range(0, batch, beams):                                        # the first beam has the prompt
        n = -(-length[b] // page)
        table[b, :n] = np.arange(at, at + n)
        at += n
    length[np.arange(batch) % beams > 0] = 0
    pages = at + prompts * 8 + batch * 2 + 6
    books = P.Books([int((table == p).sum()) for p in range(pages)], table, page, length)
    caches, hosts, devs = layers(B, rng, pages, page, [(2, 32)])
    uses, one, other = ints(books.uses), ints(table), torch.full((batch, places), 5, dtype=torch.int32, device="cuda")
    lengths = [ints(books.length), torch.zeros(batch, dtype=torch.int32, device="cuda")]
    both = [B.page_books(uses, one, page), B.page_books(uses, other, page)]
    ws, count = B.empty_workspace(B.ac_pages_workspace_bytes(both[0])), torch.zeros(1, dtype=torch.int32, device="cuda")
    for step in range(30):
        parent = np.array([b // beams * beams + (0 if step == 0 else rng.integers(0, beams)) for b in range(batch)])
        if step % 7 == 6:
            parent[rng.integers(0, batch)] = -1
        short, moves = books.fork([int(p) for p in parent])
        hosts = [P.copied(h, moves) for h in hosts]
        B.ac_op_cache_fork(caches, both[step % 2], both[1 - step % 2], ints(parent), lengths[step % 2], lengths[1 - step % 2], ws, count)
        now = both[1 - step % 2]
        assert short == 0 == count.item() and now.keep[1].tolist() == books.table and uses.tolist() == books.uses and lengths[1 - step % 2].tolist() == books.length
        check_layers(hosts, devs, [])
        grow = [books.length, [n + int(rng.integers(1, 6)) if n and n < places * page - 6 else n for n in books.length]]
        short = books.update(None, grow)
        books.length = grow[1]
        B.ac_op_pages_update(now, now, ws, None, tuple(ints(x) for x in grow), count)
        lengths[1 - step % 2].copy_(ints(grow[1]))
        assert short == 0 == count.item() and now.keep[1].tolist() == books.table and uses.tolist() == books.uses
    assert sum(books.uses) == sum(e >= 0 for row in books.table for e in row)


@pytest.mark.parametrize("same", [(), ("uses", "table")])
@pytest.mark.parametrize("pages,batch,places,page", SIZES)
def test_compact(B, pages, batch, places, page, same):
    rng = np.random.default_rng(pages * 3 + batch)
    for fill, shapes in ((0.5, [(2, 32), (1, 96)] if pages < 1000 else [(1, 32)]), (0.05, []), (1.0, [])):
        books = P.random_books(rng, pages, batch, places, page, fill)
        caches, hosts, devs = layers(B, rng, pages, page, shapes, gap=16)
        dev = Device(B, books, places, same)
        n, moves = books.compact()
        B.ac_op_cache_compact(caches, dev.books, dev.out, dev.workspace, dev.count)
        dev.check(books, n)
        check_layers(hosts, devs, moves)


def test_compact_keeps_entries_that_uses_does_not_know(B):
    """A place that names a page which uses holds for free, before and behind the pages in use; uses below zero are free."""
    books = P.Books([1, 0, -2, 0, 3, 0, 1, -1], [[0, 4, 7, 5], [4, 6, 1, -1]], 32)
    dev = Device(B, books, 4)
    n, moves = books.compact()
    assert n == 3 and moves == [(6, 1, 32), (4, 2, 32)] and books.table == [[0, 2, 7, 5], [2, 1, 1, -1]]
    B.ac_op_cache_compact(B.kv_caches([]), dev.books, dev.out, dev.workspace, dev.count)
    dev.check(books, n)


@pytest.mark.parametrize("heads,d,page", [(1, 32, 16), (2, 64, 64), (5, 96, 48), (3, 192, 16), (8, 128, 64), (2, 256, 128), (1, 256, 512)])
def test_copy_pages(B, heads, d, page):
    rng = np.random.default_rng(heads * d)
    pages = 30
    for n, gap in ((0, 0), (1, 0), (7, 16), (14, 48)):
        order = rng.permutation(pages)
        source, target = order[:n].copy(), order[n:2 * n].copy()
        if n > 5:
            source[0], target[1], source[2], target[2], target[3] = -1, pages, pages + 3, -1, source[3]
        for tokens in (None, rng.integers(-3, page + 20, n)):
            caches, hosts, devs = layers(B, rng, pages, page, [(heads, d), (1, 32)], gap)
            B.ac_op_cache_copy_pages(caches, ints(source), ints(target), None if tokens is None else ints(tokens))
            moves = [(a, b, page if tokens is None else int(tokens[i])) for i, (a, b) in enumerate(zip(source, target)) if 0 <= a < pages and 0 <= b < pages]
            check_layers(hosts, devs, moves)


def test_copies_of_many_layers_and_far_pages(B):
    """More caches than a launch takes; pages that begin past 2^32 bytes."""
    import torch
    rng = np.random.default_rng(9)
    caches, hosts, devs = layers(B, rng, 6, 16, [(1 + i % 3, 32) for i in range(37)])
    B.ac_op_cache_copy_pages(caches, ints([0, 5]), ints([3, 1]), ints([16, 3]))
    check_layers(hosts, devs, [(0, 3, 16), (5, 1, 3)])
    pages, heads, page, d = 1 << 15, 2, 128, 256
    k, v = (torch.zeros((pages, 2 * heads * page * d), dtype=torch.uint8, device="cuda") for _ in "kv")
    k, v = k[:, :heads * page * d].unflatten(1, (heads, page, d)), v[:, :heads * page * d].unflatten(1, (heads, page // 16, d, 16))
    ks, vs = (torch.zeros((pages, heads, page // 16), device="cuda") for _ in "kv")
    for t in (k, v, ks, vs):
        t[3] = (torch.rand(t[3].shape, device="cuda") * 200 + 1).to(t.dtype)
    caches = B.kv_caches([B.kv_cache(k, v, ks, vs)])
    assert caches[0].stride_page * (pages - 1) >= (1 << 32) - (1 << 18)
    B.ac_op_cache_copy_pages(caches, ints([3, pages - 1]), ints([pages - 2, 2]))
    for t in (k, v, ks, vs):
        assert torch.equal(t[pages - 2], t[3]) and not t[2].any() and not t[4].any() and not t[pages - 1].any()


def test_books_from_a_graph(B):
    """Update, fork and compact captured together and replayed, with other parents and lengths each time."""
    import torch
    rng = np.random.default_rng(5)
    batch, places, page, pages = 12, 9, 16, 90
    books = P.random_books(rng, pages, batch, places, page, fill=0.4, strange=0.0)
    caches, hosts, devs = layers(B, rng, pages, page, [(2, 32)])
    uses, table, spare = ints(books.uses), ints(books.table), torch.zeros((batch, places), dtype=torch.int32, device="cuda")
    length, length_out, parent = ints(books.length), ints([0] * batch), ints([0] * batch)
    drop, take = [ints([0] * batch) for _ in "ab"], [ints([0] * batch) for _ in "ab"]
    now, then = B.page_books(uses, table, page), B.page_books(uses, spare, page)
    ws, counts = B.empty_workspace(B.ac_pages_workspace_bytes(now)), [ints([0]) for _ in "abc"]

    def work():
        B.ac_op_pages_update(now, now, ws, drop, take, counts[0])
        B.ac_op_cache_fork(caches, now, then, parent, length, length_out, ws, counts[1])
        B.ac_op_cache_compact(caches, then, now, ws, counts[2])
        length.copy_(length_out)
    B.ac_op_pages_update(now, now, ws)
    B.ac_op_cache_fork(B.kv_caches([]), then, B.page_books(uses.clone(), table.clone(), page), parent, length, length_out, ws)     # (kernels are loaded)
    B.ac_op_cache_copy_pages(caches, ints([0]), ints([0]))
    B.ac_op_cache_compact(B.kv_caches([]), B.page_books(uses.clone(), spare, page), B.page_books(uses.clone(), spare.clone(), page), ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for step in range(6):
        d, t = (np.sort(rng.integers(0, places * page, (2, batch)), 0) for _ in "ab")
        p = rng.integers(-1, batch, batch)
        for x, y in zip((*drop, *take, parent), (*d, *t, p)):
            x.copy_(ints(y))
        if step == 3:
            work()                                                          # (eager between the replays)
        else:
            graph.replay()
        short = books.update(d, t)
        again, copies = books.fork([int(x) for x in p])
        n, moves = books.compact()
        hosts = [P.copied(P.copied(h, copies), moves) for h in hosts]
        torch.cuda.synchronize()
        assert uses.tolist() == books.uses and table.tolist() == books.table and length.tolist() == books.length
        assert [c.item() for c in counts] == [short, again, n]
        check_layers(hosts, devs, [])

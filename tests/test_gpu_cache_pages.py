"""The paged cache's books and rows, against the same calls on Python lists."""
import random

import pytest
import torch

from cache_util import Books, ancestor_sets, mask_words

pytestmark = pytest.mark.gpu
BF, F16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def b():
    from paper_2605_10453_amd import binding
    return binding


def dev(xs):
    return torch.tensor(xs, dtype=torch.int32, device="cuda")


def same_books(cache, books):
    """Equal books: lengths, holdings and counts, and the table where it means something."""
    assert cache.held.tolist() == books.held and cache.lens.tolist() == books.lens and cache.refs.tolist() == books.refs
    table = cache.table.tolist()
    for s, m in enumerate(books.held):
        assert table[s][:m] == books.table[s][:m], s


def firsts(counts):
    first = [0]
    for t in counts:
        first.append(first[-1] + t)
    return first


@pytest.mark.parametrize("pages,P,slots,slot_pages,seed", [(40, 16, 9, 12, 0), (700, 16, 60, 40, 1), (9000, 64, 300, 70, 2), (3, 32, 4, 8, 3), (4099, 16, 5, 4000, 4)])
def test_books_follow_the_lists(b, pages, P, slots, slot_pages, seed):
    """A long random run of reserving, settling, forking and freeing, calls that must be refused among them."""
    rng = random.Random(seed)
    cache = b.PagedCache.empty(1, pages, 1, P, 8, slots, slot_pages)
    books = Books(pages, P, slots, slot_pages)
    refused = {"reserve": 0, "fork": 0}
    for step in range(60):
        n = rng.randint(0, min(slots, rng.choice([1, 4, slots])))
        some = rng.sample(range(slots), n)
        do = rng.choice(["reserve", "reserve", "settle", "fork", "free"])
        if do == "reserve":
            most = rng.choice([1, 3 * P, max(1, pages * P // max(1, n))])
            counts = [rng.randint(0, most) for _ in some]
            want = books.reserve(some, counts)
            assert b.cache_reserve(cache, dev(some), dev(firsts(counts))).item() == want, step
            refused["reserve"] += want != 0
            # what was reserved is filled, or part of it
            if want == 0:
                lens = [min(books.lens[s] + rng.randint(0, t), books.held[s] * P) for s, t in zip(some, counts)]
                books.set_lens(some, lens)
                b.cache_set_lens(cache, dev(some), dev(lens))
        elif do == "settle":
            lens = [rng.randint(-1, books.held[s] * P + 3) for s in some]
            books.set_lens(some, lens)
            b.cache_set_lens(cache, dev(some), dev(lens))
        elif do == "free":
            books.set_lens(some, [0] * n)
            b.cache_set_lens(cache, dev(some))
        else:
            empty = [s for s in range(slots) if books.held[s] == 0 and books.lens[s] == 0]
            children = rng.sample(empty, min(len(empty), max(1, n)))
            parents = [rng.choice([s for s in range(slots) if s != c]) for c in children]
            want, _ = books.fork(parents, children)
            assert b.cache_fork(cache, dev(parents), dev(children)).item() == want, step
            refused["fork"] += want != 0
        same_books(cache, books)
        assert all(r >= 0 for r in books.refs) and sum(books.refs) == sum(books.held)
    print("refused", refused, flush=True)


def test_refusals_that_the_books_decide(b):
    cache = b.PagedCache.empty(1, 10, 1, 16, 8, 4, 6)
    books = Books(10, 16, 4, 6)

    def reserve(slots, counts):
        want = books.reserve(slots, counts)
        assert b.cache_reserve(cache, dev(slots), dev(firsts(counts))).item() == want
        same_books(cache, books)
        return want

    assert reserve([0, 1], [40, 17]) == 0                       # 3 + 2 pages
    assert reserve([2], [97]) == -1                             # 7 pages where a slot has 6
    assert reserve([2, 3], [96, 1]) == 2                        # 7 pages, 5 free
    assert reserve([2, 4], [1, 1]) == -1                        # no such slot
    assert reserve([2, 3], [64, 16]) == 0                       # the last five
    assert reserve([3], [17]) == 1
    assert reserve([], []) == 0
    # a range that runs backwards
    assert b.cache_reserve(cache, dev([0, 1]), dev([5, 3, 4])).item() == -1
    same_books(cache, books)
    b.cache_set_lens(cache, dev([0, 1, 7, -1]), dev([40, 16, 3, 3]))       # slots that do not exist are left out
    books.set_lens([0, 1], [40, 16])
    same_books(cache, books)
    for parents, children in (([0], [1]), ([0], [0]), ([0], [5]), ([-1], [2])):
        assert b.cache_fork(cache, dev(parents), dev(children)).item() == -1
        same_books(cache, books)
    # a parent that does not hold its tokens' pages
    b.cache_set_lens(cache, dev([2, 3]))
    books.set_lens([2, 3], [0, 0])
    cache.lens[0] = 49
    assert b.cache_fork(cache, dev([0]), dev([2])).item() == -1
    cache.lens[0] = 40
    same_books(cache, books)
    assert b.cache_fork(cache, dev([]), dev([])).item() == 0
    # more forks than there are free pages for their last pages, then as many as there are
    b.cache_reserve(cache, dev([3]), dev([0, 80]))
    books.reserve([3], [80])
    assert books.fork([0], [2]) == (0, [(books.table[0][2], books.table[2][2], 8)])
    assert b.cache_fork(cache, dev([0]), dev([2])).item() == 0
    same_books(cache, books)


def test_more_wanted_than_31_bits(b):
    """Far more pages than there are, and more than a 32-bit number counts: nothing changes."""
    n = 4096
    cache = b.PagedCache.empty(1, 5, 1, 16, 8, 1, (1 << 27) - 1)
    # the same slot again and again: not a batch that may be reserved, but one that is refused before that matters
    slots, first = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.arange(n + 1, dtype=torch.int32, device="cuda") << 18
    assert b.cache_reserve(cache, slots, first).item() == n * (1 << 14) - 5
    assert cache.held.item() == 0 and cache.refs.sum().item() == 0
    cache.lens.fill_((1 << 31) - (1 << 20))
    assert b.cache_reserve(cache, slots, first).item() == 0x7fffffff
    assert cache.held.item() == 0 and cache.refs.sum().item() == 0


@pytest.mark.parametrize("dtype", [BF, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("heads,D,P,layers,places_outer", [(8, 128, 16, 3, False), (3, 80, 32, 2, True), (1, 8, 16, 1, False), (5, 256, 64, 1, True), (2, 72, 1024, 2, False)])
def test_rows_of_a_step(b, heads, D, P, layers, places_outer, dtype):
    """Reserve, append (strided rows, all layers and single ones), compact, settle, fork: every value of the pool where it belongs."""
    rng, g = random.Random(D), torch.Generator().manual_seed(D)
    slots, slot_pages = 7, 2100 // P + 2
    pages = 5 * (1300 // P + 2)
    shape = (layers, pages, P, heads, D) if places_outer else (layers, pages, heads, P, D)
    kv = [torch.randn(shape, generator=g).to(dtype).cuda() for _ in range(2)]
    kv = [x.transpose(2, 3) if places_outer else x for x in kv]
    zeros = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    cache = b.PagedCache(kv[0], kv[1], zeros(slots, slot_pages), zeros(slots), zeros(slots), zeros(pages))
    books = Books(pages, P, slots, slot_pages)
    want = [x.cpu().clone() for x in kv]                        # [layers, pages, heads, P, D]

    def same():
        same_books(cache, books)
        for x, y in zip((cache.k, cache.v), want):
            assert torch.equal(x.cpu(), y)

    for step, (some, counts) in enumerate([([4, 1, 2], [700, 0, 33]), ([1, 4], [16, 5]), ([2, 4, 1, 0], [9, 64, 1, 65]), ([0, 4], [1, 7])]):
        assert books.reserve(some, counts) == 0
        first, total = firsts(counts), sum(counts)
        assert b.cache_reserve(cache, dev(some), dev(first)).item() == 0
        fused = torch.randn(layers, total + 1, 3 * heads, D + 8, generator=g).to(dtype)
        new = [fused[:, 1:, heads:2 * heads, 8:], fused[:, 1:, 2 * heads:, 8:]]
        on = fused.cuda()
        new_on = [on[:, 1:, heads:2 * heads, 8:], on[:, 1:, 2 * heads:, 8:]]
        if step % 2:
            for layer in range(layers):
                b.cache_append(cache, layer, new_on[0][layer], new_on[1][layer], dev(some), dev(first))
        else:
            b.cache_append(cache, 0, *new_on, dev(some), dev(first))
        for i, s in enumerate(some):
            for t in range(counts[i]):
                place = books.lens[s] + t
                for x, y in zip(want, new):
                    x[:, books.table[s][place // P], :, place % P] = y[:, first[i] + t]
        same()
        # accepted paths: none, all, some
        paths = [sorted(rng.sample(range(t), rng.choice([0, t, rng.randint(0, t)]))) for t in counts]
        width = max(len(p) for p in paths) + 1
        new_lens = b.cache_compact(cache, dev(some), dev(first), dev([p + [-9] * (width - len(p)) for p in paths]), dev([len(p) for p in paths]))
        assert new_lens.tolist() == [books.lens[s] + len(p) for s, p in zip(some, paths)]
        for s, p in zip(some, paths):
            for j, at in enumerate(p):
                a, z = books.lens[s] + at, books.lens[s] + j
                for x in want:
                    x[:, books.table[s][z // P], :, z % P] = x[:, books.table[s][a // P], :, a % P].clone()
        same()
        b.cache_set_lens(cache, dev(some), new_lens)
        books.set_lens(some, new_lens.tolist())
        same()
    children = [6, 3, 5]
    status, copies = books.fork([4, 2, 4], children)
    assert status == 0 and b.cache_fork(cache, dev([4, 2, 4]), dev(children)).item() == 0
    for a, z, rows in copies:
        for x in want:
            x[:, z, :, :rows] = x[:, a, :, :rows]
    same()


def test_paths_that_are_refused(b):
    """Paths that fall, repeat, or leave the new tokens move nothing and accept nothing; the batch's other sequences go on."""
    g = torch.Generator().manual_seed(0)
    P, n = 16, 7
    cache = b.PagedCache.empty(2, 30, 2, P, 64, n, 4, dtype=F16)
    cache.k.copy_(torch.randn(cache.k.shape, generator=g))
    cache.v.copy_(torch.randn(cache.v.shape, generator=g))
    b.cache_reserve(cache, dev(list(range(n))), dev(firsts([20] * n)))
    b.cache_set_lens(cache, dev(list(range(n))), dev([11] * n))
    b.cache_reserve(cache, dev(list(range(n))), dev(firsts([20] * n)))
    k = cache.k.clone()
    paths = [[0, 2, 4], [2, 1, 4], [1, 1, 2], [0, 5, 20], [-1, 3, 4], [3, 4, 19], [5, 6, 7]]
    accepted = [3, 3, 3, 3, 3, 3, 4]                            # the last one: more than the row is wide
    new_lens = b.cache_compact(cache, dev(list(range(n))), dev(firsts([20] * n)), dev(paths), dev(accepted))
    assert new_lens.tolist() == [14, 11, 11, 11, 11, 14, 11]
    table = cache.table.tolist()
    for s in range(n):
        if new_lens[s] > 11:
            for j, at in enumerate(paths[s]):
                k[:, table[s][(11 + j) // P], :, (11 + j) % P] = k[:, table[s][(11 + at) // P], :, (11 + at) % P].clone()
    assert torch.equal(k, cache.k)
    # a slot that does not exist, a sequence out of range, a negative count
    new_lens = b.cache_compact(cache, dev([9, 1, 2]), dev([0, 20, 10, 30]), dev([[0, 1, 2]] * 3), dev([3, 3, -1]))
    assert new_lens.tolist() == [0, 11, 11] and torch.equal(k, cache.k)


def test_long_path(b):
    """A path of more rows than are worked out at once, over many pages."""
    g = torch.Generator().manual_seed(1)
    cache = b.PagedCache.empty(1, 40, 1, 16, 8, 1, 40)
    b.cache_reserve(cache, dev([0]), dev([0, 500]))
    new = torch.randn(500, 1, 8, generator=g).to(BF).cuda()
    b.cache_append(cache, 0, new, new + 1, dev([0]), dev([0, 500]))
    path = [t for t in range(500) if t % 7 not in (0, 3)]
    assert b.cache_compact(cache, dev([0]), dev([0, 500]), dev([path]), dev([len(path)])).tolist() == [len(path)]
    pages = cache.table[0, :32].long()
    for x, y in ((cache.k, new), (cache.v, new + 1)):
        rows = x[0, pages].permute(0, 2, 1, 3).reshape(-1, 1, 8)
        assert torch.equal(rows[:len(path)], y[torch.tensor(path, device="cuda")])


def test_append_leaves_out_what_has_no_place(b):
    cache = b.PagedCache.empty(1, 4, 2, 16, 64, 2, 3)
    b.cache_reserve(cache, dev([0]), dev([0, 20]))
    cache.table[0, 1] = 99                                      # no page
    new = torch.ones(30, 2, 64, dtype=BF, device="cuda")
    b.cache_append(cache, 0, new, new, dev([0, 5]), dev([0, 20, 30]))
    assert cache.k.sum().item() == 16 * 2 * 64 and (cache.k[0, cache.table[0, 0].item()] == 1).all()
    b.cache_append(cache, 0, 2 * new, 2 * new, dev([0, 1]), dev([0, 31, 30]))      # neither range lies in the rows
    assert cache.k.max().item() == 1 and cache.v.sum().item() == 16 * 2 * 64


def test_a_step_goes_on_after_a_refused_reserve(b):
    """The report is read later: until then the calls leave out the sequences that do not hold their tokens' pages, and nobody's rows are touched."""
    cache = b.PagedCache.empty(2, 4, 2, 16, 64, 3, 4)
    rows = lambda n, x: torch.full((2, n, 2, 64), x, dtype=BF, device="cuda")  # noqa: E731
    assert b.cache_reserve(cache, dev([0, 1]), dev([0, 30, 46])).item() == 0
    b.cache_append(cache, 0, rows(46, 1.0), rows(46, 2.0), dev([0, 1]), dev([0, 30, 46]))
    b.cache_set_lens(cache, dev([0, 1]), dev([30, 16]))
    books = [x.clone() for x in (cache.table, cache.held, cache.lens, cache.refs)]
    k, v = cache.k.clone(), cache.v.clone()
    # slot 1 and slot 2 need three pages, one is free; slot 0's two tokens have room
    slots, first = dev([1, 0, 2]), dev([0, 17, 19, 28])
    report = b.cache_reserve(cache, slots, first)
    b.cache_append(cache, 0, rows(28, 5.0), rows(28, 6.0), slots, first)
    page = books[0][0, 1].item()
    k[:, page, :, 14:], v[:, page, :, 14:] = 5.0, 6.0
    assert torch.equal(cache.k, k) and torch.equal(cache.v, v)
    q = torch.randn(28, 4, 64, device="cuda").to(BF)
    out, lse = torch.full_like(q, 100.0), torch.full((28, 4), 1e9, device="cuda")
    b.tree_attention(cache, 0, q, slots, first, out=out, lse=lse)
    assert (out[:17] == 100).all() and (out[19:] == 100).all() and (lse[:17] == 1e9).all() and (lse[19:] == 1e9).all()
    assert (out[17:19] != 100).all() and (lse[17:19] != 1e9).all()
    path = torch.tensor([[1, 2], [1, 0], [0, 1]], dtype=torch.int32, device="cuda")
    new_lens = b.cache_compact(cache, slots, first, path, dev([2, 1, 2]))
    assert new_lens.tolist() == [16, 31, 0] and report.item() == 2
    k[:, page, :, 14], v[:, page, :, 14] = k[:, page, :, 15], v[:, page, :, 15]
    assert torch.equal(cache.k, k) and torch.equal(cache.v, v)
    assert all(torch.equal(x, y) for x, y in zip((cache.held, cache.lens, cache.refs), books[1:]))
    held = torch.arange(cache.table.shape[1], device="cuda")[None] < cache.held[:, None]      # (entries past them mean nothing)
    assert torch.equal(cache.table[held], books[0][held])


@pytest.mark.parametrize("counts", [[1], [8] * 64, [64, 1, 63], [65, 0, 128], [300, 1000], [4096]], ids=str)
def test_tree_masks(b, counts):
    rng = random.Random(sum(counts))
    kinds = [lambda t: t - 1, lambda t: -1, lambda t: rng.randint(-1, t - 1) if t else -1, lambda t: (t - 1) // 2 if t else -1]
    parents = [[kinds[(i + len(counts)) % 4](t) for t in range(n)] for i, n in enumerate(counts)]
    words = -(-max(counts) // 64)
    want = torch.cat([mask_words(ancestor_sets(p), words) for p in parents])
    got = b.tree_mask(dev(sum(parents, [])), dev(firsts(counts)), words)
    assert torch.equal(got.cpu(), want)
    if words > 1:                                               # too few words for the longest: its rows are empty
        few = b.tree_mask(dev(sum(parents, [])), dev(firsts(counts)), words - 1).cpu()
        at = 0
        for n in counts:
            assert torch.equal(few[at:at + n], want[at:at + n, :words - 1] if n <= 64 * (words - 1) else torch.zeros(n, words - 1, dtype=torch.int64))
            at += n


def test_parents_out_of_range(b):
    """A parent that is not an earlier token counts as the committed context."""
    got = b.tree_mask(dev([0, 5, -7, 2, 1 << 30]), dev([0, 5]), 1).view(-1).tolist()
    assert got == [1, 2, 4, 12, 16]
    out = torch.full((5, 1), 77, dtype=torch.int64, device="cuda")
    b.tree_mask(dev([-1, 0, 1, 2, 3]), dev([0, 2, 6]), 1, out=out)     # the second range leaves the rows: left out
    assert out.view(-1).tolist() == [1, 3, 77, 77, 77]


def test_forks_of_a_running_graph(b):
    """The calls of a step in a graph, replayed with the books they left and with others."""
    P = 16
    cache = b.PagedCache.empty(2, 64, 2, P, 64, 6, 8)
    books = Books(64, P, 6, 8)
    slots, first, report = dev([0, 1]), dev(firsts([20, 20])), dev([7])
    new = torch.randn(2, 40, 2, 64, device="cuda").to(BF)
    path, accepted, lens = dev([[0, 2, 3], [1, 5, 19]]), dev([3, 3]), dev([0, 0])

    def step():
        b.cache_reserve(cache, slots, first, report=report)
        b.cache_append(cache, 0, new, new, slots, first)
        b.cache_compact(cache, slots, first, path, accepted, new_lens=lens)
        b.cache_set_lens(cache, slots, lens)

    def on_lists():
        assert books.reserve([0, 1], [20, 20]) == 0
        books.set_lens([0, 1], [books.lens[0] + 3, books.lens[1] + 3])

    step()
    on_lists()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(6):
        graph.replay()
        on_lists()
        torch.cuda.synchronize()
        same_books(cache, books)
        assert report.item() == 0
        if i == 2:
            assert books.fork([0], [4])[0] == 0 and b.cache_fork(cache, dev([0]), dev([4])).item() == 0
            same_books(cache, books)

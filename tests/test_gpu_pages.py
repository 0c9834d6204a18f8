"""The cache's pages (pages_grow, _append, _fork, _free, _compact, _copy) against a plain
book in Python: every number and every copied bit has to be equal (needs a GB300)."""
import random

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def sv():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__ as g
    g.build()
    from paper_2606_10820_gb300 import serving
    return serving


class Plain:
    """The book's definition: lists, one request after another."""

    def __init__(self, n_pages, slots, width, page):
        self.ref, self.lens, self.page = [0] * n_pages, [0] * slots, page
        self.table = [[-1] * width for _ in range(slots)]

    def pages(self, n):
        return -(-n // self.page)

    def take(self, n):
        free = [p for p, r in enumerate(self.ref) if r == 0]
        return free[:n] if len(free) >= n else None

    def grow(self, slots, new):
        want = [(s, c) for s, x in zip(slots, new) for c in range(self.pages(self.lens[s]), self.pages(x))]
        got = self.take(len(want))
        if got is None:
            return False
        for (s, c), p in zip(want, got):
            self.table[s][c], self.ref[p] = p, 1
        for s, x in zip(slots, new):
            self.lens[s] = x
        return True

    def free(self, slots):
        for s in slots:
            for p in self.table[s]:
                if p >= 0:
                    self.ref[p] -= 1
            self.table[s], self.lens[s] = [-1] * len(self.table[s]), 0

    def fork(self, src, dst):
        """The copies (old page, new page), or None."""
        part = [s for s in src if self.lens[s] % self.page]
        got = self.take(len(part))
        if got is None:
            return None
        moves, row = [], 0
        for s, d in zip(src, dst):
            full = self.lens[s] // self.page
            for c in range(full):
                self.table[d][c] = self.table[s][c]
                self.ref[self.table[s][c]] += 1
            if self.lens[s] % self.page:
                self.table[d][full] = got[row]
                self.ref[got[row]] = 1
                moves.append((self.table[s][full], got[row]))
                row += 1
            self.lens[d] = self.lens[s]
        return moves

    def compact(self):
        live = [p for p, r in enumerate(self.ref) if r]
        L = len(live)
        src, dst = [p for p in live if p >= L], [p for p in range(L) if not self.ref[p]]
        to = dict(zip(src, dst))
        for s, d in to.items():
            self.ref[d], self.ref[s] = self.ref[s], 0
        self.table = [[to.get(p, p) for p in row] for row in self.table]
        return L, list(to.items())


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def same(book, plain):
    ref, table, lens = book
    assert ref.tolist() == plain.ref
    assert lens.tolist() == plain.lens
    assert table.tolist() == plain.table


def new_pool(layers, n_pages, Hkv, page, hd, seed=0, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(layers, n_pages, 2, Hkv, page, hd, generator=g, device="cuda").to(dtype)


# a book of one CTA, and ones whose teams are clusters (many pages; many entries)
@pytest.mark.parametrize("n_pages,slots,width,page,layers,Hkv,hd", [
    (40, 9, 7, 16, 2, 1, 64), (1, 2, 1, 16, 1, 1, 8), (333, 60, 12, 8, 3, 2, 64), (17001, 70, 40, 16, 1, 1, 8),
    (40000, 300, 130, 16, 1, 1, 8), (700, 1500, 30, 1, 1, 1, 8)])
@pytest.mark.parametrize("seed", range(2))
def test_random_histories(sv, n_pages, slots, width, page, layers, Hkv, hd, seed):
    """Grow, fork, free and compact at random, the pool's pages following."""
    rng = random.Random(seed * 1000 + n_pages)
    plain, book = Plain(n_pages, slots, width, page), sv.new_book(n_pages, slots, width)
    pool = new_pool(layers, n_pages, Hkv, page, hd, seed)
    want = pool.clone()

    def follow(moves):
        if moves:
            s, d = (torch.tensor(x, device="cuda") for x in zip(*moves))
            want[:, d] = want[:, s]

    for step in range(14):
        kind = rng.choice(["grow", "grow", "fork", "fork", "free", "compact"]) if step > 1 else "grow"
        used = [s for s in range(slots) if plain.lens[s]]
        empty = [s for s in range(slots) if not plain.lens[s]]
        if kind == "grow":
            pick = rng.sample(range(slots), rng.randint(1, slots))
            room = max(1, n_pages * page // (2 * slots))
            new = [min(width * page, plain.lens[s] + rng.randint(0, room)) for s in pick]
            before = (list(plain.ref), list(plain.lens))
            ok = plain.grow(pick, new)
            sv.pages_grow(*book, i32(pick), i32(new), page=page)
            if not ok:
                assert before == (plain.ref, plain.lens)
                with pytest.raises(Exception, match="flags 32"):
                    sv.status()
        elif kind == "fork" and used and empty:
            dst = rng.sample(empty, rng.randint(1, len(empty)))
            src = [rng.choice(used) for _ in dst]
            moves = plain.fork(src, dst)
            sv.pages_fork(pool, *book, i32(src), i32(dst))
            if moves is None:
                with pytest.raises(Exception, match="flags 32"):
                    sv.status()
            follow(moves)
        elif kind == "free" and used:
            pick = rng.sample(used, rng.randint(1, len(used)))
            plain.free(pick)
            sv.pages_free(*book, i32(pick), page=page)
        elif kind == "compact":
            L, moves = plain.compact()
            live = i32([-1])
            sv.pages_compact(pool, book[0], book[1], live=live)
            assert live.item() == L
            follow(moves)
        sv.status()
        same(book, plain)
        assert torch.equal(pool, want)


@pytest.mark.parametrize("page,Hkv,hd,dtype", [(16, 2, 64, torch.bfloat16), (16, 3, 128, torch.float16), (48, 1, 8, torch.bfloat16)])
@pytest.mark.parametrize("fused", [False, True])
def test_append(sv, page, Hkv, hd, dtype, fused):
    old, new = [0, 5, 16, 40, 0, 15], [1, 30, 16, 0, 100, 1]
    slots = [4, 0, 6, 2, 5, 1]
    book = sv.new_book(60, 7, 12)
    sv.pages_grow(*book, i32(slots), i32(old), page=page)
    lens = [a + b for a, b in zip(old, new)]
    sv.pages_grow(*book, i32(slots), i32(lens), page=page)
    pool = new_pool(1, 60, Hkv, page, hd, 1, dtype)[0]
    want, T = pool.clone(), sum(new)
    g = torch.Generator(device="cuda").manual_seed(3)
    if fused:
        _, k, v = torch.randn(T, 4 + 2 * Hkv, hd, generator=g, device="cuda").to(dtype).split([4, Hkv, Hkv], 1)
    else:
        k, v = (torch.randn(T, Hkv, hd, generator=g, device="cuda").to(dtype) for _ in range(2))
    starts = [0]
    for x in new:
        starts.append(starts[-1] + x)
    table = book[1].tolist()
    for i, s in enumerate(slots):
        for j in range(new[i]):
            pos = old[i] + j
            p = table[s][pos // page]
            want[p, 0, :, pos % page] = k[starts[i] + j]
            want[p, 1, :, pos % page] = v[starts[i] + j]
    sv.pages_append(pool, k, v, i32(starts), book[1], book[2], i32(slots))
    sv.status()
    assert torch.equal(pool, want)


@pytest.mark.parametrize("layers,Hkv,hd,n", [(1, 1, 8, 5), (3, 2, 64, 17), (2, 8, 128, 300), (5, 3, 72, 1)])
def test_copy(sv, layers, Hkv, hd, n):
    pool = new_pool(layers, 700, Hkv, 16, hd, 2)
    want = pool.clone()
    ids = torch.randperm(700, device="cuda")
    src, dst = ids[torch.randint(0, 300, (n,), device="cuda")], ids[300: 300 + n]
    want[:, dst] = want[:, src]
    sv.pages_copy(pool, src.int(), dst.int())
    sv.status()
    assert torch.equal(pool, want)


def test_copy_past_32_bits(sv):
    pool = torch.zeros(2, 9000, 262144, device="cuda", dtype=torch.uint8)       # 4.7 GB
    pool[:, 8999] = torch.arange(2, device="cuda", dtype=torch.uint8)[:, None] + 7
    sv.pages_copy(pool, i32([8999]), i32([4]))
    assert (pool[0, 4] == 7).all() and (pool[1, 4] == 8).all() and (pool[:, 3] == 0).all() and (pool[:, 5] == 0).all()


def test_append_past_32_bits(sv):
    """Pages past 2^32 bytes of a layer."""
    pool = torch.zeros(5000, 2, 8, 64, 1024, device="cuda", dtype=torch.float16)      # 10.5 GB
    table = i32([[4999, 2], [4998, 7]])
    k, v = (torch.randn(130, 8, 1024, device="cuda").half() for _ in range(2))
    sv.pages_append(pool, k, v, i32([0, 70, 130]), table, i32([70, 60]), i32([0, 1]))
    sv.status()
    assert torch.equal(pool[4999, 0].transpose(0, 1), k[:64]) and torch.equal(pool[2, 1, :, :6].transpose(0, 1), v[64:70])
    assert torch.equal(pool[4998, 1, :, :60].transpose(0, 1), v[70:]) and (pool[7] == 0).all() and (pool[2, :, :, 6:] == 0).all()


def test_refused_calls_change_nothing(sv):
    """What the device finds wrong with a call leaves the book and the pool as they were."""
    n_pages, slots, width = 20, 6, 4
    plain, book = Plain(n_pages, slots, width, 16), sv.new_book(n_pages, slots, width)
    plain.grow([0, 1, 2], [40, 16, 64])
    sv.pages_grow(*book, i32([0, 1, 2]), i32([40, 16, 64]))
    pool = new_pool(2, n_pages, 1, 16, 8)
    want = pool.clone()
    ref, table, lens = book

    def refused(call, bits):
        keep = [x.clone() for x in book]
        call()
        with pytest.raises(Exception, match=f"flags {bits}$"):
            sv.status()
        assert all(torch.equal(a, b) for a, b in zip(keep, book)) and torch.equal(pool, want)
        sv.status()

    for bad in ([0, 0], [6, 1], [-1, 1]):
        refused(lambda: sv.pages_grow(*book, i32(bad), i32([64, 64])), 8)
        refused(lambda: sv.pages_free(*book, i32(bad)), 8)
        refused(lambda: sv.pages_fork(pool, *book, i32([0, 0]), i32(bad)), 8)
    refused(lambda: sv.pages_grow(*book, i32([0, 1]), i32([39, 64])), 8)         # shorter than it is
    refused(lambda: sv.pages_grow(*book, i32([0]), i32([65])), 8)                # past the table
    refused(lambda: sv.pages_grow(*book, i32([3, 4, 5, 0]), i32([64, 64, 64, 64])), 32)
    refused(lambda: sv.pages_fork(pool, *book, i32([0]), i32([1])), 8)           # not empty
    refused(lambda: sv.pages_fork(pool, *book, i32([3, 0]), i32([4, 3])), 8)     # a source that is a destination
    refused(lambda: sv.pages_fork(pool, *book, i32([7]), i32([4])), 8)
    same(book, plain)
    # tables that contradict the references
    for bad in (-2, 20, 1 << 30, 19):
        table[1, 0] = bad
        refused(lambda: sv.pages_free(*book, i32([0, 1, 2])), 2)
        refused(lambda: sv.pages_fork(pool, *book, i32([0, 1]), i32([3, 4])), 2)
        refused(lambda: sv.pages_compact(pool, ref, table), 2)
    table[1, 0] = plain.table[1][0]
    ref[5] = -1
    refused(lambda: sv.pages_compact(pool, ref, table), 2)
    ref[5] = plain.ref[5]
    lens[4] = -3
    refused(lambda: sv.pages_fork(pool, *book, i32([4]), i32([3])), 8)
    lens[4] = 0
    same(book, plain)


def test_bad_appends_and_copies_are_left_out(sv):
    book = sv.new_book(10, 3, 2)
    sv.pages_grow(*book, i32([0, 1]), i32([20, 3]))
    pool = new_pool(1, 10, 1, 16, 8)[0]
    want = pool.clone()
    k = torch.randn(6, 1, 8, device="cuda").bfloat16()
    # slot 7 does not exist; slot 1 has 3 tokens, not 4 new ones
    sv.pages_append(pool, k, k, i32([0, 1, 5, 6]), book[1], book[2], i32([7, 1, 0]))
    with pytest.raises(Exception, match="flags 8$"):
        sv.status()
    p, p0 = book[1][1, 0].item(), book[1][0, 1].item()
    want[p, 0, 0, :3] = want[p, 1, 0, :3] = k[2:5, 0]
    want[p0, 0, 0, 3] = want[p0, 1, 0, 3] = k[5, 0]
    assert torch.equal(pool, want)
    five = pool[None].clone()
    sv.pages_copy(five, i32([0, 10, -1, 3]), i32([9, 1, 2, 12]))
    with pytest.raises(Exception, match="flags 2$"):
        sv.status()
    want[9] = want[0]
    assert torch.equal(five[0], want)


def test_captured(sv):
    """A fork and its end in a CUDA graph, replayed on new lengths."""
    book = sv.new_book(64, 4, 8)
    pool = new_pool(2, 64, 1, 16, 8)
    sv.pages_grow(*book, i32([0]), i32([20]))
    src, dst = i32([0, 0]), i32([1, 2])
    sv.pages_fork(pool, *book, src, dst)
    sv.pages_free(*book, dst)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        sv.pages_fork(pool, *book, src, dst)
    plain = Plain(64, 4, 8, 16)
    plain.grow([0], [20])
    sv.pages_grow(*book, i32([0]), i32([77]))
    plain.grow([0], [77])
    want = pool.clone()
    for a, b in plain.fork([0, 0], [1, 2]):
        want[:, b] = want[:, a]
    graph.replay()
    torch.cuda.synchronize()
    same(book, plain)
    assert torch.equal(pool, want)


def test_refusals(sv):
    from paper_2606_10820_gb300.kforcing import KfError
    book, pool = sv.new_book(10, 3, 2), new_pool(1, 10, 1, 16, 8)
    k = torch.zeros(1, 1, 8, device="cuda", dtype=torch.bfloat16)
    for call in (lambda: sv.pages_grow(*book, i32([0, 1, 2, 0]), i32([1, 1, 1, 1])), lambda: sv.pages_grow(*book, i32([0]), i32([1]), page=0),
                 lambda: sv.pages_free(*book, i32([0, 1, 2, 0])), lambda: sv.pages_copy(new_pool(1, 10, 1, 1, 6), i32([0]), i32([1])),
                 lambda: sv.pages_copy(pool, i32([0] * 11), i32([1] * 11)), lambda: sv.pages_compact(new_pool(1, 10, 1, 1, 6), *book[:2])):
        with pytest.raises(KfError):
            call()
    for call in (lambda: sv.pages_grow(book[0].long(), *book[1:], i32([0]), i32([1])), lambda: sv.pages_free(*book, torch.tensor([0], device="cuda")),
                 lambda: sv.pages_fork(pool[0], *book, i32([0]), i32([1])), lambda: sv.pages_compact(pool[:, :5], book[0], book[1]),
                 lambda: sv.pages_append(pool[0], k, k[:, :, :4], i32([0, 1]), book[1], book[2], i32([0])),
                 lambda: sv.pages_append(pool[0], k.float(), k.float(), i32([0, 1]), book[1], book[2], i32([0])),
                 lambda: sv.pages_append(pool[0], k, k, i32([0]), book[1], book[2], i32([0]))):
        with pytest.raises(ValueError):
            call()
    sv.status()

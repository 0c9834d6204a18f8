"""The book's kernels (grow, free, fork: one CTA) on the CPU, at lengths near the end of their range
and with tables that contradict a call; what lies around the arrays has to stay as it was."""
import ctypes

import numpy as np
import pytest

import block_on_host as host

BAD_PAGE, BAD_ROW, NO_PAGES = 2, 8, 32
PAD = 64
DRIVER = """
using namespace kf;
extern "C" {
#define TEAM(...) block::run(kThreads, std::vector<int>(order, order + kWarps), 0, [=] { __VA_ARGS__; })
static Work layout(int32_t* p, int n_pages, int slots, int n) {
  Work w;
  w.count = p;
  w.mark = p + 64;
  w.off = w.mark + slots;
  w.src = w.off + n;
  w.dst = w.src + n_pages;
  w.to = w.dst + n_pages;
  return w;
}
void grow(int n, const int* which, const int* lens, int32_t* ref, int n_pages, int32_t* table, int slots, int width, int32_t* len, int page,
          int32_t* work, int* err, const int* order) {
  TEAM(k_grow<1>(Book{ref, table, len, n_pages, slots, width, page}, n, which, lens, layout(work, n_pages, slots, n), err));
}
void fork_(int n, const int* src, const int* dst, int32_t* ref, int n_pages, int32_t* table, int slots, int width, int32_t* len, int page,
           int32_t* work, int* err, const int* order) {
  TEAM(k_fork<1>(Book{ref, table, len, n_pages, slots, width, page}, n, src, dst, layout(work, n_pages, slots, n), err));
}
void free_(int n, const int* which, int32_t* ref, int n_pages, int32_t* table, int slots, int width, int32_t* len, int page, int32_t* work,
           int* err, const int* order) {
  TEAM(k_free<1>(Book{ref, table, len, n_pages, slots, width, page}, n, which, layout(work, n_pages, slots, n), err));
}
}
"""
SHIM = """
namespace cooperative_groups {
struct Cluster { void sync() const {} template <typename T> T* map_shared_rank(T* p, int) const { return p; } };
static inline Cluster this_cluster() { return {}; }
}
namespace cg = cooperative_groups;
namespace kf {
static inline int ceil_div(int a, int b) { return (a + b - 1) / b; }
static inline int round_up(int a, int b) { return ceil_div(a, b) * b; }
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    source = SHIM + host.between("kf_pages.cu", "constexpr int kThreads = 1024", "// page src[i] to dst[i] in every layer") + "}\n"
    return host.load(str(tmp_path_factory.mktemp("pages")), "pages", source, DRIVER)


class Book:
    def __init__(self, lib, n_pages, slots, width, page):
        self.lib, self.shape, self.page = lib, (n_pages, slots, width), page
        self.whole = [np.full(n + 2 * PAD, -77, np.int32) for n in (n_pages, slots * width, slots)]
        self.ref, self.table, self.lens = (x[PAD:-PAD] for x in self.whole)
        self.ref[:], self.table[:], self.lens[:] = 0, -1, 0
        self.table = self.table.reshape(slots, width)

    def call(self, name, first, second=None, order=0):
        n_pages, slots, width = self.shape
        ints = lambda x: (ctypes.c_int32 * max(1, len(x)))(*x)  # noqa: E731
        p = lambda x: x.ctypes.data_as(ctypes.c_void_p)          # noqa: E731
        work = np.full(64 + slots + len(first) + 3 * n_pages + 2 * PAD, -77, np.int32)
        err = ctypes.c_int(0)
        lists = [ints(first)] + ([] if second is None else [ints(second)])
        getattr(self.lib, name)(len(first), *lists, p(self.ref), n_pages, p(self.table), slots, width, p(self.lens), self.page,
                                ctypes.c_void_p(work.ctypes.data + 4 * PAD), ctypes.byref(err), host.orders()[order])
        for x in self.whole + [work]:
            assert (x[:PAD] == -77).all() and (x[-PAD:] == -77).all()
        return err.value

    def refused(self, bits, *call, **kw):
        keep = [x.copy() for x in self.whole]
        assert self.call(*call, **kw) == bits
        assert all((a == b).all() for a, b in zip(keep, self.whole))


@pytest.mark.parametrize("order", range(3))
def test_ordinary_calls(lib, order):
    b = Book(lib, 40, 6, 7, 16)
    assert b.call("grow", [0, 3, 1], [40, 112, 16], order=order) == 0
    assert b.lens.tolist() == [40, 16, 0, 112, 0, 0] and (b.ref == 1).sum() == 11
    assert b.table[0].tolist() == [0, 1, 2, -1, -1, -1, -1] and b.table[3].tolist() == list(range(3, 10)) and b.table[1, 0] == 10
    assert b.call("fork_", [0, 0], [2, 5], order=order) == 0
    assert b.table[2].tolist() == [0, 1, 11, -1, -1, -1, -1] and b.table[5].tolist() == [0, 1, 12, -1, -1, -1, -1] and b.ref[:2].tolist() == [3, 3]
    assert b.call("free_", [0, 5], order=order) == 0
    assert b.ref[:3].tolist() == [1, 1, 0] and b.ref[12] == 0 and (b.table[[0, 5]] == -1).all() and b.lens[[0, 5]].tolist() == [0, 0]
    b.refused(BAD_ROW, "grow", [4, 4], [16, 16], order=order)
    b.refused(BAD_ROW, "grow", [3], [100], order=order)
    b.refused(NO_PAGES, "grow", [0, 1, 2, 4, 5], [112] * 5, order=order)


@pytest.mark.parametrize("page,width", [(1000000, 2147), (1048575, 2048), (1 << 20, 2047)])
def test_lengths_at_the_end_of_their_range(lib, page, width):
    """Lengths within a page of 2^31: their pages are counted, and missing ones refused."""
    length = width * page
    b = Book(lib, width + 3, 3, width, page)
    b.refused(NO_PAGES, "grow", [0, 1], [length, length])
    assert b.call("grow", [2, 1], [1, length]) == 0
    assert (b.ref[: width + 1] == 1).all() and (b.ref[width + 1:] == 0).all() and b.lens.tolist() == [0, length, 1]
    assert b.table[1].tolist() == list(range(1, width + 1)) and b.table[2, 0] == 0
    # a length whose pages the table does not have
    assert b.call("free_", [2]) == 0
    b.lens[0] = length
    for p in (-1, width + 3, 1 << 30):
        b.table[0] = p
        b.refused(BAD_PAGE, "fork_", [0], [2])
    b.table[0] = b.table[1]
    assert b.call("fork_", [0], [2]) == 0
    assert (b.table[2] == b.table[1]).all() and b.lens[2] == length and (b.ref[1: width + 1] == 2).all()


@pytest.mark.parametrize("order", range(3))
def test_grow_refuses_columns_that_hold_a_page(lib, order):
    """A length lowered by hand leaves pages in the row; filling their columns would lose them."""
    b = Book(lib, 400, 5, 120, 16)
    assert b.call("grow", [0, 1, 3], [100, 16, 1000], order=order) == 0
    b.lens[0] = 70                                     # (of 7 pages: 5 are left in use)
    b.refused(BAD_PAGE, "grow", [2, 0, 1], [16, 81, 17], order=order)
    b.refused(BAD_PAGE, "grow", [2, 0], [16, 1900], order=order)
    b.lens[0] = 100
    b.table[1, 1] = 399                                # a page that nobody holds
    b.refused(BAD_PAGE, "grow", [1], [17], order=order)
    b.table[1, 1], b.table[1, 60] = -1, -5
    b.refused(BAD_PAGE, "grow", [0, 1, 2], [101, 1600, 5], order=order)
    assert b.call("grow", [0, 1, 2], [101, 900, 5], order=order) == 0
    b.refused(NO_PAGES, "grow", [4, 2, 3], [1920] * 3, order=order)


@pytest.mark.parametrize("n", [40, 1500])
def test_grow_of_many_slots(lib, n):
    """More requests than a warp holds at once, with and without new pages."""
    rng = np.random.default_rng(n)
    b = Book(lib, 12 * n, n, 9, 4)
    want = np.full((n, 9), -1, np.int32)
    lens, used = np.zeros(n, np.int32), 0
    for step in range(3):
        which = rng.permutation(n)[: n - step]
        new = np.minimum(36, lens[which] + rng.integers(0, [2, 15, 5][step], len(which)))
        for s, x in zip(which, new):
            for c in range(-(-lens[s] // 4), -(-x // 4)):
                want[s, c] = used
                used += 1
            lens[s] = x
        assert b.call("grow", which.tolist(), new.tolist(), order=step) == 0
        assert (b.table == want).all() and (b.lens == lens).all() and (b.ref[:used] == 1).all() and (b.ref[used:] == 0).all()

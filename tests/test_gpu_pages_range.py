"""The cache's pages at the end of the lengths' range, and rows that hold pages past their length
(needs a GB300)."""
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


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def test_lengths_within_a_page_of_2_31(sv):
    page, width = 1000000, 2147
    length = page * width
    ref, table, lens = book = sv.new_book(width + 3, 3, width)
    sv.pages_grow(*book, i32([0, 1]), i32([length, length]), page=page)
    with pytest.raises(Exception, match="flags 32$"):
        sv.status()
    assert (ref == 0).all() and (table == -1).all() and (lens == 0).all()
    sv.pages_grow(*book, i32([1]), i32([length]), page=page)
    sv.status()
    assert torch.equal(table[1], torch.arange(width, dtype=torch.int32, device="cuda")) and lens.tolist() == [0, length, 0]
    assert (ref[:width] == 1).all() and (ref[width:] == 0).all()
    pool = torch.empty(1, width + 3, 2, 1, page, 1, dtype=torch.int8, device="cuda")
    lens[0] = length
    for p in (-1, width + 3, 1 << 30):
        table[0] = p
        keep = [x.clone() for x in book]
        sv.pages_fork(pool, *book, i32([0]), i32([2]))
        with pytest.raises(Exception, match="flags 2$"):
            sv.status()
        assert all(torch.equal(a, b) for a, b in zip(keep, book))
    sv.pages_fork(pool, *book, i32([1]), i32([2]))
    sv.status()
    assert torch.equal(table[2], table[1]) and (ref[:width] == 2).all() and lens[2].item() == length


@pytest.mark.parametrize("n_pages", [400, 20000])      # a CTA, and a cluster
def test_grow_refuses_columns_that_hold_a_page(sv, n_pages):
    ref, table, lens = book = sv.new_book(n_pages, 5, 120)
    sv.pages_grow(*book, i32([0, 1, 3]), i32([100, 16, 1000]))
    sv.status()
    lens[0] = 70
    for slots, new in (([2, 0, 1], [16, 81, 17]), ([2, 0], [16, 1900])):
        keep = [x.clone() for x in book]
        sv.pages_grow(*book, i32(slots), i32(new))
        with pytest.raises(Exception, match="flags 2$"):
            sv.status()
        assert all(torch.equal(a, b) for a, b in zip(keep, book))
    lens[0] = 100
    sv.pages_grow(*book, i32([2, 0, 1]), i32([16, 113, 17]))
    sv.status()
    assert table[2, 0].item() == 71 and table[0, 7].item() == 72 and table[1, 1].item() == 73 and lens.tolist() == [113, 17, 16, 1000, 0]

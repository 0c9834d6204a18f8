"""The serving operators on tensors as torch hands them out: strides of dimensions of one, tensors that require
gradients, versions of what a call changes (needs a GB300)."""
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


def test_a_pool_of_one_page_seen_through_a_transpose(sv):
    """The stride of a dimension of one page says nothing about the page's size."""
    layers = 20000
    pool = torch.zeros(1, layers, 2, 2, 16, 512, dtype=torch.bfloat16, device="cuda").transpose(0, 1)       # 1.3 GB
    assert pool.is_contiguous() and pool.stride(1) != pool[0].numel()
    book = sv.new_book(1, 2, 1)
    sv.pages_grow(*book, i32([1]), i32([16]))
    live = i32([-1])
    sv.pages_compact(pool, book[0], book[1], live=live)
    sv.pages_fork(pool, *book, i32([1]), i32([0]))
    sv.status()
    assert live.item() == 1 and book[0].item() == 2

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


def test_strides_of_dimensions_of_one(sv):
    """One token, one head, one sequence, one row: the strides of such dimensions are not asked about."""
    def odd(*shape):
        """shape, all of its dimensions but the last of one: strides that are no multiples of 8."""
        x = torch.randn(3, 197, 1, 1, device="cuda").bfloat16()[:1, :shape[-1]]
        return x.permute(0, 2, 3, 1)[(0,) * (4 - len(shape))]

    q, k, v = odd(1, 1, 64), odd(1, 1, 64), odd(1, 1, 64)
    assert q.shape == (1, 1, 64) and any(s % 8 for s in q.stride()[:2])
    out = torch.zeros(3, 67, 1, device="cuda", dtype=q.dtype)[:1, :64].permute(0, 2, 1)
    assert torch.equal(sv.prompt_attention(q, k, v, i32([0, 1]), 1, out=out), v)
    book = sv.new_book(3, 1, 2)
    sv.pages_grow(*book, i32([0]), i32([1]))
    pool = torch.full((3, 2, 1, 16, 64), 5.0, device="cuda", dtype=q.dtype)
    sv.pages_append(pool, k, v, i32([0, 1]), book[1], book[2], i32([0]))
    assert torch.equal(pool[0, 0, 0, 0], k[0, 0]) and torch.equal(pool[0, 1, 0, 0], v[0, 0]) and (pool[1:] == 5).all()
    q4 = odd(1, 1, 1, 64)
    assert q4.shape == (1, 1, 1, 64)
    assert torch.equal(sv.paged_attention(q4, pool, book[1], book[2])[0, 0], v[0])
    sv.status()

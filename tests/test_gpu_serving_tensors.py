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


def test_no_gradient_is_dropped_silently(sv):
    """An operator without a backward pass refuses what would need one; without grad mode it runs."""
    q, k, v = (torch.randn(5, h, 64, device="cuda").bfloat16() for h in (2, 1, 1))
    starts = i32([0, 5])
    pool, table, lens = torch.zeros(4, 2, 1, 16, 64, device="cuda", dtype=q.dtype), i32([[0]]), i32([5])
    x, tok = torch.randn(4, 100, device="cuda"), torch.arange(4, device="cuda")
    g = torch.randn(4, device="cuda")
    book = sv.new_book(4, 2, 1)
    wants = lambda t: t.detach().clone().requires_grad_()  # noqa: E731
    calls = [lambda: sv.prompt_attention(wants(q), k, v, starts, 5), lambda: sv.prompt_attention(q, wants(k), v, starts, 5),
             lambda: sv.prompt_attention(q, k, wants(v), starts, 5), lambda: sv.prompt_attention(q, k, v, starts, 5, out=wants(q)),
             lambda: sv.paged_attention(wants(q[None, -1:]), pool, table, lens), lambda: sv.paged_attention(q[None, -1:], wants(pool), table, lens),
             lambda: sv.paged_attention(q[None, -1:], pool, table, lens, out=wants(q[None, -1:])),
             lambda: sv.pages_append(pool, wants(k), v, starts, table, lens, i32([0])), lambda: sv.pages_append(pool, k, wants(v), starts, table, lens, i32([0])),
             lambda: sv.pages_append(wants(pool), k, v, starts, table, lens, i32([0])), lambda: sv.pages_copy(wants(pool[None]), i32([0]), i32([1])),
             lambda: sv.pages_fork(wants(pool[None]), *book, i32([0]), i32([1])), lambda: sv.pages_compact(wants(pool[None]), *book[:2]),
             lambda: sv.token_scores(wants(x), tok), lambda: sv.token_scores_grad(x, tok, wants(g)), lambda: sv.token_scores_grad(x, tok, g, wants(g)),
             lambda: sv.token_scores_grad(x, tok, g, out=wants(x))]
    for call in calls:
        with pytest.raises(ValueError, match="gradient"):
            call()
        with torch.no_grad():
            call()
    sv.status()
    # the gradient call is one's own backward pass: its logits may require one
    h, w = torch.randn(4, 32, device="cuda"), torch.randn(100, 32, device="cuda", requires_grad=True)
    logits = h @ w.T
    out = sv.token_scores_grad(logits, tok, torch.full((4,), -0.25, device="cuda"))
    logits.backward(out["grad"])
    ref = w.detach().clone().requires_grad_()
    torch.nn.functional.cross_entropy(h @ ref.T, tok).backward()
    assert not out["logp"].requires_grad and torch.allclose(w.grad, ref.grad, atol=1e-4)


def test_versions_of_what_a_call_changes(sv):
    """Autograd sees that a tensor it has saved was written."""
    q, k, v = (torch.randn(5, h, 64, device="cuda").bfloat16() for h in (2, 1, 1))
    starts, slots = i32([0, 5]), i32([0])
    ref, table, lens = book = sv.new_book(4, 2, 1)
    pool = torch.zeros(2, 4, 2, 1, 16, 64, device="cuda", dtype=q.dtype)
    x, tok = torch.randn(4, 100, device="cuda"), torch.arange(4, device="cuda")
    live, out, out4 = i32([0]), torch.empty_like(q), torch.empty_like(q[None, -1:])

    def changed(call, *tensors, same=()):
        before = [t._version for t in tensors + tuple(same)]
        call()
        after = [t._version for t in tensors + tuple(same)]
        assert all(b > a for a, b in zip(before, after[:len(tensors)])) and after[len(tensors):] == before[len(tensors):]

    changed(lambda: sv.pages_grow(*book, slots, i32([5])), ref, table, lens)
    changed(lambda: sv.pages_append(pool[0], k, v, starts, table, lens, slots), pool, same=(ref, table, lens, k, v))
    changed(lambda: sv.pages_fork(pool, *book, slots, i32([1])), pool, ref, table, lens)
    changed(lambda: sv.pages_free(*book, slots), ref, table, lens)
    changed(lambda: sv.pages_compact(pool, ref, table, live), pool, ref, table, live, same=(lens,))
    changed(lambda: sv.pages_copy(pool, i32([0]), i32([1])), pool)
    changed(lambda: sv.prompt_attention(q, k, v, starts, 5, out=out), out, same=(q, k, v))
    changed(lambda: sv.paged_attention(q[None, -1:], pool[0], table[1:], lens[1:], out=out4), out4, same=(q, pool))
    changed(lambda: sv.token_scores_grad(x, tok, out=x), x)
    changed(lambda: sv.token_scores_grad(x, tok), same=(x,))
    sv.status()
    w = torch.ones_like(x, requires_grad=True)
    y = (x * w).sum()
    sv.token_scores_grad(x, tok, out=x)
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        y.backward()
    # tensors of inference mode have no versions
    with torch.inference_mode():
        z = torch.empty_like(q)
        sv.prompt_attention(q, k, v, starts, 5, out=z)
    sv.prompt_attention(q, k, v, starts, 5, out=z)

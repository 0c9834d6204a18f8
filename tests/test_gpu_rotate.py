"""rotate_heads, rotate_append and rotate_heads_grad against plain 64-bit formulas (needs a GB300).

Tolerances, before any run; u = finfo.eps / 2 of the heads' type, the one rounding of an output.  In fp32 the sum of
squares of 128 elements is off by at most 21 2^-24 relative (16 in a chain, then pairs), r = rsqrt by half of
that and 2^-22, x r w by three roundings more: below 2^-19 relative; cos and sin are off by 2^-22.  So an
element of the turned pair (a, b) is within u |y| + 2^-18 (|a| + |b|), and half of the least subnormal.
Gradients: dx = r (g w - xh m) with m a mean of hd products, |dx - ref| <= u |ref| + 2^-17 r (|g w| + |xh| mean |g w xh|) where |g|
stands for |dy_a| + |dy_b|; dw is a sum of T H products of which a lane adds fewer than 64 in a chain and the
rest go by pairs or 32 at a time: 2^-16 of the sum of |g xh|.
"""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
TINY = {torch.bfloat16: 1e-38, torch.float16: 2.0 ** -25}


@pytest.fixture(scope="module")
def sv():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__ as g
    g.build()
    from paper_2606_10820_gb300 import serving
    return serving


def u_of(dtype):
    return torch.finfo(dtype).eps / 2


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def make(T, Hq, Hkv, hd, rot, dtype, seed=0, theta=1e4, far=5000, norm=True):
    g = gen(seed)

    def rand(*shape):
        return torch.randn(*shape, generator=g, device="cuda").to(dtype)

    qkv = rand(T, Hq + 2 * Hkv, hd)
    q, k, v = qkv.split([Hq, Hkv, Hkv], 1)
    pos = torch.randint(0, far, (T,), generator=g, device="cuda", dtype=torch.int32)
    freq = theta ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64, device="cuda") / max(rot, 1))
    how = {}
    if norm:
        how = {"eps": 1e-6, "q_weight": 1 + 0.3 * rand(hd), "k_weight": 1 + 0.3 * rand(hd)}
    return q, k, v, pos, freq, how


def turn(x, pos, freq, neighbours, sign=1):
    """Pairs turned in 64 bits, and |a| + |b| of each element's pair."""
    n = len(freq)
    a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if neighbours else (slice(0, n), slice(n, 2 * n))
    angle = sign * pos.double()[:, None, None] * freq
    c, s = angle.cos(), angle.sin()
    y, size = x.clone(), x.abs()
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
    return y, size


def normed(x, eps, w):
    x = x.double()
    if eps is None:
        return x
    x = x / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    return x if w is None else x * w.double()


def near(got, x, pos, freq, neighbours, eps=None, w=None):
    want, size = turn(normed(x, eps, w), pos, freq, neighbours)
    err = (got.double() - want).abs()
    assert (err <= u_of(got.dtype) * want.abs() + 2.0 ** -18 * size + TINY[got.dtype]).all(), (err / size.clamp(min=1e-6)).max().item()


def check(sv, q, k, pos, freq, neighbours, how):
    gq, gk = sv.rotate_heads(q, k, pos, freq, neighbours=neighbours, **how)
    assert gq.is_contiguous() and gk.is_contiguous() and gq.dtype == q.dtype
    near(gq, q, pos, freq, neighbours, how.get("eps"), how.get("q_weight"))
    near(gk, k, pos, freq, neighbours, how.get("eps"), how.get("k_weight"))
    return gq, gk


CASES = [(1, 1, 1), (3, 12, 4), (7, 5, 1), (129, 32, 8), (1000, 3, 3), (5003, 7, 2)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("hd,rot", [(64, 64), (64, 32), (64, 16), (64, 0), (128, 128), (128, 64), (128, 16), (128, 112)])
@pytest.mark.parametrize("T,Hq,Hkv", CASES)
def test_matches_plain(sv, dtype, neighbours, hd, rot, T, Hq, Hkv):
    q, k, _, pos, freq, how = make(T, Hq, Hkv, hd, rot, dtype, seed=T + rot)
    check(sv, q, k, pos, freq, neighbours, how)
    check(sv, q, k, pos, freq, neighbours, {})
    check(sv, q, k, pos, freq, neighbours, {"eps": 1e-5, "k_weight": how["k_weight"]})


@pytest.mark.parametrize("neighbours", [False, True])
def test_far_positions(sv, neighbours):
    """Positions up to the ends of 32 bits, and frequencies of one turn and more a token."""
    q, k, _, _, freq, how = make(64, 4, 2, 128, 128, torch.float16)
    pos = torch.tensor([0, 1, 2 ** 31 - 1, -1, -2 ** 31, 2 ** 24 + 1, 1000003, -77] * 8, dtype=torch.int32, device="cuda")
    # (64-bit angles of a radian a token are off by 2^31 2^-53: nothing against 2^-18)
    check(sv, q, k, pos, freq, neighbours, how)
    check(sv, q, k, pos, -freq, neighbours, how)
    few = torch.arange(64, dtype=torch.int32, device="cuda")
    check(sv, q, k, few, freq * 100 + 2 * math.pi, neighbours, {})
    tiny = torch.full_like(freq, 5e-324)
    assert torch.equal(sv.rotate_heads(q, k, pos, tiny)[0], q)
    wild = freq.clone()
    wild[3], wild[9], wild[20] = math.nan, math.inf, 2.0 ** 32
    got = sv.rotate_heads(q, k, few, wild)[0]
    bad = torch.isnan(got).all(0).all(0)
    assert torch.isnan(got).any(0).any(0).equal(bad) and bad.nonzero().flatten().tolist() == [3, 9, 20, 67, 73, 84]


def test_strides_in_place_and_values(sv):
    q, k, _, pos, freq, how = make(40, 6, 2, 64, 64, torch.bfloat16)
    want = sv.rotate_heads(q, k, pos, freq, **how)
    buf = torch.zeros(40, 11, 72, device="cuda", dtype=q.dtype)
    oq, ok = buf[:, 1:7, :64], buf[:, 8:10, 8:]
    before = buf._version
    got = sv.rotate_heads(q.clone(), k, pos, freq, q_out=oq, k_out=ok, **how)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and buf._version > before
    assert (buf[:, 0] == 0).all() and (buf[:, 7] == 0).all() and (buf[:, 1:7, 64:] == 0).all() and (buf[:, 8:, :8] == 0).all()
    # over the projection's output itself
    sv.rotate_heads(q, k, pos, freq, q_out=q, k_out=k, **how)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])
    # zeros stay zeros; an infinity or NaN stays in its head
    q[0, 0], q[1, 2, 5], q[2, 3, 7] = 0, math.inf, math.nan
    got = sv.rotate_heads(q, k, pos, freq, **how)[0]
    assert (got[0, 0] == 0).all() and torch.isnan(got[2, 3]).all()
    bad = ~torch.isfinite(got).all(-1)
    assert bad.nonzero().tolist() == [[1, 2], [2, 3]]
    empty = sv.rotate_heads(q[:0], k[:0], pos[:0], freq, **how)
    assert empty[0].shape == (0, 6, 64) and empty[1].shape == (0, 2, 64)


def cache(lens, counts, slots, Hkv, hd, page, dtype, g):
    n_slots = max(slots) + 2
    width = max(-(-x // page) for x in lens) + 1
    need = sum(-(-x // page) for x in lens)
    ids = torch.randperm(need + 3, generator=g, device="cuda").tolist()
    table = torch.full((n_slots, width), -1, dtype=torch.int32)
    all_lens = torch.zeros(n_slots, dtype=torch.int32)
    for s, x in zip(slots, lens):
        all_lens[s] = x
        for c in range(-(-x // page)):
            table[s, c] = ids.pop()
    pool = torch.full((need + 3, 2, Hkv, page, hd), 7.0, device="cuda", dtype=dtype)
    starts = torch.tensor([sum(counts[:i]) for i in range(len(counts) + 1)], dtype=torch.int32, device="cuda")
    return pool, starts, table.cuda(), all_lens.cuda(), torch.tensor(slots, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("lens,counts,Hq,Hkv,hd,page", [
    ([1], [1], 1, 1, 64, 16), ([5, 40, 17], [5, 8, 1], 12, 4, 64, 16), ([33, 7, 0, 300], [0, 7, 0, 131], 8, 2, 128, 16),
    ([20 + i for i in range(70)], [i % 3 for i in range(70)], 6, 3, 64, 5), ([9 + i for i in range(1100)], [1 + i % 2 for i in range(1100)], 2, 1, 128, 8),
    ([700], [700], 32, 8, 128, 48),
])
def test_append(sv, dtype, neighbours, lens, counts, Hq, Hkv, hd, page):
    T, n = sum(counts), len(lens)
    q, k, v, _, freq, how = make(T, Hq, Hkv, hd, hd // 2, dtype, seed=n)
    g = gen(n + page)
    slots = torch.randperm(n + 3, generator=g, device="cuda")[:n].tolist()
    pool, starts, table, book_lens, which = cache(lens, counts, slots, Hkv, hd, page, dtype, g)
    pos = torch.cat([torch.arange(x - c, x, device="cuda") for x, c in zip(lens, counts)]).int()
    want_q, want_k = check(sv, q, k, pos, freq, neighbours, how)
    want = pool.clone()
    sv.pages_append(want, want_k, v, starts, table, book_lens, which)
    before = pool._version
    got = sv.rotate_append(q, k, v, pool, starts, table, book_lens, which, freq, neighbours=neighbours, **how)
    sv.status()
    assert torch.equal(got, want_q) and torch.equal(pool, want) and pool._version > before


def test_append_of_bad_tokens(sv):
    """A slot, position or page out of range: flagged, nothing of that token in the pool, and zeros for q where no position is known."""
    counts, lens, slots = [2, 3, 2, 1], [20, 3, 40, 9], [0, 1, 2, 3]
    q, k, v, _, freq, how = make(8, 4, 2, 64, 64, torch.bfloat16)
    pool, starts, table, book_lens, which = cache(lens, counts, slots, 2, 64, 16, torch.bfloat16, gen(3))
    good = sv.rotate_append(q, k, v, pool.clone(), starts, table, book_lens, which, freq, **how)
    sv.status()

    def run(bit, **kw):
        args = {"starts": starts, "table": table, "lens": book_lens, "slots": which, **kw}
        p = pool.clone()
        got = sv.rotate_append(q, k, v, p, args["starts"], args["table"], args["lens"], args["slots"], freq, **how)
        with pytest.raises(Exception, match=f"flags {bit}$"):
            sv.status()
        return got, (p != 7).flatten(1).any(1).sum().item()

    whole = 4            # pages that the four sequences' new tokens touch
    got, pages = run(8, slots=torch.tensor([0, 9, 2, 3], dtype=torch.int32, device="cuda"))
    assert (got[2:5] == 0).all() and torch.equal(got[:2], good[:2]) and torch.equal(got[5:], good[5:]) and pages == whole - 1
    short = book_lens.clone()
    short[2] = 1         # two new tokens of a sequence of one
    got, _ = run(8, lens=short)
    assert (got[5] == 0).all() and (got[6] != 0).any()
    bad = table.clone()
    bad[1, 0] = 1 << 30
    got, pages = run(2, table=bad)
    assert torch.equal(got, good) and pages == whole - 1
    got, pages = run(8, starts=torch.tensor([0, 2, 5, 7, 7], dtype=torch.int32, device="cuda"))       # a row behind the last
    assert (got[7] == 0).all() and torch.equal(got[:7], good[:7]) and pages == whole - 1


def plain_back(dq, x, pos, freq, neighbours, eps, w):
    """dx, dw and the sizes that their errors go by."""
    g, size = turn(dq.double(), pos, freq, neighbours, -1)
    x = x.double()
    if eps is None:
        return g, size, None, None
    r = 1 / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    xh = x * r
    w = torch.ones(x.shape[-1], device=x.device, dtype=torch.float64) if w is None else w.double()
    dx = r * (g * w - xh * (g * w * xh).mean(-1, keepdim=True))
    bound = r * (size * w.abs() + xh.abs() * (size * w * xh).abs().mean(-1, keepdim=True))
    return dx, bound, (g * xh).sum((0, 1)), (size * xh).abs().sum((0, 1))


def check_back(sv, dq, dk, q, k, pos, freq, neighbours, how):
    got = sv.rotate_heads_grad(dq, dk, q, k, pos, freq, neighbours=neighbours, **how)
    assert set(got) == {"q", "k"} | {x for x in ("q_weight", "k_weight") if how.get(x) is not None}
    for name, dy, x in (("q", dq, q), ("k", dk, k)):
        dx, size, dw, wsize = plain_back(dy, x, pos, freq, neighbours, how.get("eps"), how.get(name + "_weight"))
        err = (got[name].double() - dx).abs()
        assert (err <= u_of(q.dtype) * dx.abs() + 2.0 ** -17 * size + TINY[q.dtype]).all(), err.max().item()
        if name + "_weight" in got:
            gw = got[name + "_weight"]
            assert gw.dtype == torch.float32 and ((gw.double() - dw).abs() <= 2.0 ** -16 * wsize).all()
    return got


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("hd,rot", [(64, 64), (64, 16), (128, 128), (128, 64), (128, 0)])
@pytest.mark.parametrize("T,Hq,Hkv", CASES)
def test_gradients(sv, dtype, neighbours, hd, rot, T, Hq, Hkv):
    q, k, _, pos, freq, how = make(T, Hq, Hkv, hd, rot, dtype, seed=T + rot)
    g = gen(5)
    dq, dk = (torch.randn(T, 2 * h, hd, generator=g, device="cuda").to(dtype)[:, ::2] for h in (Hq, Hkv))
    got = check_back(sv, dq, dk, q, k, pos, freq, neighbours, how)
    again = sv.rotate_heads_grad(dq, dk, q, k, pos, freq, neighbours=neighbours, **how)
    assert all(torch.equal(got[x], again[x]) for x in got)
    check_back(sv, dq, dk, q, k, pos, freq, neighbours, {})
    check_back(sv, dq, dk, q, k, pos, freq, neighbours, {"eps": 1e-5})
    check_back(sv, dq, dk, q, k, pos, freq, neighbours, {"eps": 1e-5, "q_weight": how["q_weight"]})


def test_gradients_against_differences(sv):
    """d/dh of sum(dy y(x + h d)) in 64 bits is <dx, d>: the formula that the others are held to, and the kernel (u of its sizes)."""
    q, k, _, pos, freq, how = make(6, 3, 2, 64, 32, torch.float16, seed=8)
    g = gen(9)
    dq, dk, d = (torch.randn(6, h, 64, generator=g, device="cuda").half() for h in (3, 2, 3))
    got = sv.rotate_heads_grad(dq, dk, q, k, pos, freq, **how)

    def f(x, w):
        return (dq.double() * turn(normed(x, how["eps"], w), pos, freq, False)[0]).sum()

    h, w = 1e-4, how["q_weight"]
    by = (f(q.double() + h * d.double(), w) - f(q.double() - h * d.double(), w)) / (2 * h)
    dx, size, dw, _ = plain_back(dq, q, pos, freq, False, how["eps"], w)
    assert abs((dx * d.double()).sum() - by) <= 1e-5 * (dx * d.double()).abs().sum()
    assert abs((got["q"].double() * d.double()).sum() - by) <= ((u_of(torch.float16) * dx.abs() + 2.0 ** -17 * size) * d.double().abs()).sum() + 1e-5 * (dx * d.double()).abs().sum()
    e = torch.randn(64, generator=g, device="cuda").double()
    by = (f(q, w.double() + h * e) - f(q, w.double() - h * e)) / (2 * h)
    assert abs((got["q_weight"].double() * e).sum() - by) <= 1e-5 * (got["q_weight"].double() * e).abs().sum() + 1e-4


def test_many_tokens_and_strides_past_32_bits(sv):
    """Rows whose offsets pass 2^31 elements."""
    base = torch.empty(3, 1 << 30, device="cuda", dtype=torch.bfloat16)      # 6.4 GB
    rows = base[:, : 6 * 64].view(3, 6, 64) if base[:, : 6 * 64].is_contiguous() else base[:, : 6 * 64].unflatten(1, (6, 64))
    rows.copy_(torch.randn(3, 6, 64, device="cuda"))
    q, k = rows.split([4, 2], 1)
    assert q.stride(0) == 1 << 30
    _, _, _, pos, freq, how = make(3, 4, 2, 64, 64, torch.bfloat16)
    check(sv, q, k, pos, freq, False, how)
    check_back(sv, q, k, q, k, pos, freq, False, how)


def test_captured_and_on_another_stream(sv):
    q, k, _, pos, freq, how = make(300, 8, 2, 128, 128, torch.bfloat16)
    want, back = sv.rotate_heads(q, k, pos, freq, **how), sv.rotate_heads_grad(q, k, q, k, pos, freq, **how)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = sv.rotate_heads(q, k, pos, freq, **how)
    s.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = sv.rotate_heads(q, k, pos, freq, **how)
        b = sv.rotate_heads_grad(q, k, q, k, pos, freq, **how)
    q.copy_(torch.randn_like(q))
    graph.replay()
    want, back2 = sv.rotate_heads(q, k, pos, freq, **how), sv.rotate_heads_grad(q, k, q, k, pos, freq, **how)
    assert torch.equal(y[0], want[0]) and all(torch.equal(b[x], back2[x]) for x in b)
    assert not torch.equal(back["q"], b["q"])


def test_refusals(sv):
    q, k, v, pos, freq, how = make(4, 4, 2, 64, 64, torch.bfloat16)
    from paper_2606_10820_gb300.kforcing import KfError
    for bad in (dict(q=q.float(), k=k.float()), dict(k=k.half()), dict(k=k[:3]), dict(q=q.transpose(1, 2)), dict(pos=pos.long()),
                dict(pos=pos[:3]), dict(freq=freq.float()), dict(freq=freq.cpu()), dict(q=q[0]), dict(q=q.cpu()),
                dict(q_weight=how["q_weight"].float(), eps=1e-6), dict(q_weight=how["q_weight"][:32], eps=1e-6), dict(eps=-1.0),
                dict(eps="x"), dict(q_out=k), dict(k_out=k.float())):
        args = {"q": q, "k": k, "pos": pos, "freq": freq, **bad}
        with pytest.raises(ValueError):
            sv.rotate_heads(**args)
    for bad in (dict(freq=freq[:12]), dict(freq=torch.cat([freq, freq])), dict(q_weight=how["q_weight"]), dict(eps=math.inf),
                dict(q_out=torch.empty(4, 4, 68, device="cuda", dtype=q.dtype)[..., 4:]),
                dict(q=torch.zeros(4, 4, 96, device="cuda", dtype=q.dtype), k=torch.zeros(4, 2, 96, device="cuda", dtype=q.dtype))):
        args = {"q": q, "k": k, "pos": pos, "freq": freq, **bad}
        with pytest.raises(KfError):
            sv.rotate_heads(**args)
    grad = q.clone().requires_grad_()
    with pytest.raises(ValueError):
        sv.rotate_heads(grad, k, pos, freq)
    with torch.no_grad():
        sv.rotate_heads(grad, k, pos, freq)
    with pytest.raises(ValueError):
        sv.rotate_heads_grad(q[:, :3], k, q, k, pos, freq)
    pool = torch.zeros(3, 2, 2, 16, 64, device="cuda", dtype=q.dtype)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    fine = dict(q=q, k=k, v=v, pool=pool, starts=i32([0, 4]), table=i32([[0]]), lens=i32([4]), slots=i32([0]), freq=freq)
    sv.rotate_append(**fine)
    sv.status()
    for bad in (dict(v=v[:, :1]), dict(pool=pool.half()), dict(pool=pool[:, :1]), dict(starts=i32([0, 2, 4])), dict(lens=i32([4, 4])),
                dict(slots=i32([[0]])), dict(v=v.half())):
        with pytest.raises(ValueError):
            sv.rotate_append(**{**fine, **bad})
    with pytest.raises(KfError):
        sv.rotate_append(**{**fine, "slots": i32([]), "starts": i32([0])})


def test_append_past_32_bits_and_captured(sv):
    """Pages past 2^31 elements of a pool; a captured call follows the book that its replay finds."""
    pool = torch.full((70000, 2, 8, 16, 128), 7.0, device="cuda", dtype=torch.bfloat16)       # 4.6 GB
    q, k, v, _, freq, how = make(5, 32, 8, 128, 128, torch.bfloat16, seed=4)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    starts, slots, lens = i32([0, 3, 5]), i32([1, 0]), i32([18, 3])
    table = i32([[69999, 68000], [1, 69000]])

    def expect(lens):
        n0, n1 = lens.tolist()
        pos = i32([n1 - 3, n1 - 2, n1 - 1, n0 - 2, n0 - 1])
        wq, wk = sv.rotate_heads(q, k, pos, freq, **how)
        at = [(table[s, p // 16].item(), p % 16) for s, p in zip([1, 1, 1, 0, 0], pos.tolist())]
        return wq, wk, at

    def held(wk, at):
        return all(torch.equal(pool[p, 0, :, r], wk[i]) and torch.equal(pool[p, 1, :, r], v[i]) for i, (p, r) in enumerate(at))

    got = sv.rotate_append(q, k, v, pool, starts, table, lens, slots, freq, **how)
    sv.status()
    wq, wk, at = expect(lens)
    assert torch.equal(got, wq) and held(wk, at)
    assert (pool[[1, 68000, 69000, 69999]] != 7).any(-1).any(2).sum() == 2 * 5 and (pool[:1] == 7).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = sv.rotate_append(q, k, v, pool, starts, table, lens, slots, freq, **how)
    lens.copy_(i32([31, 22]))
    graph.replay()
    sv.status()
    wq, wk, at = expect(lens)
    assert torch.equal(y, wq) and held(wk, at)

"""paged_attention against plain attention in 64 bits (needs a GB300).

Tolerance, before any run: an output row is a convex combination of V rows with
probabilities rounded to the cache's type (u = 2^-9 bf16, 2^-12 fp16 relative), scores
and sums in fp32, and the output rounded once more (u |out|).  |out - ref| <= u max|V| + u |ref| +
fp32 terms (scores of size 8 with hd products: below 2^-16 of max|V|): 2.2 u max|V| + 2^-15 max|V|.
"""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
U = {torch.bfloat16: 2.0 ** -9, torch.float16: 2.0 ** -12}


@pytest.fixture(scope="module")
def sv():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__ as g
    g.build()
    from paper_2606_10820_gb300 import serving
    return serving


def make(lens, rows, Hq, Hkv, hd, dtype=torch.bfloat16, page=16, spare=3, extra_width=2, seed=0, std=1.0):
    """q, pool (unused pages and slots hold NaN), table, lens on the GPU."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    need = [-(-x // page) for x in lens]
    n_pages = sum(need) + spare
    pool = torch.full((n_pages, 2, Hkv, page, hd), math.nan, device="cuda", dtype=dtype)
    ids = torch.randperm(n_pages, generator=g, device="cuda").tolist()
    width = max(need + [0]) + extra_width
    table = torch.full((len(lens), width), -1, dtype=torch.int32)
    for b, x in enumerate(lens):
        for i in range(need[b]):
            pg = ids.pop()
            table[b, i] = pg
            n = min(page, x - i * page)
            pool[pg, :, :, :n] = torch.randn(2, Hkv, n, hd, generator=g, device="cuda").to(dtype)
    q = (torch.randn(len(lens), rows, Hq, hd, generator=g, device="cuda") * std).to(dtype)
    return q, pool, table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")


def plain(q, pool, table, lens, scale=None):
    B, rows, Hq, hd = q.shape
    Hkv = pool.shape[2]
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    big = torch.zeros(B, device=q.device, dtype=torch.float64)
    scale = scale or 1 / math.sqrt(hd)
    for b, n in enumerate(lens.tolist()):
        if n == 0:
            continue
        pages = table[b, : -(-n // pool.shape[3])].long()
        kv = pool[pages].permute(1, 2, 0, 3, 4).flatten(2, 3)[:, :, :n].double().repeat_interleave(Hq // Hkv, 1)
        w = torch.einsum("rhd,hkd->hrk", q[b].double(), kv[0]) * scale
        last = n - rows + torch.arange(rows, device=q.device)
        seen = torch.arange(n, device=q.device)[None] <= last[:, None]
        w = w.masked_fill(~seen, -math.inf)
        p = torch.nan_to_num(torch.softmax(w, -1)) if (last < 0).any() else torch.softmax(w, -1)
        out[b] = torch.einsum("hrk,hkd->rhd", p, kv[1])
        big[b] = kv[1].abs().max()
    return out, big


def check(sv, q, pool, table, lens, scale=None):
    got = sv.paged_attention(q, pool, table, lens, scale=scale)
    ref, big = plain(q, pool, table, lens, scale)
    err = (got.double() - ref).abs().amax((1, 2, 3))
    assert torch.isfinite(got).all()
    assert (err <= (2.2 * U[q.dtype] + 2.0 ** -15) * big).all(), (err / big.clamp(min=1e-9)).max().item()
    sv.status()
    return got


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("lens,rows,Hq,Hkv", [
    ([1], 1, 1, 1), ([0], 1, 2, 1), ([3, 0, 1], 1, 4, 2), ([15, 16, 17, 31, 32, 33], 1, 6, 2), ([64, 65, 127, 1], 1, 8, 8),
    ([1000], 1, 4, 1), ([5000, 3], 1, 7, 1), ([129, 700, 2], 1, 40, 2), ([260, 5, 33], 3, 6, 2), ([8, 9, 200], 8, 12, 4),
    ([5, 2, 0, 40], 8, 4, 4), ([300] * 40, 1, 4, 2), (list(range(1, 90)), 1, 3, 3), ([20011], 2, 16, 2),
])
def test_matches_plain(sv, hd, dtype, lens, rows, Hq, Hkv):
    check(sv, *make(lens, rows, Hq, Hkv, hd, dtype, seed=len(lens) + rows))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("lens,rows,Hq,Hkv", [
    ([20011, 5], 5, 32, 8), ([3000, 0, 1, 15, 16, 17, 4099], 8, 8, 2), ([700 + 37 * i for i in range(40)], 7, 8, 1),
    (list(range(0, 2400, 7)), 3, 6, 1), ([9000, 4], 17, 1, 1), ([2500, 2, 33], 7, 16, 2), ([5001], 33, 2, 2), ([0, 0], 8, 8, 2),
])
@pytest.mark.parametrize("wide", [False, True])
def test_many_rows_of_long_sequences(sv, dtype, lens, rows, Hq, Hkv, wide):
    """Two and more tiles of 16 rows of a group, past what one CTA takes as a whole; tiles that are full, ragged
    and without a partner.  wide: a cache past the L2's size, where two tiles share a segment."""
    more = (140 << 20) // (16 * Hkv * 512) if wide else 0
    check(sv, *make(lens, rows, Hq, Hkv, 128, dtype, seed=len(lens) + rows, spare=3 + more, extra_width=30 + -(-more // len(lens))))


@pytest.mark.parametrize("page", [32, 48, 128])
def test_page_sizes(sv, page):
    check(sv, *make([1, 47, 48, 49, 500, 1300], 2, 8, 2, 128, page=page, seed=page))


@pytest.mark.parametrize("seed", range(4))
def test_random_batches(sv, seed):
    """Ragged batches that end parts inside segments, segments inside units."""
    g = torch.Generator().manual_seed(seed)
    n = [3, 40, 333, 700][seed]
    lens = torch.randint(0, [9000, 1500, 300, 70][seed], (n,), generator=g).tolist()
    check(sv, *make(lens, [1, 4, 1, 2][seed], [8, 6, 4, 5][seed], [2, 2, 1, 5][seed], [128, 64, 64, 128][seed],
                    [torch.bfloat16, torch.float16][seed % 2], seed=seed))


def test_peaked_and_scaled(sv):
    """Scores in the hundreds (one key takes all), and a scale of one's own."""
    args = make([700, 90, 1], 1, 8, 2, 64, torch.float16, std=30.0, seed=3)
    check(sv, *args)
    check(sv, *make([700, 90, 1], 1, 8, 2, 64, torch.bfloat16, seed=4), scale=0.37)


def test_same_bits_whatever_the_pages(sv):
    q, pool, table, lens = make([900, 17, 333], 1, 8, 2, 128, seed=9)
    a = sv.paged_attention(q, pool, table, lens)
    perm = torch.randperm(len(pool), device="cuda")
    inv = torch.argsort(perm)
    moved = torch.where(table >= 0, inv[table.clamp(min=0).long()].to(torch.int32), -1)
    for _ in range(3):
        assert torch.equal(a, sv.paged_attention(q, pool[perm].contiguous(), moved, lens))


def test_shared_pages(sv):
    """Two sequences over the same prompt pages (a fork)."""
    q, pool, table, lens = make([200, 200], 1, 4, 2, 64, seed=2)
    table[1] = table[0]
    check(sv, q, pool, table, lens)


def test_strides_stream_graph(sv):
    """q as a part of a projection's output, on another stream, and captured."""
    q, pool, table, lens = make([333, 40], 2, 6, 2, 64, seed=6)
    wide = torch.zeros(2, 2, 10, 64, device="cuda", dtype=q.dtype)
    wide[:, :, 2:8] = q
    want = sv.paged_attention(q, pool, table, lens)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = sv.paged_attention(wide[:, :, 2:8], pool, table, lens)
    s.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = sv.paged_attention(q, pool, table, lens)
    lens.copy_(torch.tensor([100, 7], dtype=torch.int32))
    graph.replay()
    torch.cuda.synchronize()
    ref, big = plain(q, pool, table, lens)
    assert ((out.double() - ref).abs().amax((1, 2, 3)) <= (2.2 * U[q.dtype] + 2.0 ** -15) * big).all()


def test_large_pool_offsets(sv):
    """Pages past 2^31 elements of the pool."""
    n_pages, hd = 70000, 128
    pool = torch.empty(n_pages, 2, 16, 16, hd, device="cuda", dtype=torch.bfloat16)     # 4.6e9 elements
    g = torch.Generator(device="cuda").manual_seed(1)
    table = torch.tensor([[69999, 3, 50000], [40000, 69998, 0]], dtype=torch.int32, device="cuda")
    for p in table.flatten().tolist():
        pool[p] = torch.randn(2, 16, 16, hd, generator=g, device="cuda")
    q = torch.randn(2, 1, 16, hd, generator=g, device="cuda").bfloat16()
    check(sv, q, pool, table, torch.tensor([48, 35], dtype=torch.int32, device="cuda"))


def test_bad_tables_and_lengths(sv):
    """Page ids outside the pool count as unseen keys; lengths are clamped; both are reported."""
    from paper_2606_10820_gb300.kforcing import KfError
    q, pool, table, lens = make([64, 40], 1, 4, 2, 128, extra_width=0, seed=8)
    bad = table.clone()
    bad[0, 1], bad[0, 3], bad[1, 0] = -7, len(pool), 1 << 30
    got = sv.paged_attention(q, pool, bad, lens)
    with pytest.raises(KfError) as e:
        sv.status()
    assert "flags 2" in str(e.value)
    # sequence 0 with its keys 16..31 and 48..63 taken out
    keep = table[0, [0, 2]].long()
    kv = pool[keep].permute(1, 2, 0, 3, 4).flatten(2, 3).double().repeat_interleave(2, 1)
    w = torch.softmax(torch.einsum("rhd,hkd->hrk", q[0].double(), kv[0]) / math.sqrt(128), -1)
    ref = torch.einsum("hrk,hkd->rhd", w, kv[1])
    assert (got[0].double() - ref).abs().max() <= (2.2 * U[q.dtype] + 2.0 ** -15) * kv[1].abs().max()
    sv.status()
    long = torch.tensor([1000, -5], dtype=torch.int32, device="cuda")
    got = sv.paged_attention(q, pool, table, long)
    with pytest.raises(KfError):
        sv.status()
    want = sv.paged_attention(q, pool, table, torch.tensor([64, 0], dtype=torch.int32, device="cuda"))
    assert torch.equal(got, want) and (got[1] == 0).all()
    sv.status()


def test_refusals(sv):
    from paper_2606_10820_gb300.kforcing import KfError
    q, pool, table, lens = make([64, 40], 1, 4, 2, 64)
    for call in (lambda: sv.paged_attention(q[..., :32].contiguous(), pool[..., :32].contiguous(), table, lens),   # head_dim
                 lambda: sv.paged_attention(q[:, :, :3], pool, table, lens),                                        # heads
                 lambda: sv.paged_attention(q, pool[:, :, :, :8].contiguous(), table, lens),                        # page
                 lambda: sv.paged_attention(q, pool, table, lens, scale=0.0),
                 lambda: sv.paged_attention(q, pool, table, lens, scale=math.nan)):
        with pytest.raises(KfError):
            call()
    for call in (lambda: sv.paged_attention(q.float(), pool.float(), table, lens), lambda: sv.paged_attention(q.half(), pool, table, lens),
                 lambda: sv.paged_attention(q, pool.transpose(3, 4), table, lens), lambda: sv.paged_attention(q, pool, table.long(), lens),
                 lambda: sv.paged_attention(q, pool, table, lens[:1]), lambda: sv.paged_attention(q.cpu(), pool, table, lens),
                 lambda: sv.paged_attention(q, pool, table.cpu(), lens)):
        with pytest.raises(ValueError):
            call()
    assert sv.paged_attention(q[:0], pool, table[:0], lens[:0]).shape == (0, 1, 4, 64)
    sv.status()

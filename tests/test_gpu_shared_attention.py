"""shared_attention against plain attention in 64 bits (needs a GB300).

Tolerance, before any run: an output row is a convex combination of V rows; with u = finfo.eps / 2 of the
type the rounded probabilities move it by at most u max|V|, the output's own rounding by u |out| <= u max|V|, and what is
fp32 (scores of size 8 with hd products, sums, joins) by less than 2^-15 max|V|: 2 u max|V| + 2^-15 max|V|.
"""
import math

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


WAYS = ["paged", "rows", "tiles"]      # what reads the prefixes: paged attention, 16 or 32 rows at a time, 256


def room(way, B, n, rows, Hq, Hkv, hd, page):
    """Pages of a pool and of the table's width that make a call of these sizes choose the way (kf_shared_attention.cu: the reads
    that they would allow for, 48 MB of all sequences' and 128 MB of all tiles')."""
    per = rows * Hq // Hkv
    seg = 32 if hd == 64 and per > 16 else 16
    bytes_ = page * hd * 4 * Hkv
    if way == "rows":
        return (50 << 20) // (B * -(-per // seg) * bytes_) + 1
    return (135 << 20) // (max(1, B * per // seg) * bytes_) + 1 if way == "tiles" else 0


def make(groups, rows, Hq, Hkv, hd, dtype=torch.bfloat16, page=16, extra_width=2, seed=0, std=1.0, hide=False, spare=3, way="paged"):
    """groups: (shared tokens, lengths of the sequences) each.  Full pages of a prefix are in all tables, the rest of it is copied
    (hide: in no table but the first's); pages that nothing uses and slots past the lengths hold NaN."""
    wide = room(way, sum(len(lens) for _, lens in groups), len(groups), rows, Hq, Hkv, hd, page)
    spare, extra_width = spare + wide, extra_width + wide
    g = torch.Generator(device="cuda").manual_seed(seed)
    need = sum(n // page + sum(-(-x // page) - n // page for x in lens) for n, lens in groups) + spare
    pool = torch.full((need, 2, Hkv, page, hd), math.nan, device="cuda", dtype=dtype)
    ids = torch.randperm(need, generator=g, device="cuda").tolist()
    width = max([-(-x // page) for _, lens in groups for x in lens] + [0]) + extra_width
    B = sum(len(lens) for _, lens in groups)
    table = torch.full((B, width), -1, dtype=torch.int32)

    def rand(n):
        return torch.randn(2, Hkv, n, hd, generator=g, device="cuda").to(dtype)

    b, starts = 0, [0]
    for n, lens in groups:
        full, kept, part = n // page, [], rand(n % page)
        for _ in range(full):
            kept.append(ids.pop())
            pool[kept[-1]] = rand(page)
        for i, x in enumerate(lens):
            table[b, :full] = torch.tensor(kept, dtype=torch.int32) if not hide or i == 0 else -1
            for c in range(full, -(-x // page)):
                p = ids.pop()
                table[b, c] = p
                m = min(page, x - c * page)
                pool[p, :, :, :m] = rand(m)
                if c == full and n % page:
                    pool[p, :, :, : n % page] = part if not hide or i == 0 else math.nan
            b += 1
        starts.append(b)
    q = (torch.randn(B, rows, Hq, hd, generator=g, device="cuda") * std).to(dtype)
    return q, pool, table.cuda(), i32([x for _, lens in groups for x in lens]), i32(starts), i32([n for n, _ in groups])


def plain(q, pool, table, lens, starts, shared, scale=None):
    B, rows, Hq, hd = q.shape
    Hkv, page = pool.shape[2:4]
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    big = torch.zeros(B, device=q.device, dtype=torch.float64)
    scale = scale or 1 / math.sqrt(hd)
    lens, starts, shared = lens.tolist(), starts.tolist(), shared.tolist()
    for a, e, n in zip(starts, starts[1:], shared):
        for b in range(a, e):
            if lens[b] == 0:
                continue
            at = torch.arange(lens[b], device=q.device)
            row = torch.where(at < n, a, b)
            kv = pool[table[row, at // page].long(), :, :, at % page].double().permute(1, 2, 0, 3).repeat_interleave(Hq // Hkv, 1)
            w = torch.einsum("rhd,hkd->hrk", q[b].double(), kv[0]) * scale
            last = lens[b] - rows + torch.arange(rows, device=q.device)
            w = w.masked_fill(at[None] > last[:, None], -math.inf)
            p = torch.nan_to_num(torch.softmax(w, -1))
            out[b] = torch.einsum("hrk,hkd->rhd", p, kv[1])
            big[b] = kv[1].abs().max()
    return out, big


def check(sv, *args, scale=None):
    got = sv.shared_attention(*args, scale=scale)
    sv.status()
    want, big = plain(*args, scale=scale)
    assert torch.isfinite(got).all()
    err = (got.double() - want).abs().amax((1, 2, 3))
    u = torch.finfo(args[0].dtype).eps / 2
    assert (err <= (2 * u + 2.0 ** -15) * big).all(), (err / big.clamp(min=1e-9)).max().item()
    return got


BATCHES = [
    ([(1, [1, 2])], 1, 1, 1), ([(0, [5, 0, 17])], 1, 4, 2), ([(16, [16, 17, 40]), (15, [30, 15])], 1, 6, 2),
    ([(129, [130, 700, 129]), (0, [3, 0]), (128, [128, 300])], 1, 8, 8), ([(517, [518 + 7 * i for i in range(8)])], 1, 12, 4),
    ([(1000, [1000 + i for i in range(64)])], 1, 32, 8), ([(5000, [5001, 5900]), (33, [34] * 5), (2, [1000, 3, 2])], 1, 7, 1),
    ([(300, [308 + i for i in range(16)]), (127, [200, 136]), (250, [258])], 8, 12, 4), ([(20, [24, 25, 400]), (0, [5, 3, 0, 1])], 5, 4, 4),
    ([(4000, [4010 + 9 * i for i in range(40)])], 3, 16, 2), ([(700, [701] * 3), (90, [95, 100])], 1, 40, 2),
    ([(17 * i, [17 * i + 1 + j for j in range(1 + i % 4)]) for i in range(40)], 1, 3, 3), ([(63, [64 + i for i in range(130)])], 2, 8, 4),
]


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("groups,rows,Hq,Hkv", BATCHES)
@pytest.mark.parametrize("way", WAYS)
def test_matches_plain(sv, hd, dtype, groups, rows, Hq, Hkv, way):
    check(sv, *make(groups, rows, Hq, Hkv, hd, dtype, seed=len(groups) + rows, way=way))


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("way", WAYS[1:])
def test_the_prefix_is_read_through_the_first_table(sv, hd, way):
    """(What these two ways do beyond what is promised: it shows that they read a prefix once.)"""
    check(sv, *make([(333, [340, 900, 333 + 8]), (48, [56, 57]), (5, [13, 14, 15, 40])], 8, 8, 2, hd, hide=True, seed=5, way=way))


@pytest.mark.parametrize("page", [32, 48, 128])
@pytest.mark.parametrize("way", WAYS)
def test_page_sizes(sv, page, way):
    check(sv, *make([(500, [501, 640, 900]), (47, [48, 49]), (128, [129, 128])], 1, 8, 2, 128, page=page, seed=page, way=way))


@pytest.mark.parametrize("way", WAYS)
def test_one_call_over_many_tiles(sv, way):
    """A prefix in more pieces than CTAs take whole, and one of a group's many rows over several pairs of sub-tiles."""
    check(sv, *make([(32771, [32772 + 100 * i for i in range(6)])], 1, 8, 2, 128, seed=1, way=way))
    check(sv, *make([(700, [710 + i for i in range(150)]), (64, [72] * 9)], 8, 24, 4, 64, torch.float16, seed=2, way=way))


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("way", WAYS)
def test_random_groups(sv, seed, way):
    g = torch.Generator().manual_seed(seed)

    def r(lo, hi):
        return int(torch.randint(lo, hi, (1,), generator=g))

    rows = [1, 4, 1, 2, 8, 1][seed]
    groups = []
    for _ in range([3, 20, 60, 1, 9, 200][seed]):
        n = r(0, [3000, 600, 100, 9000, 700, 40][seed])
        groups.append((n, [n + r(0, [200, 900, 30, 40, 300, 20][seed]) for _ in range(r(0, [5, 6, 9, 30, 12, 4][seed]))]))
    groups.append((4, [9]))
    check(sv, *make(groups, rows, [8, 6, 4, 16, 12, 5][seed], [2, 2, 1, 4, 4, 5][seed], [128, 64, 64, 128, 64, 128][seed],
                    [torch.bfloat16, torch.float16][seed % 2], seed=seed, hide=seed % 2 == 0 and way != "paged", way=way))


@pytest.mark.parametrize("way", WAYS)
def test_rows_that_see_part_of_the_prefix(sv, way):
    """A prefix that reaches into the newest rows, to the last token: row i still sees keys 0 .. len - rows + i."""
    check(sv, *make([(200, [200, 201, 203, 300]), (6, [6, 7]), (3, [3, 3, 4])], 8, 8, 2, 64, seed=3, way=way))
    check(sv, *make([(129, [129, 129, 130])], 140, 2, 1, 128, seed=4, way=way))


@pytest.mark.parametrize("way", WAYS)
def test_shared_with_the_whole_of_paged_attention(sv, way):
    """Tables as a fork leaves them: both attentions give the same rows, within the tolerances of both."""
    args = make([(400 + 50 * i, [400 + 50 * i + 8 + 13 * j for j in range(9)]) for i in range(7)], 4, 12, 4, 64, torch.float16, seed=6, way=way)
    got, whole = check(sv, *args), sv.paged_attention(*args[:4])
    assert ((got.double() - whole.double()).abs().max() <= 2 * (2 * 2.0 ** -11 + 2.0 ** -15) * args[1].nan_to_num().abs().max())
    # groups of one are paged attention
    B = len(args[3])
    singles = sv.shared_attention(*args[:4], i32(list(range(B + 1))), i32([8] * B))
    assert torch.equal(singles, whole)


@pytest.mark.parametrize("way", WAYS)
def test_peaked_and_scaled(sv, way):
    check(sv, *make([(700, [701, 790]), (90, [91])], 1, 8, 2, 64, torch.float16, std=30.0, seed=3, way=way))
    check(sv, *make([(700, [701, 790]), (90, [91])], 1, 8, 2, 128, torch.bfloat16, std=30.0, seed=3, way=way))
    check(sv, *make([(700, [701, 790]), (90, [91])], 1, 8, 2, 64, seed=4, way=way), scale=0.37)


@pytest.mark.parametrize("way", WAYS)
def test_infinities_stay_in_their_group(sv, way):
    args = make([(300, [301, 400]), (300, [305, 310])], 1, 4, 2, 64, seed=7, way=way)
    q, pool, table = args[:3]
    want = sv.shared_attention(*args)
    pool[table[0, 3].long(), 1, 0, 5, 7] = math.nan
    pool[table[3, 19].long(), 1, 1, 2, 1] = math.inf          # an own key of the last sequence
    got = sv.shared_attention(*args)
    assert torch.isnan(got[:2, :, :2, 7]).all() and torch.isinf(got[3, :, 2:, 1]).all()
    got[:2, :, :2, 7] = want[:2, :, :2, 7]
    got[3, :, 2:, 1] = want[3, :, 2:, 1]
    assert torch.equal(got, want)


@pytest.mark.parametrize("way", WAYS)
def test_same_bits_and_strides(sv, way):
    """The same call gives the same bits, whatever the pages' order and q's strides."""
    q, pool, table, lens, starts, shared = make([(900, [901 + 40 * i for i in range(20)]), (77, [100, 2000])], 2, 16, 4, 128, seed=8, way=way)
    want = sv.shared_attention(q, pool, table, lens, starts, shared)
    perm = torch.randperm(len(pool), device="cuda")
    back = torch.argsort(perm)
    moved = torch.where(table >= 0, back[table.clamp(min=0).long()].int(), table)
    wide = torch.zeros(q.shape[0], q.shape[1], 20, 136, device="cuda", dtype=q.dtype)
    wide[:, :, 2:18, :128] = q
    out = torch.empty_like(q)
    got = sv.shared_attention(wide[:, :, 2:18, :128], pool[perm].contiguous(), moved, lens, starts, shared, out=out)
    assert got.data_ptr() == out.data_ptr() and torch.equal(got, want)
    assert torch.equal(sv.shared_attention(q, pool, table, lens, starts, shared), want)


@pytest.mark.parametrize("way", WAYS)
def test_bad_pages_and_rows(sv, way):
    args = make([(300, [301, 400, 310]), (40, [50, 60])], 1, 4, 2, 64, seed=9, way=way)
    q, pool, table, lens, starts, shared = args
    good = sv.shared_attention(*args)

    def run(bit, **kw):
        a = {"q": q, "pool": pool, "table": table, "lens": lens, "groups": starts, "shared": shared, **kw}
        got = sv.shared_attention(**a)
        with pytest.raises(Exception, match=f"flags {bit}$"):
            sv.status()
        return got

    for bad_id in (-1, len(pool), 1 << 30, -5):
        bad = table.clone()
        bad[0, 4] = bad_id                                    # of the first group's prefix: unseen by all of it (or by the first)
        got = run(2, table=bad)
        assert torch.equal(got[3:], good[3:]) and torch.isfinite(got).all() and not torch.equal(got[0], good[0])
        assert all(torch.equal(got[i], good[i]) == (way == "paged") for i in (1, 2))
        bad = table.clone()
        bad[4, 3] = bad_id                                    # of a sequence's own
        got = run(2, table=bad)
        assert torch.equal(got[:4], good[:4]) and torch.isfinite(got).all()
    for kw in (dict(shared=i32([-1, 40])), dict(shared=i32([300, 1 << 30])), dict(groups=i32([0, 7, 5])), dict(groups=i32([1, 3, 5])),
               dict(groups=i32([0, 3, 4])), dict(groups=i32([0, -9, 5])), dict(groups=i32([0, 4, 3])), dict(lens=i32([301, 400, -1, 50, 60]))):
        if way == "paged" and "lens" not in kw:
            assert torch.equal(sv.shared_attention(q, pool, table, lens, kw.get("groups", starts), kw.get("shared", shared)), good)
        else:
            run(8, **kw)
    # an unseen page leaves the rest as it is: against keys cut out by hand
    one = make([(64, [70, 71])], 1, 2, 1, 64, seed=10, way=way)
    bad = one[2].clone()
    bad[:, 1] = -1
    got = sv.shared_attention(one[0], one[1], bad, *one[3:])
    with pytest.raises(Exception, match="flags 2$"):
        sv.status()
    for b, n in ((0, 70), (1, 71)):
        at = torch.tensor([x for x in range(n) if not 16 <= x < 32], device="cuda")
        kv = one[1][one[2][b, at // 16].long(), :, 0, at % 16].double()
        w = torch.softmax(one[0][b, 0].double() @ kv[:, 0].T / 8, -1) @ kv[:, 1]
        assert (got[b, 0].double() - w).abs().max() <= (2 * 2.0 ** -8 + 2.0 ** -15) * kv[:, 1].abs().max()


@pytest.mark.parametrize("way", WAYS)
def test_captured_and_on_another_stream(sv, way):
    """A captured call follows its lists; two captured graphs with scratch of their own; another stream."""
    args = make([(300, [310 + i for i in range(6)]), (500, [501, 700])], 1, 8, 2, 64, seed=11, way=way)
    q, pool, table, lens, starts, shared = args
    want = sv.shared_attention(*args)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            graphs.append((graph, sv.shared_attention(*args)))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        graphs[0][0].replay()
        other = sv.shared_attention(*args)
    graphs[1][0].replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for x in (graphs[0][1], graphs[1][1], other))
    lens.sub_(i32([3, 3, 3, 3, 3, 3, 0, 100]))
    shared.copy_(i32([200, 480]))
    starts.copy_(i32([0, 6, 8]))
    want = check(sv, *args)
    graphs[0][0].replay()
    assert torch.equal(graphs[0][1], want)


def test_refusals(sv):
    from paper_2606_10820_gb300.kforcing import KfError
    q, pool, table, lens, starts, shared = make([(16, [20, 21]), (5, [6])], 1, 4, 2, 64)
    fine = dict(q=q, pool=pool, table=table, lens=lens, groups=starts, shared=shared)
    for bad in (dict(groups=starts[:2]), dict(groups=starts.long()), dict(shared=shared.cpu()), dict(shared=shared[None]), dict(lens=lens[:2]),
                dict(table=table[:2]), dict(pool=pool.half()), dict(q=q[0]), dict(out=q[:1]), dict(q=q.float())):
        with pytest.raises(ValueError):
            sv.shared_attention(**{**fine, **bad})
    for bad in (dict(scale=0.0), dict(scale=math.inf), dict(q=torch.zeros(3, 1, 5, 64, device="cuda", dtype=q.dtype)),
                dict(groups=starts[:1], shared=shared[:0])):
        with pytest.raises(KfError):
            sv.shared_attention(**{**fine, **bad})
    with pytest.raises(ValueError):
        sv.shared_attention(**{**fine, "q": q.clone().requires_grad_()})
    none = sv.shared_attention(q[:0], pool, table[:0], lens[:0], starts[:1], shared[:0])
    assert none.shape == (0, 1, 4, 64)


@pytest.mark.parametrize("way", WAYS)
def test_a_pool_past_32_bits(sv, way):
    """Pages whose elements lie past 2^31 (and bytes past 2^32) in the pool."""
    args = list(make([(70, [71, 90, 75]), (33, [40])], 1, 32, 8, 128, seed=12, way=way))
    small, table = args[1], args[2]
    big = torch.empty(max(70000, len(small) + 66000), 2, 8, 16, 128, dtype=torch.bfloat16, device="cuda")       # 4.6 GB
    big[-len(small):] = small
    if way == "paged":
        table = table[:, :8].contiguous()
    args[1], args[2] = big, torch.where(table >= 0, table + (len(big) - len(small)), table)
    got = sv.shared_attention(*args)
    sv.status()
    want, top = plain(*args)
    assert ((got.double() - want).abs().amax((1, 2, 3)) <= (2 * 2.0 ** -8 + 2.0 ** -15) * top).all()

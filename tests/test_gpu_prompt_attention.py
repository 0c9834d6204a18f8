"""prompt_attention against plain causal attention in 64 bits (needs a GB300).

Tolerance, before any run: an output row is a convex combination of V rows with
probabilities rounded to the inputs' type (u = 2^-9 bf16, 2^-12 fp16 relative; the sum uses the
unrounded ones), scores and sums in fp32, and the output rounded once more (u |out|):
|out - ref| <= 2.2 u max|V| + 2^-15 max|V| (max over the row's keys' sequence).
"""
import math
import random

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


def make(lens, Hq, Hkv, hd, dtype=torch.bfloat16, seed=0, std=1.0, fused=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    T = sum(lens)
    x = torch.randn(T, Hq + 2 * Hkv, hd, generator=g, device="cuda")
    x[:, :Hq] *= std
    q, k, v = x.to(dtype).split([Hq, Hkv, Hkv], 1)
    if not fused:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    starts = [0]
    for n in lens:
        starts.append(starts[-1] + n)
    return q, k, v, torch.tensor(starts, dtype=torch.int32, device="cuda")


def plain_seq(q, k, v, scale):
    """One sequence in 64 bits, head by head."""
    n, Hq, hd = q.shape
    G = Hq // k.shape[1]
    out = torch.empty(n, Hq, hd, dtype=torch.float64, device=q.device)
    for h in range(Hq):
        w = (q[:, h].double() @ k[:, h // G].double().T) * scale
        w.masked_fill_(torch.ones(n, n, dtype=torch.bool, device=q.device).triu(1), -math.inf)
        out[:, h] = torch.softmax(w, 1) @ v[:, h // G].double()
    return out


def check(sv, q, k, v, starts, longest=None, scale=None, got=None):
    st = starts.tolist()
    if got is None:
        got = sv.prompt_attention(q, k, v, starts, longest or max(b - a for a, b in zip(st, st[1:])), scale=scale)
    assert torch.isfinite(got).all()
    for a, b in zip(st, st[1:]):
        if a == b:
            continue
        ref = plain_seq(q[a:b], k[a:b], v[a:b], scale or 1 / math.sqrt(q.shape[2]))
        err, big = (got[a:b].double() - ref).abs().max(), v[a:b].abs().max().double()
        assert err <= (2.2 * U[q.dtype] + 2.0 ** -15) * big, (a, b, (err / big).item())
    sv.status()
    return got


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("lens,Hq,Hkv", [
    ([1], 1, 1), ([2, 1, 1], 2, 1), ([127, 128, 129], 2, 2), ([255, 256, 257, 0, 1], 3, 1), ([64, 65], 4, 2), ([300, 33, 5, 700], 6, 2),
    ([1000], 12, 4), ([511, 513], 5, 5), ([0, 0, 40, 0], 8, 2), ([1] * 200, 2, 1), ([2311, 17], 4, 1), ([90] * 37, 7, 1),
])
def test_matches_plain(sv, hd, dtype, lens, Hq, Hkv):
    check(sv, *make(lens, Hq, Hkv, hd, dtype, seed=sum(lens) + Hq))


@pytest.mark.parametrize("seed", range(4))
def test_random_batches(sv, seed):
    rng = random.Random(seed)
    hkv = rng.choice([1, 2, 3])
    lens = [rng.randint(0, rng.choice([3, 200, 900])) for _ in range(rng.choice([9, 60, 400]))]
    check(sv, *make(lens, hkv * rng.choice([1, 2, 3, 4]), hkv, rng.choice([64, 128]), rng.choice([torch.bfloat16, torch.float16]),
                    seed=seed, fused=bool(seed % 2)), longest=rng.choice([900, 1000, 5000]))


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(4, 2), (3, 1)])
def test_long(sv, hd, Hq, Hkv):
    check(sv, *make([5003, 4096, 1], Hq, Hkv, hd, seed=hd))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_references_that_rise(sv, dtype):
    """Scores whose maximum grows along the keys by hundreds: every tile raises the reference; and a row
    whose first key takes all."""
    q, k, v, starts = make([900, 300], 4, 2, 64, dtype, seed=4)
    q[:] = 0
    q[..., 0] = 8
    k[:, :, 0] = (torch.arange(1200, device="cuda") % 900).to(dtype)[:, None] / 8
    check(sv, q, k, v, starts)
    k[:, :, 0] = -k[:, :, 0]
    check(sv, q, k, v, starts)
    check(sv, *make([700, 90], 4, 2, 128, dtype, std=40.0, seed=5))
    check(sv, *make([700, 90], 4, 2, 128, dtype, seed=6), scale=0.29)


def test_strides(sv):
    """Heads first in memory, token strides wider than the heads, an output within a wider array."""
    q, k, v, starts = make([200, 131], 4, 2, 64, seed=7)
    want = sv.prompt_attention(q, k, v, starts, 200)
    t = lambda x: x.transpose(0, 1).contiguous().transpose(0, 1)  # noqa: E731
    assert torch.equal(sv.prompt_attention(t(q), t(k), t(v), starts, 200), want)
    wide = torch.full((331, 9, 64), 3.0, device="cuda", dtype=q.dtype)
    sv.prompt_attention(q, k, v, starts, 200, out=wide[:, 2:6])
    assert torch.equal(wide[:, 2:6], want) and (wide[:, :2] == 3).all() and (wide[:, 6:] == 3).all()


def test_far_rows(sv):
    """Token strides that pass 2^31 elements within the call."""
    T, stride = 2500, 1 << 20
    buf = torch.zeros(T * stride, device="cuda", dtype=torch.bfloat16)           # 5.2 GB
    wide = buf.view(T, stride // 64, 64)
    q, k, v, starts = make([700, 1800], 4, 2, 64, seed=11)
    parts = [wide[:, 0:4], wide[:, 4:6], wide[:, 6:8], wide[:, 100:104]]
    for x, y in zip(parts, (q, k, v)):
        x.copy_(y)
    sv.prompt_attention(*parts[:3], starts, 1800, out=parts[3])
    assert torch.equal(parts[3], sv.prompt_attention(q, k, v, starts, 1800))


def test_what_is_not_a_number_stays_in_its_sequence(sv):
    """NaN and infinity in K, V and Q of a neighbour, and past the end of the tokens."""
    lens = [70, 130, 200, 129]
    q, k, v, starts = make(lens, 4, 2, 128, seed=8)
    want = sv.prompt_attention(q, k, v, starts, 200)
    for x, bad in ((k, math.nan), (v, math.nan), (v, math.inf), (q, math.nan), (k, math.inf)):
        y = x.clone()
        y[70:200] = bad
        y[400:] = bad
        args = [y if z is x else z for z in (q, k, v)]
        got = sv.prompt_attention(*args, starts, 200)
        assert torch.equal(got[:70], want[:70]) and torch.equal(got[200:400], want[200:400])
        assert not torch.isfinite(got[70:200].float()).all()
    # a key that is not a number: the rows before it are as they were
    y = k.clone()
    y[200 + 150] = math.nan
    got = sv.prompt_attention(q, y, v, starts, 200)
    assert torch.equal(got[:350], want[:350]) and torch.isnan(got[350:400]).all()


def test_repeats_streams_graphs(sv):
    q, k, v, starts = make([333, 140, 1000], 6, 2, 64, seed=6)
    want = check(sv, q, k, v, starts)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = [sv.prompt_attention(q, k, v, starts, 1000) for _ in range(3)]
    s.synchronize()
    assert all(torch.equal(x, want) for x in got)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = sv.prompt_attention(q, k, v, starts, 1000)
    starts.copy_(torch.tensor([0, 700, 703, 1473], dtype=torch.int32))
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        check(sv, q, k, v, starts, got=out)


def test_bad_starts(sv):
    from paper_2606_10820_gb300.kforcing import KfError
    q, k, v, starts = make([100, 50], 2, 1, 64)
    for bad in ([0, 100, 151], [0, 100, 149], [0, 120, 100], [1, 100, 150], [0, 150, 150], [-5, 100, 150], [0, 1 << 30, 150]):
        out = torch.full((150, 2, 64), 7.0, device="cuda", dtype=q.dtype)
        sv.prompt_attention(q, k, v, torch.tensor(bad, dtype=torch.int32, device="cuda"), 100, out=out)
        with pytest.raises(KfError, match="flags 8$"):
            sv.status()
        assert (out == 7).all()
    check(sv, q, k, v, starts)


def test_refusals(sv):
    from paper_2606_10820_gb300.kforcing import KfError
    q, k, v, starts = make([100, 50], 4, 2, 64)
    for call in (lambda: sv.prompt_attention(q[..., :32].contiguous(), k[..., :32].contiguous(), v[..., :32].contiguous(), starts, 100),
                 lambda: sv.prompt_attention(q[:, :3], k, v, starts, 100), lambda: sv.prompt_attention(q, k, v, starts, -1),
                 lambda: sv.prompt_attention(q, k, v, starts, 1 << 20), lambda: sv.prompt_attention(q, k, v, starts, 100, scale=-1.0),
                 lambda: sv.prompt_attention(q, k, v, starts[:1], 100)):
        with pytest.raises(KfError):
            call()
    for call in (lambda: sv.prompt_attention(q.float(), k.float(), v.float(), starts, 100), lambda: sv.prompt_attention(q, k.half(), v, starts, 100),
                 lambda: sv.prompt_attention(q, k, v[:1], starts, 100), lambda: sv.prompt_attention(q, k, v, starts.long(), 100),
                 lambda: sv.prompt_attention(q, k, v, starts.cpu(), 100), lambda: sv.prompt_attention(q.transpose(1, 2), k, v, starts, 100)):
        with pytest.raises(ValueError):
            call()
    assert sv.prompt_attention(q[:0], k[:0], v[:0], starts[:1], 0).shape == (0, 4, 64)
    sv.status()

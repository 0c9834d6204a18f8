"""token_scores and token_scores_grad against plain 64-bit formulas (needs a GB300).

Tolerances, before any run.  The numbers are fp32 sums against the row's maximum: exp has
a relative error of about 2^-22 plus that of its argument, |x - m| 2^-24 (|x - m| <= 100 where exp
matters: 6e-6), so S and T / S are within 1e-5 relative, lse and logp within 1e-5 + |x| 2^-22,
the entropy within 1e-5 (1 + its T / S <= log V).  2e-5 (1 + |value|) covers them.  A
gradient is p times a number of the size of c = |g_logp| + |g_entropy| (1 + |lp| + H): 3e-5 of
p c / tau in fp32, plus the output's own rounding (2^-9 bf16, 2^-12 fp16 relative, and half
of the least subnormal).
"""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
EPS = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 1e-38, torch.bfloat16: 1e-38, torch.float16: 2.0 ** -24}


@pytest.fixture(scope="module")
def sv():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__ as g
    g.build()
    from paper_2606_10820_gb300 import serving
    return serving


def formulas(logits, tokens, tau, gl=None, gh=None):
    x = (logits.float() * (1.0 / torch.tensor(tau, dtype=torch.float32))).double()
    closed = torch.isneginf(x)
    empty = closed.all(1)
    # (against the maximum: a lowest value of -3e38 would swallow the logarithm)
    m = torch.where(empty, 0.0, x.amax(1))
    logs = torch.log(torch.where(closed, 0.0, (x - m[:, None]).exp()).sum(1))
    lse = m + logs
    lp = torch.where(closed, -math.inf, (x - m[:, None]) - torch.where(empty, 0.0, logs)[:, None])
    p = lp.exp()
    plp = torch.where(closed, 0.0, p * torch.where(closed, 0.0, lp))
    H = -plp.sum(1)
    has = tokens >= 0
    logp = torch.where(has, lp.gather(1, tokens.clamp(min=0)[:, None])[:, 0], 0.0)
    out = {"logp": logp, "entropy": H, "lse": lse, "x": x, "p": p, "lp": lp}
    if gl is not None:
        a = torch.where(has, gl.double(), 0.0)[:, None]
        d = -a * p - gh.double()[:, None] * (plp + p * H[:, None])
        d.scatter_add_(1, tokens.clamp(min=0)[:, None], a)
        out["grad"] = d / tau
    return out


def near(got, want):
    want = want.to(got.device)
    fin = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got[~fin & ~torch.isnan(want)].double(), want[~fin & ~torch.isnan(want)])
    err = (got.double() - want).abs()[fin]
    assert (err <= 2e-5 * (1 + want.abs()[fin])).all(), err.max().item()


def check_top(got, ref, top):
    # a stable sort of the same fp32 values: largest first, then lowest id
    v, i = ref["x"].float().sort(dim=-1, descending=True, stable=True)
    assert torch.equal(got["top_ids"].long(), i[:, :top])
    near(got["top_logp"], ref["lp"].gather(1, i[:, :top]))


def rows(R, V, dtype, seed, std=3.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (torch.randn(R, V, device="cuda", generator=g) * std).to(dtype)
    tok = torch.randint(0, V, (R,), device="cuda", generator=g)
    return x, tok, torch.randn(R, device="cuda", generator=g), torch.randn(R, device="cuda", generator=g) * 0.3


SHAPES = [(1, 1), (3, 2), (5, 7), (2, 33), (4, 511), (7, 1000), (3, 4097), (2, 8200), (40, 16411), (37, 30522),
          (1, 50257), (39, 50257), (90, 50257), (300, 50257), (2, 130001)]


@pytest.mark.parametrize("R,V", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("tau", [1.0, 0.7])
def test_scores(sv, R, V, dtype, tau):
    x, tok, _, _ = rows(R, V, dtype, R * 7 + V)
    if R > 2:
        tok[1] = -1
    for top in sorted({0, 1, min(5, V), min(20, V), min(64, V)}):
        got = sv.token_scores(x, tok, top=top, tau=tau)
        ref = formulas(x, tok, tau)
        for k in ("logp", "entropy", "lse"):
            near(got[k], ref[k])
        if top:
            check_top(got, ref, top)
        else:
            assert "top_ids" not in got
    sv.status()


def grad_near(got, ref, gl, gh, tau, dtype):
    lp = torch.where(torch.isneginf(ref["lp"]), 0.0, ref["lp"])
    size = (gl.abs()[:, None] + gh.abs()[:, None] * (1 + lp.abs() + ref["entropy"][:, None]))
    bound = 3e-5 * ref["p"] * size / tau + EPS[dtype] * ref["grad"].abs() + TINY[dtype]
    # the token's own entry is a difference from g_logp
    bound += 3e-5 * (ref["grad"].abs() + (ref["p"] * size) / tau)
    err = (got.double() - ref["grad"]).abs()
    assert (err <= bound).all(), (err - bound).max().item()


@pytest.mark.parametrize("R,V", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_gradient(sv, R, V, dtype):
    x, tok, gl, gh = rows(R, V, dtype, R * 11 + V)
    if R > 2:
        tok[1] = -1
    for tau in (1.0, 1.3):
        ref = formulas(x, tok, tau, gl, gh)
        got = sv.token_scores_grad(x, tok, gl, gh, tau=tau)
        for k in ("logp", "entropy", "lse"):
            near(got[k], ref[k])
        grad_near(got["grad"], ref, torch.where(tok >= 0, gl, 0.0), gh, tau, dtype)
    # over the logits themselves: the same bits
    y = x.clone()
    assert sv.token_scores_grad(y, tok, gl, gh, tau=1.3, out=y)["grad"] is y
    assert torch.equal(y, got["grad"])
    sv.status()


def test_gradient_against_differences(sv):
    """d loss / d logit by central differences of the 64-bit loss of the fp32 operator's own scores: a
    step of 1e-2 leaves h^2 / 6 f''' <= 1e-4 and rounding 2 * 4e-5 / 2e-2 = 4e-3 of a loss of O(1)."""
    x, tok, gl, gh = rows(3, 40, torch.float32, 5, std=1.0)
    tok[2] = -1
    grad = sv.token_scores_grad(x, tok, gl, gh)["grad"]
    h = 1e-2

    def loss(z):
        o = sv.token_scores(z, tok)
        return o["logp"].double() * torch.where(tok >= 0, gl, 0.0) + o["entropy"].double() * gh

    for v in range(40):
        up, dn = x.clone(), x.clone()
        up[:, v] += h
        dn[:, v] -= h
        d = (loss(up) - loss(dn)) / ((up - dn)[:, v].double())
        assert (d - grad[:, v]).abs().max() <= 1e-2


@pytest.mark.parametrize("R", [6, 200])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_closed_tokens(sv, R, dtype):
    """-inf and the type's lowest value as masks, rows with few, one or no open token."""
    V = 9000
    x, tok, gl, gh = rows(R, V, dtype, 3)
    low = torch.finfo(dtype).min
    x[0, 5:] = -math.inf
    x[1, :] = -math.inf
    x[2, :] = low
    x[3, 1:] = low
    x[4, : V - 3] = -math.inf
    x[5, 100:] = -math.inf
    tok[:6] = torch.tensor([2, 7, 9, 0, 4, 200], device="cuda")
    ref = formulas(x, tok, 1.0, gl, gh)
    got = sv.token_scores(x, tok, top=8)
    for k in ("logp", "entropy", "lse"):
        near(got[k], ref[k])
    check_top(got, ref, 8)
    g = sv.token_scores_grad(x, tok, gl, gh)
    ref["grad"][1] = 0.0          # a row without open tokens
    fine = torch.arange(R, device="cuda") != 5
    # (row 5's token is closed: logp -inf, its gradient the formula's)
    assert got["logp"][5] == -math.inf and fine.sum() == R - 1
    grad_near(g["grad"], ref, gl, gh, 1.0, dtype)
    assert (g["grad"][1] == 0).all()
    sv.status()


@pytest.mark.parametrize("R", [4, 200])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_ties_and_orders(sv, R, dtype):
    """Constant rows, few distinct values, sorted rows: more candidates than the list holds."""
    V = 20011
    x = torch.zeros(R, V, device="cuda", dtype=dtype)
    x[1] = (torch.arange(V, device="cuda") % 3).to(dtype)
    x[2] = torch.linspace(30, -30, V, device="cuda").to(dtype)
    x[3] = torch.linspace(-30, 30, V, device="cuda").to(dtype)
    tok = torch.arange(R, device="cuda")
    for top in (1, 5, 64):
        got = sv.token_scores(x, tok, top=top)
        check_top(got, formulas(x, tok, 1.0), top)


@pytest.mark.parametrize("R,V", [(3, 9001), (3, 50257), (70, 50257), (640, 18003)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_masks_of_the_lowest_value(sv, R, V, dtype):
    """A few open tokens, all others at the type's lowest value: thousands tie at the bound.  And a
    staircase, where more than the list holds stand above any first bound."""
    x, tok, _, _ = rows(R, V, dtype, 17)
    low = torch.finfo(dtype).min
    x[0, 11:] = low
    x[1] = low
    x[1, V - 2:] = 1.0
    x[2] = low
    x[2, ::64 * 8] = torch.arange(x[2, ::64 * 8].numel(), device="cuda").to(dtype)      # few threads hold what is open
    if R > 3:
        x[3:, 20:] = low
        x[4] = -math.inf
        x[4, :3000] = (torch.arange(3000, device="cuda") // 4).to(dtype)
        x[5, 2000:] = -math.inf
    ref = formulas(x, tok, 1.0)
    for top in (1, 8, 48, 49, 64):
        got = sv.token_scores(x, tok, top=top)
        check_top(got, ref, top)
        near(got["lse"], ref["lse"])
    sv.status()


@pytest.mark.parametrize("V", [50, 50257])
def test_not_numbers(sv, V):
    x, tok, gl, gh = rows(5, V, torch.float32, 1)
    x[0, V - 1] = math.nan
    x[1, 3] = math.inf
    x[2] = math.nan
    tok[2] = -1
    got = sv.token_scores(x, tok, top=4)
    grad = sv.token_scores_grad(x, tok, gl, gh)["grad"]
    for r in range(3):
        assert math.isnan(got["entropy"][r]) and math.isnan(got["lse"][r])
        assert (got["top_ids"][r] == -1).all() and torch.isnan(got["top_logp"][r]).all()
        assert torch.isnan(grad[r]).all()
    assert math.isnan(got["logp"][0]) and math.isnan(got["logp"][1]) and got["logp"][2] == 0
    ref = formulas(x[3:], tok[3:], 1.0)
    near(got["logp"][3:], ref["logp"])
    assert torch.isfinite(grad[3:]).all()


@pytest.mark.parametrize("V", [1, 2, 33, 130, 1000, 4097, 6144, 8200, 16411, 24500, 50257])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_many_rows(sv, V, dtype):
    """More rows than one wave of CTAs (which take other shapes then), ordinary ones between masked,
    tied and broken ones; the odd widths start rows at every alignment."""
    R = 700
    x, tok, gl, gh = rows(R, V, dtype, V + 5)
    x[::7, V // 3 + 1:] = -math.inf
    x[1::7, V // 2 + 1:] = torch.finfo(dtype).min
    x[2::7] = (torch.arange(V, device="cuda") % 3).to(dtype)
    tok[::7] = 0
    tok[3::7] = -1
    dead, broken = list(range(4, R, 70)), list(range(5, R, 70))
    x[dead] = -math.inf
    x[broken, V - 1] = math.nan
    fine = torch.ones(R, dtype=torch.bool, device="cuda")
    fine[broken] = False
    ref = formulas(x[fine], tok[fine], 1.0, gl[fine], gh[fine])
    for top in sorted({0, 1, min(8, V), min(64, V)}):
        got = sv.token_scores(x, tok, top=top)
        assert torch.isnan(got["lse"][broken]).all() and torch.isnan(got["entropy"][broken]).all()
        good = {k: v[fine] for k, v in got.items()}
        for k in ("logp", "entropy", "lse"):
            near(good[k], ref[k])
        if top:
            check_top(good, ref, top)
            assert (got["top_ids"][broken] == -1).all()
    got = sv.token_scores_grad(x, tok, gl, gh)
    assert torch.isnan(got["grad"][broken]).all()
    assert (got["grad"][dead] == 0).all()
    none = torch.isneginf(ref["lse"])
    ref["grad"][none] = 0.0       # rows without open tokens
    grad_near(got["grad"][fine], ref, torch.where(tok >= 0, gl, 0.0)[fine], gh[fine], 1.0, dtype)
    sv.status()


def test_strides_streams_and_repeats(sv):
    """Rows of a wider array at odd offsets, another stream, twice the same bits."""
    x, tok, gl, gh = rows(9, 5003, torch.bfloat16, 2)
    wide = torch.full((9, 5003 + 10), 50.0, device="cuda", dtype=torch.bfloat16)
    part = wide[:, 3:5006]
    part.copy_(x)
    want, wg = sv.token_scores(x, tok, top=6), sv.token_scores_grad(x, tok, gl, gh)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got, gg = sv.token_scores(part, tok, top=6), sv.token_scores_grad(part, tok, gl, gh)
    torch.cuda.current_stream().wait_stream(s)
    ref = formulas(x, tok, 1.0)
    for k in ("logp", "entropy", "lse"):
        near(got[k], ref[k])
    assert torch.equal(got["top_ids"], want["top_ids"])
    again = sv.token_scores(x, tok, top=6)
    assert all(torch.equal(again[k], want[k]) for k in want)
    assert (wide[:, :3] == 50).all() and (wide[:, 5006:] == 50).all()
    # a gradient into a part of a wider array leaves the rest alone
    sv.token_scores_grad(x, tok, gl, gh, out=part)
    assert torch.equal(part, wg["grad"]) and (wide[:, :3] == 50).all() and (wide[:, 5006:] == 50).all()


def test_far_rows(sv):
    """Offsets past 2^31 elements."""
    V, stride = 1000, 1 << 29
    buf = torch.zeros(5 * stride + V, device="cuda", dtype=torch.bfloat16)
    x = buf.as_strided((6, V), (stride, 1))
    g = torch.Generator(device="cuda").manual_seed(1)
    x.copy_(torch.randn(6, V, device="cuda", generator=g))
    tok = torch.arange(6, device="cuda")
    near(sv.token_scores(x, tok)["logp"], formulas(x, tok, 1.0)["logp"])


def test_refusals(sv):
    from paper_2606_10820_gb300.kforcing import KfError
    x, tok, gl, _ = rows(4, 100, torch.float32, 1)
    for bad in (dict(tau=0.0), dict(tau=-1.0), dict(tau=math.nan), dict(tau=1e-45), dict(tau=math.inf)):
        with pytest.raises(KfError):
            sv.token_scores(x, tok, **bad)
    for call in (lambda: sv.token_scores(x, tok, top=65), lambda: sv.token_scores(x[:, :3], tok, top=4),
                 lambda: sv.token_scores(x, tok[:3]), lambda: sv.token_scores(x, tok.int()),
                 lambda: sv.token_scores(x.t(), tok), lambda: sv.token_scores(x.double(), tok),
                 lambda: sv.token_scores(x.cpu(), tok), lambda: sv.token_scores_grad(x, tok, gl[:2]),
                 lambda: sv.token_scores_grad(x, tok, gl, out=x[:2])):
        with pytest.raises(ValueError):
            call()
    assert sv.token_scores(x[:0], tok[:0])["logp"].shape == (0,)
    sv.status()
    tok[1] = 100
    got = sv.token_scores(x, tok)
    assert math.isnan(got["logp"][1]) and math.isfinite(got["entropy"][1])
    with pytest.raises(KfError):
        sv.status()
    sv.status()

"""policy_loss against plain 64-bit formulas (needs a GB300).

Tolerances, before any run.  A term 2^d of S has d rounded at 2^-24 |d| (|d| <= 60 where a term counts: 2.5e-6 relative)
and the unit's 2^-22; a chain of at most 100 terms and the joins add 110 2^-24: lse is within 1e-5, and so is lp (the
token's own difference is kept in two parts; its last rounding is 2^-24 |lp|): L = 1e-5 + 2^-23 |lp|.  H: 2e-5 (1 + H), as of
token_scores.  ratio: 1.1 L ratio + 2^-22 ratio, the difference lp - old adding 2^-23 |lp - old| to L.  kl: |e^u - 1| L +
2^-21 (kl + |u e^u - u|).  loss: its terms' tolerances times their weights.  grad = p c / tau with c = |gl| + |gh| (1 + |lp| + H): 3e-5 p c / tau (the
two passes' exponents), plus p times the tolerance of gl, plus the output's rounding and half of the least subnormal.
"""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
TINY = {torch.float32: 1e-37, torch.bfloat16: 1e-37, torch.float16: 2.0 ** -25}
ROWS = ("loss", "logp", "entropy", "ratio", "kl")


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


def formulas(logits, tokens, old, adv, ref=None, weight=None, clip=(0.2, 0.2), klw=0.0, hw=0.0, tau=1.0):
    """The definition in 64 bits; rows that the loss leaves out are zeros."""
    x = logits.double() / tau
    lp = torch.log_softmax(x, 1)
    p = lp.exp()
    plp = torch.special.xlogy(p, p)
    H = -plp.sum(1)
    has, at = tokens >= 0, tokens.clamp(min=0)[:, None]
    w = torch.ones(len(x), device=x.device, dtype=torch.float64) if weight is None else weight.double()
    logp = lp.gather(1, at)[:, 0]
    ratio = (logp - old.double()).exp()
    A = adv.double()
    u = (ref.double() if ref is not None else logp.detach()) - logp
    kl = torch.expm1(u) - u
    gain = torch.minimum(ratio * A, ratio.clamp(1 - clip[0], 1 + clip[1]) * A)
    inside = has & (w != 0)
    loss = torch.where(inside, w * ((klw * kl if klw else 0) - gain - (hw * H if hw else 0)), 0.0)
    return {"loss": loss, "logp": torch.where(has, logp, 0.0), "entropy": H, "ratio": torch.where(has, ratio, 1.0),
            "kl": torch.where(has, kl, 0.0), "p": p, "lp": lp, "u": u, "A": A, "w": w, "inside": inside}


def exact(logits, tokens, old, adv, ref=None, weight=None, clip=(0.2, 0.2), klw=0.0, hw=0.0, tau=1.0):
    """And the gradient, by hand: autograd makes NaN of closed tokens."""
    f = formulas(logits, tokens, old, adv, ref, weight, clip, klw, hw, tau)
    A = f["A"]
    open_ = torch.where(A > 0, f["ratio"] <= 1 + clip[1], f["ratio"] >= 1 - clip[0])
    gl = f["w"] * ((-klw * torch.expm1(f["u"]) if klw else 0) - torch.where(open_, f["ratio"] * A, 0.0))
    gh = -f["w"] * hw
    d = -gl[:, None] * f["p"] - gh[:, None] * (torch.special.xlogy(f["p"], f["p"]) + f["p"] * f["entropy"][:, None])
    d.scatter_add_(1, tokens.clamp(min=0)[:, None], gl[:, None])
    f["grad"] = torch.where(f["inside"][:, None], d / tau, 0.0)
    return f


def test_the_formulas_gradient_is_autograds(sv):
    logits, tokens, old, adv, ref, weight = make(20, 300, seed=11)
    tokens[1], weight[2] = -1, 0
    x = logits.double().requires_grad_()
    formulas(x, tokens, old, adv, ref, weight, (0.2, 0.28), 0.1, 0.02, 0.8)["loss"].sum().backward()
    by_hand = exact(logits, tokens, old, adv, ref, weight, (0.2, 0.28), 0.1, 0.02, 0.8)["grad"]
    assert (x.grad - by_hand).abs().max() < 1e-12


def check(sv, logits, tokens, old, adv, ref=None, weight=None, clip=(0.2, 0.28), klw=0.0, hw=0.0, tau=1.0, out=None):
    f = exact(logits, tokens, old, adv, ref, weight, clip, klw, hw, tau)
    dtype = logits.dtype
    got = sv.policy_loss(logits, tokens, old, adv, ref_logp=ref, weight=weight, clip=clip, kl_weight=klw, entropy_weight=hw, tau=tau, out=out)
    sv.status()
    assert set(got) == {"loss", "logp", "entropy", "ratio", "grad"} | ({"kl"} if ref is not None else set())
    L = 1e-5 + 2.0 ** -23 * f["logp"].abs()
    Lr = L + 2.0 ** -23 * (f["logp"] - old.double()).abs()
    e1 = torch.expm1(f["u"]).abs()
    tol = {"logp": L, "entropy": 2e-5 * (1 + f["entropy"]), "ratio": f["ratio"] * (1.1 * Lr + 2.0 ** -22),
           "kl": e1 * (L + 2.0 ** -23 * f["u"].abs()) + 2.0 ** -21 * (f["kl"] + (f["u"] * e1).abs())}
    tol["loss"] = f["w"].abs() * (abs(klw) * tol["kl"] + tol["ratio"] * f["A"].abs() + abs(hw) * tol["entropy"]
                                  + 2.0 ** -21 * (abs(klw) * f["kl"] + (f["ratio"] + 1) * f["A"].abs() + abs(hw) * f["entropy"]))
    for k in ROWS:
        if k in got:
            assert got[k].dtype == torch.float32
            err = (got[k].double() - f[k]).abs()
            assert (err <= tol[k] + 1e-37).all(), (k, (err / (tol[k] + 1e-37)).max().item())
    gl = f["w"].abs() * (abs(klw) * e1 + f["ratio"] * f["A"].abs())
    dgl = f["w"].abs() * (abs(klw) * (e1 + 1) * L * 1.1 + tol["ratio"] * f["A"].abs()) + 2.0 ** -21 * gl
    gh = (f["w"] * hw).abs()
    lp = torch.where(torch.isinf(f["lp"]), 0.0, f["lp"].abs())
    at = torch.nn.functional.one_hot(tokens.clamp(min=0), logits.shape[1]).bool()
    bound = f["p"] * (3e-5 * (gl[:, None] + gh[:, None] * (1 + lp + f["entropy"][:, None])) + dgl[:, None]) + torch.where(at, dgl[:, None], 0.0)
    err = (got["grad"].double() - f["grad"]).abs()
    bound = bound / tau + u_of(dtype) * f["grad"].abs() + TINY[dtype]
    ok = err <= bound
    assert ok[f["inside"]].all(), (err / bound)[f["inside"]].max().item()
    assert (got["grad"][~f["inside"]] == 0).all() and (got["loss"][~f["inside"]] == 0).all()
    return got, f


def make(R, V, dtype=torch.float32, seed=0, std=3.0, tau=1.0, stride=None, far=0.3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.randn(R, stride or V, generator=g, device="cuda")
    logits = (buf * std).to(dtype)[:, :V]
    tokens = torch.randint(0, V, (R,), generator=g, device="cuda")
    lp = torch.log_softmax(logits.double() / tau, 1).gather(1, tokens[:, None])[:, 0]
    old = (lp + far * torch.randn(R, generator=g, device="cuda")).float()
    # ratios at the clip's ends would leave the side to the last bit
    for end in (0.8, 1.28):
        near = ((lp - old.double()) - math.log(end)).abs() < 1e-3
        old = torch.where(near, old + 2e-3, old)
    ref = (lp + 0.2 * torch.randn(R, generator=g, device="cuda")).float()
    adv = torch.randn(R, generator=g, device="cuda")
    weight = torch.rand(R, generator=g, device="cuda")
    return logits, tokens, old, adv, ref, weight


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("R,V,stride", [(1, 1, None), (3, 2, 5), (1, 8, None), (7, 33, 37), (64, 1000, None), (5, 4099, 4101), (700, 6001, None),
                                        (330, 50257, None), (3, 131072, None), (2, 200003, None), (1300, 257, 264)])
def test_matches_formulas(sv, dtype, R, V, stride):
    logits, tokens, old, adv, ref, weight = make(R, V, dtype, seed=R + V, stride=stride)
    if R > 2:
        tokens[1], weight[2] = -1, 0
    check(sv, logits, tokens, old, adv, ref, weight, klw=0.1, hw=0.02)
    check(sv, logits, tokens, old, adv)
    check(sv, logits, tokens, old, adv, ref, clip=(0.0, 0.0), hw=0.5)


@pytest.mark.parametrize("tau", [0.07, 0.8, 1.3, 12.0])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_temperatures_and_clips(sv, tau, dtype):
    args = make(90, 3001, dtype, seed=int(tau * 10), tau=tau, far=1.0, std=2.0 * min(1, tau))
    logits, tokens, old, adv, ref, weight = args
    check(sv, logits, tokens, old, adv, ref, weight, klw=0.3, hw=0.1, tau=tau)
    check(sv, logits, tokens, old, adv, ref, weight, clip=(1.0, math.inf), klw=0.3, tau=tau)
    got = sv.policy_loss(logits, tokens, old, adv, clip=0.2, tau=tau)
    want = sv.policy_loss(logits, tokens, old, adv, clip=(0.2, 0.2), tau=tau)
    assert all(torch.equal(got[k], want[k]) for k in got)


def test_clip_decides(sv):
    """Each side of both ends under either sign of the advantage: where the clip decides, the ratio's term has no gradient."""
    logits = torch.randn(8, 500, device="cuda", dtype=torch.float32)
    tokens = torch.arange(8, device="cuda")
    lp = torch.log_softmax(logits.double(), 1).gather(1, tokens[:, None])[:, 0]
    want = torch.tensor([0.5, 0.9, 1.1, 1.6] * 2, device="cuda", dtype=torch.float64)
    adv = torch.tensor([1.0] * 4 + [-1.0] * 4, device="cuda")
    got, _ = check(sv, logits, tokens, (lp - want.log()).float(), adv)
    closed = (got["grad"] == 0).all(1)
    assert closed.tolist() == [False, False, False, True, True, False, False, False]


def test_masks(sv):
    """Closed tokens (-inf), masks of the type's lowest value, rows without an open token, NaN and infinities."""
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        logits, tokens, old, adv, ref, weight = make(12, 3000, dtype, seed=4)
        low = torch.finfo(dtype).min
        logits[0, 100:] = -math.inf
        logits[1, 100:] = low
        logits[2, 1:] = -math.inf
        tokens[:3] = torch.tensor([5, 7, 0], device="cuda")
        lp = torch.log_softmax(logits[:3].double(), 1).gather(1, tokens[:3, None])[:, 0]
        old[:3], ref[:3] = (lp + 0.1).float(), (lp - 0.05).float()
        check(sv, logits, tokens, old, adv, ref, weight, klw=0.1, hw=0.02)
        # rows that hold anything, left out by their weight or without a token
        x = logits.clone()
        x[4, 9], x[5, 2999], x[6] = math.nan, math.inf, -math.inf
        x[7, 0] = math.nan
        w, t = weight.clone(), tokens.clone()
        w[4:7], t[7] = 0, -5
        got = sv.policy_loss(x, t, old, adv, ref_logp=ref, weight=w, kl_weight=0.1, entropy_weight=0.1)
        assert (got["loss"][4:8] == 0).all() and (got["grad"][4:8] == 0).all()
        assert torch.isnan(got["entropy"][[4, 5, 7]]).all() and got["logp"][7] == 0 and got["ratio"][7] == 1 and got["kl"][7] == 0
        # and the same rows in the loss
        got = sv.policy_loss(x, tokens, old, adv, ref_logp=ref, kl_weight=0.1, entropy_weight=0.1)
        for r in (4, 5, 7):
            assert all(torch.isnan(got[k][r]) for k in ROWS) and torch.isnan(got["grad"][r]).all()
        assert (got["grad"][6] == 0).all() and got["logp"][6] == -math.inf and got["entropy"][6] == 0
        # a closed token: ratio 0; without a KL term its row is plain
        x = logits.clone()
        x[0, 5] = -math.inf
        got = sv.policy_loss(x, tokens, old, adv.abs(), ref_logp=ref, entropy_weight=0.1)
        assert got["ratio"][0] == 0 and got["kl"][0] == math.inf and torch.isfinite(got["grad"]).all() and torch.isfinite(got["loss"]).all()
        assert sv.policy_loss(x, tokens, old, adv, ref_logp=ref, kl_weight=0.1)["loss"][0] == math.inf
        sv.status()


def test_overflowing_ratio_of_a_row_left_out(sv):
    logits, tokens, old, adv, ref, weight = make(4, 300, seed=2)
    old[1], ref[1], weight[1] = -1e4, 1e4, 0
    got = sv.policy_loss(logits, tokens, old, -adv.abs(), ref_logp=ref, weight=weight, kl_weight=0.1)
    assert got["ratio"][1] == math.inf and got["loss"][1] == 0 and (got["grad"][1] == 0).all() and torch.isfinite(got["loss"]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("R,V", [(5, 50257), (400, 3001), (1, 100003)])
def test_over_the_logits_and_strided(sv, dtype, R, V):
    logits, tokens, old, adv, ref, weight = make(R, V, dtype, seed=R)
    want, _ = check(sv, logits, tokens, old, adv, ref, weight, klw=0.1, hw=0.1)
    buf = torch.zeros(R, V + 9, device="cuda", dtype=dtype)
    got, _ = check(sv, logits, tokens, old, adv, ref, weight, klw=0.1, hw=0.1, out=buf[:, 3:V + 3])
    assert torch.equal(got["grad"], want["grad"]) and (buf[:, :3] == 0).all() and (buf[:, V + 3:] == 0).all()
    before = logits._version
    got = sv.policy_loss(logits, tokens, old, adv, ref_logp=ref, weight=weight, clip=(0.2, 0.28), kl_weight=0.1, entropy_weight=0.1, out=logits)
    assert got["grad"].data_ptr() == logits.data_ptr() and logits._version > before
    assert all(torch.equal(got[k], want[k]) for k in want)


def test_against_differences_and_scores_grad(sv):
    """The gradient along a direction against differences of the kernel's own losses: 2^-21 of their sizes (sum of |loss| below 10)
    over 2 h, and the third derivative's h^2 / 6 (all derivatives here below 10 in size).  And against token_scores_grad with the same row weights."""
    h = 0.02
    logits, tokens, old, adv, ref, weight = make(12, 50, seed=6, std=1.0, far=0.1)
    # (ratios that stay on their side of the clip over the step)
    how = dict(ref_logp=ref, weight=weight, clip=(0.9, 3.0), kl_weight=0.2, entropy_weight=0.1)
    g = torch.Generator(device="cuda").manual_seed(1)
    d = torch.randn(12, 50, generator=g, device="cuda")
    got = sv.policy_loss(logits, tokens, old, adv, **how)
    up, down = (sv.policy_loss(logits + x * d, tokens, old, adv, **how)["loss"].double() for x in (h, -h))
    by = (up - down) / (2 * h)
    along = (got["grad"] * d).double().sum(1)
    assert ((along - by).abs() <= 12 * 2.0 ** -20 / (2 * h) + h * h / 6 * 10 * d.abs().amax(1) ** 3).all(), (along - by).abs().max().item()
    f = exact(logits, tokens, old, adv, ref, weight, (0.9, 3.0), 0.2, 0.1)
    gl = (f["w"] * (-0.2 * torch.expm1(f["u"]) - f["ratio"] * f["A"])).float()
    same = sv.token_scores_grad(logits, tokens, gl, (-0.1 * f["w"]).float())
    assert ((same["grad"] - got["grad"]).abs() <= 1e-4 * f["p"] * (gl.abs()[:, None] + 1) + 1e-5).all()


def test_bad_tokens(sv):
    logits, tokens, old, adv, ref, weight = make(6, 1000, seed=1)
    want = sv.policy_loss(logits, tokens, old, adv, ref_logp=ref, kl_weight=0.1)
    tokens[3] = 1000
    got = sv.policy_loss(logits, tokens, old, adv, ref_logp=ref, kl_weight=0.1)
    with pytest.raises(Exception, match="flags 1$"):
        sv.status()
    assert all(torch.isnan(got[k][3]) for k in ("loss", "logp", "ratio", "kl")) and (got["grad"][3] == 0).all()
    rest = [0, 1, 2, 4, 5]
    assert all(torch.equal(got[k][rest], want[k][rest]) for k in got)


def test_captured(sv):
    logits, tokens, old, adv, ref, weight = make(200, 4001, torch.bfloat16, seed=3)
    logits = logits.contiguous()
    how = dict(ref_logp=ref, weight=weight, kl_weight=0.1, entropy_weight=0.01)
    sv.policy_loss(logits, tokens, old, adv, **how)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = sv.policy_loss(logits, tokens, old, adv, **how)
    logits.copy_(torch.randn(200, 4001, device="cuda"))
    graph.replay()
    want = sv.policy_loss(logits, tokens, old, adv, **how)
    assert all(torch.equal(y[k], want[k]) for k in want)


def test_refusals(sv):
    from paper_2606_10820_gb300.kforcing import KfError
    logits, tokens, old, adv, ref, weight = make(4, 100)
    fine = dict(logits=logits, tokens=tokens, old_logp=old, advantage=adv)
    for bad in (dict(old_logp=old.double()), dict(advantage=adv[:3]), dict(tokens=tokens.int()), dict(weight=weight.cpu()), dict(ref_logp=ref[None]),
                dict(clip=("x", 1.0)), dict(logits=logits.double()), dict(out=logits[:3]), dict(old_logp=old.clone().requires_grad_()),
                dict(advantage=None), dict(old_logp=None)):
        with pytest.raises((ValueError, TypeError)):
            sv.policy_loss(**{**fine, **bad})
    for bad in (dict(clip=(-0.1, 0.2)), dict(clip=(1.1, 0.2)), dict(clip=(0.1, -0.2)), dict(clip=math.nan), dict(kl_weight=0.1), dict(tau=0.0),
                dict(tau=-1.0), dict(tau=math.nan), dict(entropy_weight=math.inf), dict(kl_weight=math.nan, ref_logp=ref)):
        with pytest.raises(KfError):
            sv.policy_loss(**{**fine, **bad})
    # the logits may want the gradient that the call gives
    leaf = logits.clone().requires_grad_()
    got = sv.policy_loss(leaf, tokens, old, adv)
    leaf.backward(got["grad"])
    assert torch.equal(leaf.grad, got["grad"])
    empty = sv.policy_loss(logits[:0], tokens[:0], old[:0], adv[:0])
    assert empty["loss"].shape == (0,) and empty["grad"].shape == (0, 100)

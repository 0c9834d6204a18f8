"""policy_loss where log p in one fp32 number would not do: tokens of very small probability (needs a GB300).

For |log p| of 64 to 128 half a unit of the last place is 3.8e-6, and log2(e) / tau in fp32 loses up to 2^-25 of 90 to 180 units of base 2,
3.7e-6; the ratio, kl and the gradient are functions of small differences of such numbers.  Tolerance of the difference, before any run: a term
2^d of S is off by 2^-22 (the unit) and by 2^-24 |d| ln 2 (its exponent), on average over p; at most 26 additions
(32 elements a thread in two lanes, 16 in a chain, and the joins) by 2^-24 each; log2 of S's fraction and the sums of the two parts by
2^-22 together:  L = 2^-22 + 2^-24 ln 2 E|d| + 26 2^-24 + 2^-22, about 2.2e-6.
kl: |e^u - 1| (L + 2^-23 |u|) + 2^-21 (kl + |u (e^u - 1)|); ratio: ratio (L + 2^-23 |log p - old| + 2^-22); log p itself: L and its own rounding.
"""
import math

import pytest

from test_gpu_policy_loss import exact, sv  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("tau", [0.7, 1.0, 1.3])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("R", [64, 1000])      # CTAs of 512 threads, and of 64
def test_unlikely_tokens(sv, dtype, tau, R):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(R)
    V = 2048
    logits = 3 * tau * torch.randn(R, V, generator=g, device="cuda")
    tokens = torch.randint(0, V, (R,), generator=g, device="cuda")
    at = tokens[:, None]
    logits = logits.scatter(1, at, -tau * (60 + 35 * torch.rand(R, 1, generator=g, device="cuda"))).to(dtype)
    x = logits.double() / tau
    lp = torch.log_softmax(x, 1)
    own = lp.gather(1, at)[:, 0]
    assert ((own.abs() > 64) & (own.abs() < 128)).all()
    old, ref = (own + 0.2 * torch.randn(R, generator=g, device="cuda")).float(), (own + 0.2 * torch.randn(R, generator=g, device="cuda")).float()
    adv = torch.randn(R, generator=g, device="cuda")
    f = exact(logits, tokens, old, adv, ref, None, (0.9, 9.0), 0.1, 0.0, tau)
    got = sv.policy_loss(logits, tokens, old, adv, ref_logp=ref, clip=(0.9, 9.0), kl_weight=0.1, tau=tau)
    sv.status()
    # |d|: the distance to the reference, which is the largest of the threads' first 16 (fp32) or 32 elements, the row's first half or more
    top = x.amax(1, keepdim=True)
    far = ((f["p"] * (top - x)).sum(1) + (top - x[:, : V // 2].amax(1, keepdim=True))[:, 0]) / math.log(2)
    L = 2.0 ** -21 + 2.0 ** -24 * math.log(2) * far + 26 * 2.0 ** -24
    u, e1 = f["u"], torch.expm1(f["u"]).abs()
    bounds = {"logp": L + 2.0 ** -24 * own.abs(), "ratio": f["ratio"] * (L + 2.0 ** -23 * (own - old.double()).abs() + 2.0 ** -22),
              "kl": e1 * (L + 2.0 ** -23 * u.abs()) + 2.0 ** -21 * (f["kl"] + (u * e1).abs())}
    for k, bound in bounds.items():
        worst = ((got[k].double() - f[k]).abs() / bound).max().item()
        assert worst <= 1, (k, worst)
    gl = (-0.1 * torch.expm1(u) - f["ratio"] * f["A"])
    dgl = 0.1 * (e1 + 1) * L + f["ratio"] * f["A"].abs() * (L + 2.0 ** -22) + 2.0 ** -21 * gl.abs() + 2.0 ** -22 * f["ratio"] * f["A"].abs()
    mine = got["grad"].gather(1, at)[:, 0].double()
    want = f["grad"].gather(1, at)[:, 0]
    assert ((mine - want).abs() <= dgl / tau + torch.finfo(dtype).eps / 2 * want.abs() + 2.0 ** -22 * gl.abs() / tau).all()

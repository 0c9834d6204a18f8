"""token_scores and token_scores_grad where x = logits / tau is large: rows closed with a finite
mask, small tau, references on both sides of where their rounding would count (needs a GB300).

The scores depend on the differences to the largest logit, which are exact or within 2^-24 of themselves whatever
the logits' size, so the tolerances of test_gpu_token_scores.py hold here too; the 64-bit formulas take
x = logits * (1 / tau) with 1 / tau in fp32 and the product unrounded; where it leaves fp32's range the
token is closed, and a probability below fp32's least normal number is 0.  (The order of the
alternatives goes by x in fp32.)
"""
import math

import pytest

from test_gpu_token_scores import check_top, grad_near, near, rows, sv  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def formulas(logits, tokens, tau, gl, gh):
    inv = 1.0 / torch.tensor(tau, dtype=torch.float32, device=logits.device)
    x32 = logits.float() * inv
    x = torch.where(torch.isneginf(x32), -math.inf, logits.double() * inv.double())
    none = torch.isneginf(x).all(1)
    m = torch.where(none, 0.0, x.amax(1))
    d = x - m[:, None]
    logs = torch.log(d.exp().sum(1))
    lp = d - torch.where(none, 0.0, logs)[:, None]
    p = torch.where(lp.exp() < 2.0 ** -126, 0.0, lp.exp())
    plp = torch.where(p > 0, p * torch.where(p > 0, lp, 0.0), 0.0)
    H = -plp.sum(1)
    has = tokens >= 0
    at = tokens.clamp(min=0)[:, None]
    a = torch.where(has & ~none, gl.double(), 0.0)[:, None]
    g = -a * p - gh.double()[:, None] * (plp + p * H[:, None])
    g.scatter_add_(1, at, a)
    return {"logp": torch.where(has, lp.gather(1, at)[:, 0], 0.0), "entropy": H, "lse": m + logs, "lp": lp, "p": p,
            "grad": g * inv.double(), "x": x32.double()}


def check(sv, x, tok, gl, gh, tau, top=5):  # noqa: F811
    ref = formulas(x, tok, tau, gl, gh)
    got = sv.token_scores(x, tok, top=top, tau=tau)
    for k in ("logp", "entropy", "lse"):
        near(got[k], ref[k])
    check_top(got, ref, top)
    got = sv.token_scores_grad(x, tok, gl, gh, tau=tau)
    for k in ("logp", "entropy", "lse"):
        near(got[k], ref[k])
    grad_near(got["grad"], ref, torch.where(tok >= 0, gl, 0.0), gh, tau, x.dtype)
    sv.status()


@pytest.mark.parametrize("R,V", [(28, 1000), (28, 50257), (700, 1000), (640, 18003)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tau", [1.0, 1.3, 0.7])
def test_finite_masks(sv, R, V, dtype, tau):  # noqa: F811
    """Rows closed as a whole, rows with a few open tokens, and masks beside large open ones."""
    x, tok, gl, gh = rows(R, V, dtype, V + R)
    masks = [-1e4, -1e7, -3e7, -1e8, -1e9, -1e10, -1e20, -1e30, torch.finfo(dtype).min]
    for i, m in enumerate(masks):
        x[i] = m
        x[9 + i, 7:] = m
    x[18] = 1e10
    x[19, 5:] = -1e10
    x[19, :5] = 1e9
    x[20] = torch.linspace(-1e9, 1e9, V, device="cuda").to(dtype)
    x[21] = -x[20]
    x[22] = 2.0 ** 24 + torch.arange(V, device="cuda").to(dtype) % 13
    x[23] = -(2.0 ** 27) - 16 * (torch.arange(V, device="cuda") % 5).to(dtype)
    # references on both sides of 2^24 and 2^27, of either sign
    step = (torch.arange(V, device="cuda") % 41 - 20).float()
    for i, at in enumerate((2.0 ** 24, -(2.0 ** 24), 2.0 ** 27, -(2.0 ** 27))):
        x[24 + i] = (round(at * tau) + step * (1 if abs(at) < 2e7 else 8)).to(dtype)
    tok[3] = -1
    check(sv, x, tok, gl, gh, tau)


@pytest.mark.parametrize("R,V", [(40, 1000), (700, 5003), (3, 50257)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tau", [1e-6, 1e-8, 1e-9, 1e-12, 1e-30])
def test_small_tau(sv, R, V, dtype, tau):  # noqa: F811
    x, tok, gl, gh = rows(R, V, dtype, V)
    x += 5
    x[1] = 0
    check(sv, x, tok, gl * 1e-6, gh * 1e-6, tau)


@pytest.mark.parametrize("R", [4, 700])
def test_half_precision(sv, R):  # noqa: F811
    """fp16's lowest value at a small tau."""
    x, tok, gl, gh = rows(R, 6000, torch.float16, 3)
    x[0] = -65504
    x[1, 9:] = -65504
    x[2] = 60000 + 32 * (torch.arange(6000, device="cuda") % 3)
    check(sv, x, tok, gl * 1e-3, gh * 1e-3, 1e-3)


def test_padding_closed_with_a_finite_mask_has_no_gradient(sv):  # noqa: F811
    x, tok, gl, gh = rows(6, 30522, torch.bfloat16, 4)
    x[2:] = -1e10
    tok[2:] = -1
    grad = sv.token_scores_grad(x, tok, gl)["grad"]
    assert torch.isfinite(grad).all() and (grad[2:] == 0).all()
    assert math.isfinite((grad.T.float() @ torch.ones(6, 8, device="cuda")).sum().item())

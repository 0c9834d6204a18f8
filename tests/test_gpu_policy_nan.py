"""policy_loss of rows that hold NaN or infinities, in its default form: what is not a number stays none (needs a GB300)."""
import math

import pytest

from test_gpu_policy_loss import ROWS, make, sv  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
SIZES = [(12, 3000), (700, 257), (5, 50257)]      # whole CTAs a row, CTAs of two warps, a cluster a row


def both_signs(adv):
    return torch.where(torch.arange(len(adv), device="cuda") % 2 == 0, adv.abs() + 0.1, -adv.abs() - 0.1)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("R,V", SIZES)
@pytest.mark.parametrize("clip", [0.2, (0.2, math.inf), (1.0, 0.0)])
def test_logits(sv, dtype, R, V, clip):  # noqa: F811
    """Rows 0 to 3: a NaN or +inf under either sign of the advantage; the others are as they were."""
    logits, tokens, old, adv, _, _ = make(R, V, dtype, seed=R)
    logits, adv = logits.contiguous(), both_signs(adv)
    want = sv.policy_loss(logits, tokens, old, adv, clip=clip)
    logits[0, 9], logits[1, V - 1], logits[2, 0], logits[3, 7] = math.nan, math.nan, math.inf, math.inf
    got = sv.policy_loss(logits, tokens, old, adv, clip=clip)
    sv.status()
    for k in ROWS:
        if k in got:
            assert torch.isnan(got[k][:4]).all() and torch.equal(got[k][4:], want[k][4:]), k
    assert torch.isnan(got["grad"][:4]).all() and torch.equal(got["grad"][4:], want["grad"][4:])


@pytest.mark.parametrize("how", [{}, {"kl_weight": 0.1}, {"kl_weight": 0.1, "entropy_weight": 0.1}])
@pytest.mark.parametrize("R,V", SIZES)
def test_rows_own_numbers(sv, R, V, how):  # noqa: F811
    """A NaN in old_logp (under either sign), in the advantage (on either side of the clip) or in the weight: a NaN loss and
    gradient, also where the other side of the clip would have had none."""
    logits, tokens, old, adv, ref, weight = make(R, V, seed=R, far=0.0)
    adv, weight = both_signs(adv), weight + 0.1
    lp = old.clone()
    want = sv.policy_loss(logits, tokens, old, adv, ref_logp=ref, weight=weight, **how)
    old[:2] = math.nan
    old[2], old[3] = lp[2] - 2.0, lp[3] + 2.0      # ratios far above and below the clip
    adv[2:4] = math.nan
    weight[4] = math.nan
    got = sv.policy_loss(logits, tokens, old, adv, ref_logp=ref, weight=weight, **how)
    sv.status()
    assert torch.isnan(got["loss"][:5]).all() and torch.isnan(got["grad"][:5]).all()
    assert torch.isnan(got["ratio"][:2]).all() and torch.isfinite(got["ratio"][2:]).all()
    assert torch.isfinite(got["logp"]).all() and torch.isfinite(got["kl"]).all()
    assert all(torch.equal(got[k][5:], want[k][5:]) for k in want)
    # and rows that the loss leaves out have none of it
    weight[:5] = 0
    got = sv.policy_loss(logits, tokens, old, adv, ref_logp=ref, weight=weight, **how)
    assert (got["loss"][:5] == 0).all() and (got["grad"][:5] == 0).all()


def test_the_clips_ends_and_no_advantage(sv):  # noqa: F811
    """What the selects of the clip give to numbers: the values of minimum and clamp."""
    logits = torch.randn(12, 500, device="cuda")
    tokens = torch.arange(12, device="cuda")
    lp = torch.log_softmax(logits.double(), 1).gather(1, tokens[:, None])[:, 0]
    ratio = torch.tensor([0.0, 0.5, 1.0, 2.0] * 3, device="cuda", dtype=torch.float64)
    adv = torch.tensor([1.5] * 4 + [-1.5] * 4 + [0.0] * 4, device="cuda")
    old = torch.where(ratio == 0, 200.0, lp - ratio.clamp(min=0.1).log()).float()
    got = sv.policy_loss(logits, tokens, old, adv)
    want = -torch.minimum(ratio * adv.double(), ratio.clamp(0.8, 1.2) * adv.double())
    # (lp within 1e-5, old within 2^-24 of its size of at most 20, the rest a few roundings: below 2e-5 of ratio A, which is at most 3)
    assert (got["loss"].double() - want).abs().max() <= 6e-5
    closed = (got["grad"] == 0).all(1)
    assert closed.tolist() == [True, False, False, True] + [True, True, False, False] + [True] * 4

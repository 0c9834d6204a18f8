"""How near policy_loss' log p (seen through kl) is over a batch of wide rows (needs a GB300).

A row's log p is off by what S loses.  Deviations of roundings that are even over their intervals (bound / sqrt 3), q = sum p^2:
each term p of S by 2^-22 (the unit), and by half a unit of the last place of its exponent d, which is taken against its thread's reference,
the largest of some first elements, 16 at least (times ln 2); a lane's sum that holds the term by 2^-24 of it an addition, of which on average 12 follow (half of a batch
of 16, and at most 4 batches); the joins of 512 sums to one, ten levels of W = 512 .. 1 sums, each by 2^-24 of a sum, whose squares are q + (1 - q) / W of
S's where the terms are spread over them at random; log2 of S's fraction by 2^-24 ln 2:
  var = [sum p^2 (2^-44 + (ln 2 ulp(d) / 2)^2) + 12 q 2^-48 + (10 q + 2 (1 - q)) 2^-48 + (2^-24 ln 2)^2] / 3,
about (1e-7)^2 for logits that deviate by four.  Over 600 and 2,400 rows the root of the mean is held within 1.1 of that (one chain of fifty additions and
references that round, bf16: 1.2 of it).
"""
import math

import pytest

from test_gpu_policy_loss import sv  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def var_of(x):
    """From rows of logits / tau."""
    y = x / math.log(2)
    p = torch.softmax(x, 1)
    q = p.square().sum(1)
    ref = y[:, : y.shape[1] // 32 * 32].unflatten(1, (-1, 32)).amax(2).mean(1, keepdim=True)
    half = torch.exp2(torch.floor(torch.log2((y - ref).abs().clamp(min=1e-3)))) * 2.0 ** -24 * math.log(2)
    return ((p.square() * (2.0 ** -44 + half.square())).sum(1) + (12 * q + 10 * q + 2 * (1 - q)) * 2.0 ** -48 + (2.0 ** -24 * math.log(2)) ** 2) / 3


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("R,V", [(600, 50257), (600, 16000), (2400, 50257)])
def test_rows_of_a_batch(sv, dtype, R, V):  # noqa: F811
    g, tau = torch.Generator(device="cuda").manual_seed(V), 0.8
    logits = (3 * torch.randn(R, V, generator=g, device="cuda")).to(dtype)
    parts = []
    for x in logits.split(300):
        x = x.double() / tau
        lp = torch.log_softmax(x, 1)
        tokens = torch.multinomial(lp.exp(), 1, generator=g)
        parts.append((tokens[:, 0], lp.gather(1, tokens)[:, 0], var_of(x)))
    tokens, own, var = (torch.cat(z) for z in zip(*parts))
    ref = (own + torch.where(torch.rand(R, generator=g, device="cuda") < 0.5, 0.2, -0.2)).float()
    got = sv.policy_loss(logits, tokens, own.float(), torch.ones(R, device="cuda"), ref_logp=ref, kl_weight=0.1, tau=tau)
    sv.status()
    u = ref.double() - own
    off = (got["kl"].double() - (torch.expm1(u) - u)) / torch.expm1(u)
    rms, bound = off.square().mean().sqrt().item(), var.mean().sqrt().item()
    assert rms <= 1.1 * bound, (rms, bound)

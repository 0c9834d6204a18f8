"""best_of_n.py with one answer a prompt: a policy step on it has a loss and a gradient (needs a GB300)."""
import pytest

from test_gpu_best_of_n import bn  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("shared", [False, True])
def test_policy_step_of_one_answer(bn, shared):  # noqa: F811
    """An answer without others has no advantage: without a KL term nothing moves, with one the loss is the term."""
    cfg = bn.Config(layers=1, d=256, heads=4, kv_heads=2, hd=64, ff=512, vocab=1000)
    model = bn.Model(cfg, seed=2)
    noise = torch.rand(5, 2, generator=torch.Generator().manual_seed(1)).cuda()
    out = bn.best_of_n(model, [[1, 2, 3], [4] * 20], 1, 5, noise, shared=shared)
    reward = torch.tensor([[0.3], [-2.0]], device="cuda")
    loss, grad = bn.policy_step(model, out, reward, kl_weight=0.0)
    assert loss == 0 and (grad == 0).all()
    loss, grad = bn.policy_step(model, out, reward, kl_weight=0.1, ref_logp=out["logp"] + 0.5)
    # every token's e^u - 1 - u at u = 0.5.  The logits are the drawn ones again by another product, rounded to bf16: a step of 2^-7 at most for
    # sizes below 2 (their deviation is 0.3), which moves u, and the term by 0.65 of that: 0.1 0.65 2^-7 = 5.1e-4
    assert abs(loss.item() - 0.1 * 0.14872127) <= 6e-4
    assert torch.isfinite(grad).all() and (grad != 0).any()


def test_command(bn, capsys, monkeypatch):  # noqa: F811
    monkeypatch.setattr("sys.argv", ["best_of_n", "--prompts", "2", "--n", "1", "--tokens", "4", "--policy"])
    bn.main()
    text = capsys.readouterr().out
    assert "policy loss" in text and "nan" not in text.lower()

"""Rotated heads, attention over shared prefixes and the policy loss as best_of_n.py runs them together (needs a GB300).

Tolerances, before any run, as in test_gpu_best_of_n.py: bf16 activations rounded at different points on the two sides, hidden rows
and logits within 3e-2 of their range; the head's gradient within 2e-2 of its norm.
"""
import math

import pytest

from test_gpu_best_of_n import bn, dense  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def run(bn, qk_norm, heads, kv_heads, hd):  # noqa: F811
    cfg = bn.Config(layers=2, d=256, heads=heads, kv_heads=kv_heads, hd=hd, ff=512, vocab=1000, qk_norm=qk_norm)
    model = bn.Model(cfg, seed=2)
    g = torch.Generator().manual_seed(4)
    lens, n, steps = [1, 33, 300, 48], 6, 19
    prompts = [torch.randint(0, cfg.vocab, (x,), generator=g).tolist() for x in lens]
    noise = torch.rand(steps, len(lens) * n, generator=g).cuda()
    return model, prompts, n, steps, bn.best_of_n(model, prompts, n, steps, noise, shared=True)


@pytest.mark.parametrize("qk_norm", [False, True])
@pytest.mark.parametrize("heads,kv_heads,hd", [(12, 4, 64), (4, 2, 128)])
def test_scores_and_cache(bn, qk_norm, heads, kv_heads, hd):  # noqa: F811
    model, prompts, n, steps, out = run(bn, qk_norm, heads, kv_heads, hd)
    assert len({tuple(t) for t in out["tokens"].view(-1, steps).tolist()}) == len(prompts) * n
    for p, prompt in enumerate(prompts):
        for c in range(n):
            ids = torch.tensor(prompt + out["tokens"][p, c].tolist(), device="cuda")
            keep = []

            def attend(layer, q, k, v):
                keep.append((k, v))
                return dense(q, k, v)

            rows = model.run(ids, torch.arange(len(ids), device="cuda"), attend)
            logits = rows[len(prompt) - 1: -1].float() @ model.head.float().T
            want = torch.log_softmax(logits, -1).gather(1, out["tokens"][p, c][:, None])[:, 0]
            assert ((out["logp"][p, c] - want).abs() <= 3e-2 * (logits.amax(1) - logits.amin(1))).all(), (p, c)
            if c != int(out["best"][p]):
                continue
            slot, length = out["kept"].tolist()[p], len(prompt) + steps
            pages = out["cache"].table[slot][: -(-length // bn.PAGE)].long()
            for layer, (k, v) in enumerate(keep):
                got = out["cache"].pool[layer][pages].permute(1, 0, 3, 2, 4).flatten(1, 2)[:, :length]
                for x, y in ((got[0], k), (got[1], v)):
                    assert (x.float() - y.float()).abs().max() <= 3e-2 * (y.amax() - y.amin()).float()


@pytest.mark.parametrize("kl_weight,entropy_weight", [(0.0, 0.0), (0.1, 0.01)])
def test_policy_step(bn, kl_weight, entropy_weight):  # noqa: F811
    """The loss and the head's gradient against autograd's of the written formula on the same rows."""
    model, _, n, steps, out = run(bn, True, 4, 2, 64)
    g = torch.Generator(device="cuda").manual_seed(3)
    reward = torch.rand(4, n, generator=g, device="cuda")
    ref = out["logp"] + 0.1 * torch.randn(out["logp"].shape, generator=g, device="cuda")
    model.head += (0.01 * torch.randn(model.head.shape, generator=g, device="cuda")).bfloat16()       # the policy has moved since
    loss, grad = bn.policy_step(model, out, reward, kl_weight=kl_weight, entropy_weight=entropy_weight, ref_logp=ref)
    head = model.head.float().requires_grad_()
    logits = out["rows"].flatten(0, 1).float() @ head.T
    # (the step's logits are rounded to bf16: so are these, with the gradient passed through)
    logits = logits + (logits.bfloat16().float() - logits).detach()
    lp_all = torch.log_softmax(logits, -1)
    lp = lp_all.gather(1, out["tokens"].flatten()[:, None])[:, 0]
    A = ((reward - reward.mean(1, keepdim=True)) / (reward.std(1, keepdim=True) + 1e-6)).repeat_interleave(steps)
    ratio, u = (lp - out["logp"].flatten()).exp(), ref.flatten() - lp
    entropy = -(lp_all.exp() * lp_all).sum(1)
    want = (kl_weight * (u.exp() - 1 - u) - torch.minimum(ratio * A, ratio.clamp(0.8, 1.28) * A) - entropy_weight * entropy).mean()
    want.backward()
    assert abs(loss.item() - want.item()) <= 1e-4
    assert (grad.float() - head.grad).norm() <= 2e-2 * head.grad.norm()


def test_an_attention_layer_learns_through_the_rotation(bn):  # noqa: F811
    """rotate_heads and rotate_heads_grad around plain attention, as an autograd function of a user's: gradients of the
    projection and of the norms' weights against autograd's of the formulas in 64 bits (activations are fp16: 2^-11 a rounding, a handful
    of them, 5e-3 of the norms)."""
    from paper_2606_10820_gb300 import serving

    class Rotate(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, pos, freq, wq, wk):
            ctx.save_for_backward(q, k, pos, freq, wq, wk)
            return serving.rotate_heads(q, k, pos, freq, wq, wk, eps=1e-6)

        @staticmethod
        def backward(ctx, dq, dk):
            q, k, pos, freq, wq, wk = ctx.saved_tensors
            g = serving.rotate_heads_grad(dq, dk, q, k, pos, freq, wq, wk, eps=1e-6)
            return g["q"], g["k"], None, None, g["q_weight"].half(), g["k_weight"].half()

    T, d, Hq, Hkv, hd = 70, 96, 4, 2, 64
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(T, d, generator=g, device="cuda").half()
    w = (torch.randn((Hq + 2 * Hkv) * hd, d, generator=g, device="cuda") * 0.1).half().requires_grad_()
    wq, wk = ((1 + 0.2 * torch.randn(hd, generator=g, device="cuda")).half().requires_grad_() for _ in range(2))
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    freq = 1e4 ** (-2.0 * torch.arange(hd // 2, dtype=torch.float64, device="cuda") / hd)
    dout = torch.randn(T, Hq, hd, generator=g, device="cuda")

    def attention(q, k, v):
        k, v = (y.repeat_interleave(Hq // Hkv, 1) for y in (k, v))
        s = torch.einsum("qhd,khd->hqk", q, k) / math.sqrt(hd)
        s = s.masked_fill(torch.ones(T, T, dtype=torch.bool, device="cuda").triu(1), -math.inf)
        return torch.einsum("hqk,khd->qhd", torch.softmax(s, -1), v)

    q, k, v = (x @ w.T).view(T, -1, hd).split([Hq, Hkv, Hkv], 1)
    q, k = Rotate.apply(q, k, pos, freq, wq, wk)
    (attention(q.float(), k.float(), v.float()) * dout).sum().backward()

    w64, wq64, wk64 = (y.detach().double().requires_grad_() for y in (w, wq, wk))
    q, k, v = (x.double() @ w64.T).view(T, -1, hd).split([Hq, Hkv, Hkv], 1)

    def rotate(y, weight):
        y = y / (y.square().mean(-1, keepdim=True) + 1e-6).sqrt() * weight
        angle = pos.double()[:, None, None] * freq
        a, b = y.split(hd // 2, -1)
        return torch.cat([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], -1)

    (attention(rotate(q, wq64), rotate(k, wk64), v) * dout).sum().backward()
    for got, want in ((w.grad, w64.grad), (wq.grad, wq64.grad), (wk.grad, wk64.grad)):
        assert (got.double() - want).norm() <= 5e-3 * want.norm()


def test_command_with_everything(bn, capsys, monkeypatch):  # noqa: F811
    monkeypatch.setattr("sys.argv", ["best_of_n", "--prompts", "2", "--n", "3", "--tokens", "5", "--shared", "--policy", "--qk-norm"])
    bn.main()
    text = capsys.readouterr().out
    assert "best of 3" in text and "policy loss" in text

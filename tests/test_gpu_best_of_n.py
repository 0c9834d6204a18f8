"""The serving operators together (best_of_n.py) against the same model recomputed from its
tokens without a cache, in fp32 attention and products on the bf16 weights (needs a GB300).

Tolerance, before any run: activations and K, V are rounded to bf16 at different points on
the two sides (2^-9 relative each, a handful of roundings a layer, four layers): hidden rows
within 3e-2 of their range, and a token's log probability within 3e-2 of its row's logit range
(the bound that the decode step's logits have).
"""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def bn():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__ as g
    g.build()
    from paper_2606_10820_gb300 import best_of_n
    return best_of_n


def dense(q, k, v):
    G = q.shape[1] // k.shape[1]
    k, v = (x.float().repeat_interleave(G, 1) for x in (k, v))
    w = torch.einsum("qhd,khd->hqk", q.float(), k) / math.sqrt(q.shape[2])
    w.masked_fill_(torch.ones(len(q), len(q), dtype=torch.bool, device=q.device).triu(1), -math.inf)
    return torch.einsum("hqk,khd->qhd", torch.softmax(w, -1), v).bfloat16()


@pytest.mark.parametrize("heads,kv_heads,hd", [(12, 4, 64), (4, 2, 128)])
def test_scores_cache_and_gradient(bn, heads, kv_heads, hd):
    cfg = bn.Config(layers=2, d=256, heads=heads, kv_heads=kv_heads, hd=hd, ff=512, vocab=1000)
    model = bn.Model(cfg, seed=2)
    g = torch.Generator().manual_seed(4)
    lens, n, steps = [1, 33, 130, 48], 5, 19
    prompts = [torch.randint(0, cfg.vocab, (x,), generator=g).tolist() for x in lens]
    noise = torch.rand(steps, len(lens) * n, generator=g).cuda()
    out = bn.best_of_n(model, prompts, n, steps, noise)
    assert out["tokens"].shape == (4, n, steps) and (out["tokens"] >= 0).all() and (out["tokens"] < cfg.vocab).all()
    assert len({tuple(t) for t in out["tokens"].view(-1, steps).tolist()}) == 4 * n      # the candidates differ

    kv = {}
    for p, prompt in enumerate(prompts):
        for c in range(n):
            ids = torch.tensor(prompt + out["tokens"][p, c].tolist(), device="cuda")
            keep = []

            def attend(layer, q, k, v):
                keep.append((k, v))
                return dense(q, k, v)

            rows = model.run(ids, torch.arange(len(ids), device="cuda"), attend)
            kv[p, c] = keep
            logits = rows[len(prompt) - 1: -1].float() @ model.head.float().T
            want = torch.log_softmax(logits, -1).gather(1, out["tokens"][p, c][:, None])[:, 0]
            bound = 3e-2 * (logits.amax(1) - logits.amin(1))
            assert ((out["logp"][p, c] - want).abs() <= bound).all(), (p, c)

    # the kept answers' K and V are where the compacted table says, page by page
    cache = out["cache"]
    for p, slot in enumerate(out["kept"].tolist()):
        length = lens[p] + steps
        assert cache.lens[slot].item() == length
        pages = cache.table[slot][: -(-length // bn.PAGE)].long()
        for layer, (k, v) in enumerate(kv[p, int(out["best"][p])]):
            got = cache.pool[layer][pages].permute(1, 0, 3, 2, 4).flatten(1, 2)[:, :length]
            for x, y in ((got[0], k), (got[1], v)):
                assert (x.float() - y.float()).abs().max() <= 3e-2 * (y.amax() - y.amin()).float()
    used = sum(-(-(x + steps) // bn.PAGE) for x in lens)
    assert out["live"] == used and int((cache.ref > 0).sum()) == used and int(cache.table.max()) < used
    assert (cache.ref[:used] == 1).all() and (cache.ref[used:] == 0).all()

    # the head's gradient against autograd's on the same rows
    loss, grad = bn.head_step(model, out)
    at = torch.arange(4, device="cuda") * n + out["best"]
    x = out["rows"][at].flatten(0, 1).float()
    tok = out["tokens"].view(-1, steps)[at].flatten()
    head = model.head.float().requires_grad_()
    ref = torch.nn.functional.cross_entropy(x @ head.T, tok)
    ref.backward()
    assert abs(loss.item() - ref.item()) <= 3e-2
    assert (grad.float() - head.grad).norm() <= 2e-2 * head.grad.norm()


def test_command(bn, capsys, monkeypatch):
    monkeypatch.setattr("sys.argv", ["best_of_n", "--prompts", "2", "--n", "3", "--tokens", "5"])
    bn.main()
    text = capsys.readouterr().out
    assert "best of 3" in text and "pages live" in text

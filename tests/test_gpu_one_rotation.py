"""best_of_n.py with shared prefixes: all keys of a cache are rotated alike, with and without norms of the heads (needs a GB300)."""
import pytest

from test_gpu_best_of_n import bn  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("qk_norm", [False, True])
def test_a_prompts_keys_are_rotate_heads(bn, qk_norm):  # noqa: F811
    """The first layer's keys of each kept answer, prompt and drawn tokens, to the bit: rotate_heads of the same projections."""
    from paper_2606_10820_gb300 import serving
    cfg = bn.Config(layers=1, d=256, heads=4, kv_heads=2, hd=64, ff=512, vocab=1000, qk_norm=qk_norm)
    model, n, steps = bn.Model(cfg, seed=2), 3, 4
    g = torch.Generator().manual_seed(4)
    prompts = [torch.randint(0, cfg.vocab, (x,), generator=g).tolist() for x in (900, 1700)]
    noise = torch.rand(steps, 2 * n, generator=g).cuda()
    calls, run = [], model.run

    def spy(tokens, pos, attend, **how):
        def keep(layer, q, k, v):
            calls.append((pos, q.clone(), k.clone()))
            return torch.zeros_like(q)
        run(tokens, pos, keep, raw=True)
        return run(tokens, pos, attend, **how)

    model.run = spy
    out = bn.best_of_n(model, prompts, n, steps, noise, shared=True)
    keys = [serving.rotate_heads(q, k, pos.int(), model.freq, **model.turn[0])[1] for pos, q, k in calls]
    pool, table = out["cache"].pool[0], out["cache"].table
    for p, x in enumerate(len(t) for t in prompts):
        held = pool[table[out["kept"].tolist()[p]][: -(-(x + steps) // bn.PAGE)].long(), 0].permute(0, 2, 1, 3).flatten(0, 1)
        at = sum(len(t) for t in prompts[:p])
        assert torch.equal(held[:x], keys[0][at: at + x])
        row = p * n + int(out["best"][p])
        for i in range(steps):
            assert torch.equal(held[x + i], keys[1 + i][row])

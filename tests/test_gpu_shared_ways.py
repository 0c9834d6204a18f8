"""shared_attention in each of its three ways at sizes that choose that way, the largest ones among them; and best_of_n.py at sizes
that reach the two that read a prefix once (needs a GB300).  Tolerances as in test_gpu_shared_attention.py and test_gpu_best_of_n.py."""
import pytest

import shared_ways
from test_gpu_best_of_n import bn, dense  # noqa: F401
from test_gpu_shared_attention import check, make, sv  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def way(q, pool, table, n):
    B, rows, Hq, hd = q.shape
    return shared_ways.way_of(B, rows, Hq, pool.shape[2], hd, len(pool), pool.shape[3], table.shape[1], n)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("name,at", [(w, i) for w in shared_ways.CASES for i in range(len(shared_ways.CASES[w]))])
def test_each_way_matches_plain(sv, dtype, name, at):  # noqa: F811
    groups, rows, Hq, Hkv, hd, more = shared_ways.CASES[name][at]
    # (the two ways of a prefix read once take it from the first sequence's row alone: hidden from the others' every other time)
    args = make(groups, rows, Hq, Hkv, hd, dtype, seed=at, extra_width=2 + more, spare=3 + more, hide=name != "paged" and at % 2 == 1)
    assert way(args[0], args[1], args[2], len(groups)) == name
    got = check(sv, *args)
    assert torch.equal(sv.shared_attention(*args), got)


@pytest.mark.parametrize("name,lens,n,qk_norm", [("rows", [500, 333], 64, False), ("rows", [700, 81, 16], 40, True), ("tiles", [1490, 700], 256, True)])
def test_many_candidates(bn, name, lens, n, qk_norm):  # noqa: F811
    """The scores of some candidates against the whole model's on their tokens."""
    cfg = bn.Config(layers=2, d=256, heads=12, kv_heads=4, hd=64, ff=512, vocab=1000, qk_norm=qk_norm)
    model, steps = bn.Model(cfg, seed=2), 5
    g = torch.Generator().manual_seed(4)
    prompts = [torch.randint(0, cfg.vocab, (x,), generator=g).tolist() for x in lens]
    noise = torch.rand(steps, len(lens) * n, generator=g).cuda()
    out = bn.best_of_n(model, prompts, n, steps, noise, shared=True)
    pool, table = out["cache"].pool[0], out["cache"].table
    assert way(torch.empty(len(lens) * n, 1, 12, 64), pool, table, len(lens)) == name
    for p, prompt in enumerate(prompts):
        for c in (0, 1, n // 2, n - 1):
            ids = torch.tensor(prompt + out["tokens"][p, c].tolist(), device="cuda")
            rows = model.run(ids, torch.arange(len(ids), device="cuda"), lambda layer, q, k, v: dense(q, k, v))
            logits = rows[len(prompt) - 1: -1].float() @ model.head.float().T
            want = torch.log_softmax(logits, -1).gather(1, out["tokens"][p, c][:, None])[:, 0]
            assert ((out["logp"][p, c] - want).abs() <= 3e-2 * (logits.amax(1) - logits.amin(1))).all(), (p, c)

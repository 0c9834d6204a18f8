"""Best of n over a paged cache: the serving operators together, as a server would use them.

A small causal Transformer with grouped heads (random weights; projections are
library products) answers each prompt n times.  The prompts run once: their attention and their
K and V rows into pages.  Then each prompt's sequence is forked n times (full pages
shared, the last one copied), and every candidate draws its own tokens, one noise value a
token, by the noise -> token map of the LM head (kf_op_head_tokens).  Each
token is scored under the model; the best candidate of each prompt stays, the others' pages
go back, and what is left of the cache is moved together.  ``head_step`` gives the
loss of the kept tokens and the LM head's gradient, the step that would train on them.

    python -m paper_2606_10820_gb300.best_of_n --prompts 4 --n 8 --tokens 32
"""
from __future__ import annotations

import argparse
import ctypes
import math
from dataclasses import dataclass

import torch

from . import kforcing as kf
from . import serving

PAGE = 16


@dataclass
class Config:
    layers: int = 4
    d: int = 768
    heads: int = 12
    kv_heads: int = 4
    hd: int = 64
    ff: int = 2048
    vocab: int = 30522


class Model:
    def __init__(self, cfg: Config, seed=0):
        self.cfg = cfg
        g = torch.Generator(device="cuda").manual_seed(seed)

        def w(*shape):
            return (torch.randn(*shape, generator=g, device="cuda") * 0.02).bfloat16()

        c = cfg
        self.emb = w(c.vocab, c.d)
        self.head = w(c.vocab, c.d)
        self.layers = [(w((c.heads + 2 * c.kv_heads) * c.hd, c.d), w(c.d, c.heads * c.hd), w(c.ff, c.d), w(c.d, c.ff))
                       for _ in range(c.layers)]

    @staticmethod
    def norm(h):
        return (h * torch.rsqrt(h.square().mean(-1, keepdim=True) + 1e-6)).bfloat16()

    def rotate(self, x, pos):
        """Rotary positions of x [T, heads, hd] at pos [T] (halves paired)."""
        half = self.cfg.hd // 2
        angle = pos[:, None].float() * torch.exp(-math.log(1e4) / half * torch.arange(half, device=x.device))[None]
        cos, sin = angle.cos()[:, None], angle.sin()[:, None]
        a, b = x[..., :half].float(), x[..., half:].float()
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1).bfloat16()

    def run(self, tokens, pos, attend):
        """The final hidden rows [T, d] bf16 of tokens at pos; attend(layer, q, k, v) -> [T, heads, hd]."""
        c = self.cfg
        h = self.emb[tokens].float()
        for i, (wqkv, wo, up, down) in enumerate(self.layers):
            qkv = (self.norm(h) @ wqkv.T).view(len(h), -1, c.hd)
            q, k, v = qkv.split([c.heads, c.kv_heads, c.kv_heads], 1)
            o = attend(i, self.rotate(q, pos), self.rotate(k, pos), v)
            h = h + (o.reshape(len(h), -1) @ wo.T).float()
            h = h + (torch.nn.functional.gelu(self.norm(h) @ up.T, approximate="tanh") @ down.T).float()
        return self.norm(h)


def draw_tokens(x, head, noise, tau=1.0):
    """One token per row of x [R, d]: the inverse CDF of softmax(x . head^T / tau) at noise [R]."""
    lib = kf.load_library()
    f = lib.kf_op_head_tokens
    f.argtypes = [ctypes.c_int32] * 3 + [ctypes.c_void_p] * 3 + [ctypes.c_float, ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p]
    f.restype = ctypes.c_int
    out = torch.empty(len(x), dtype=torch.int32, device=x.device)
    kf._check(f(len(x), len(head), x.shape[1], x.data_ptr(), head.data_ptr(), noise.data_ptr(), tau, kf.KF_MAP_ICDF, out.data_ptr(),
                torch.cuda.current_stream().cuda_stream))
    return out.long()


class Cache:
    """Pages of every layer and their book."""

    def __init__(self, cfg: Config, slots, longest, n_pages):
        self.pool = torch.zeros(cfg.layers, n_pages, 2, cfg.kv_heads, PAGE, cfg.hd, dtype=torch.bfloat16, device="cuda")
        self.ref, self.table, self.lens = self.book = serving.new_book(n_pages, slots, -(-longest // PAGE))

    def append(self, layer, k, v, starts, slots):
        serving.pages_append(self.pool[layer], k, v, starts, self.table, self.lens, slots)


def _ints(x):
    return torch.as_tensor(x, dtype=torch.int32, device="cuda")


def best_of_n(model: Model, prompts, n, steps, noise, tau=1.0):
    """n answers of `steps` tokens to each prompt (lists of ids), noise [steps, prompts * n] in [0, 1).

    A dict: tokens [prompts, n, steps]; logp [prompts, n, steps], their scores; best [prompts], the
    answer of the highest total; rows, the hidden rows that the tokens were drawn from; cache, with
    the best answers in slots `kept`; live, the pages in use."""
    cfg, P = model.cfg, len(prompts)
    lens = [len(p) for p in prompts]
    longest = max(lens) + steps
    n_pages = sum(-(-x // PAGE) for x in lens) + P * n * (-(-steps // PAGE) + 2)
    cache = Cache(cfg, P * (1 + n), longest, n_pages)
    starts = _ints([sum(lens[:i]) for i in range(P + 1)])
    owners = _ints(range(P))
    ids = torch.tensor([t for p in prompts for t in p], device="cuda")
    pos = torch.cat([torch.arange(x, device="cuda") for x in lens])

    serving.pages_grow(*cache.book, owners, _ints(lens))

    def whole(layer, q, k, v):
        cache.append(layer, k, v, starts, owners)
        return serving.prompt_attention(q, k, v, starts, max(lens))

    rows = model.run(ids, pos, whole)[(starts[1:] - 1).long()]

    # candidate i of prompt p in slot P + p n + i
    slots = _ints(range(P, P * (1 + n)))
    serving.pages_fork(cache.pool, *cache.book, owners.repeat_interleave(n), slots)
    serving.pages_free(*cache.book, owners)
    rows = rows.repeat_interleave(n, 0).contiguous()
    at = _ints(lens).repeat_interleave(n)
    one_each = _ints(range(P * n + 1))
    tokens, logp, drawn_from = [], [], []

    def newest(layer, q, k, v):
        cache.append(layer, k, v, one_each, slots)
        return serving.paged_attention(q[:, None], cache.pool[layer], table, at + 1)[:, 0]

    for step in range(steps):
        drawn_from.append(rows)
        tokens.append(draw_tokens(rows, model.head, noise[step].contiguous(), tau))
        logp.append(serving.token_scores(rows @ model.head.T, tokens[-1], tau=tau)["logp"])
        serving.pages_grow(*cache.book, slots, at + 1)
        table = cache.table[P:]
        rows = model.run(tokens[-1], at, newest)
        at = at + 1

    logp = torch.stack(logp, 1).view(P, n, steps)
    best = logp.sum(-1).argmax(1)
    keep = torch.zeros(P, n, dtype=torch.bool, device="cuda").scatter_(1, best[:, None], True).flatten()
    serving.pages_free(*cache.book, slots[~keep].contiguous())
    live = _ints([0])
    serving.pages_compact(cache.pool, cache.ref, cache.table, live)
    serving.status()
    return {"tokens": torch.stack(tokens, 1).view(P, n, steps), "logp": logp, "best": best, "rows": torch.stack(drawn_from, 1),
            "cache": cache, "kept": slots[keep], "live": int(live)}


def head_step(model: Model, answer, tau=1.0):
    """The mean negative log probability of the best answers' tokens and the LM head's gradient [V, d]."""
    P, n, steps = answer["tokens"].shape
    at = torch.arange(P, device="cuda") * n + answer["best"]
    rows = answer["rows"][at].flatten(0, 1)
    tok = answer["tokens"].view(P * n, steps)[at].flatten()
    out = serving.token_scores_grad(rows @ model.head.T, tok, torch.full((len(tok),), -1.0 / len(tok), device="cuda"), tau=tau)
    return -out["logp"].mean(), out["grad"].T @ rows


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--prompts", type=int, default=4)
    ap.add_argument("--n", type=int, default=8)
    ap.add_argument("--tokens", type=int, default=32)
    a = ap.parse_args()
    model, g = Model(Config()), torch.Generator().manual_seed(1)
    lens = torch.randint(20, 400, (a.prompts,), generator=g).tolist()
    prompts = [torch.randint(0, model.cfg.vocab, (x,), generator=g).tolist() for x in lens]
    noise = torch.rand(a.tokens, a.prompts * a.n, generator=g).cuda()
    out = best_of_n(model, prompts, a.n, a.tokens, noise)
    loss, grad = head_step(model, out)
    for p in range(a.prompts):
        total = out["logp"][p].sum(-1)
        print(f"prompt of {lens[p]}: best of {a.n} is {int(out['best'][p])}, log p {total.max():.2f} (mean {total.mean():.2f})")
    print(f"{out['live']} pages live; loss of the kept tokens {loss:.4f}, head gradient norm {grad.float().norm():.4f}")


if __name__ == "__main__":
    main()

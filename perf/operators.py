"""Performance cases of the serving operators (include/kforcing_serving.h).

Seven kinds of case, each a plain dict:

  prompt   prompt_attention: causal attention over packed prompts, grouped heads
  decode   paged_attention: the newest rows of each sequence over a paged cache
  append   pages_grow + pages_append: room for new tokens, and their K and V rows
  fork     pages_fork + pages_free: candidates of each prompt, and the losers' end
  compact  pages_compact: the live pages moved below the cache's live count
  score    token_scores: log probabilities, entropy and top alternatives
  grad     token_scores_grad: the scores and the gradient of the logits

Model shapes are those of ``synth.WORKLOADS`` (12 heads of 64, vocabulary
50257, 16-token pages, prompts of 128 to 896 tokens), with grouped heads, and
generic wider ones.  Sequence lengths are spread evenly over [lo, hi] and
shuffled by the seed, so that every seed asks for the same work.
"""
import math

import torch

own = False
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
PAGE = 16


def listed():
    return [
        # a few odd short requests at once (one of a single token): latency
        {"name": "prompt_small", "kind": "prompt", "n": 5, "lo": 1, "hi": 77, "Hq": 7, "Hkv": 1, "hd": 128,
         "dtype": "fp16", "fused": False},
        # a group of new requests of the serving workload, heads in groups of
        # three, q, k and v views of one projection's output
        {"name": "prompt_ragged", "kind": "prompt", "n": 16, "lo": 128, "hi": 896, "Hq": 12, "Hkv": 4, "hd": 64,
         "dtype": "bf16", "fused": True},
        # two long documents
        {"name": "prompt_long", "kind": "prompt", "n": 2, "lo": 7411, "hi": 8192, "Hq": 16, "Hkv": 4, "hd": 128,
         "dtype": "bf16", "fused": True},
        # one user with a long context: the cache's length is all there is to split
        {"name": "decode_one_long", "kind": "decode", "n": 1, "lo": 37013, "hi": 37013, "rows": 1, "Hq": 32, "Hkv": 8,
         "hd": 128, "dtype": "bf16"},
        # the paged serving workload at k = 4: eight rows per sequence
        {"name": "decode_joint", "kind": "decode", "n": 256, "lo": 128, "hi": 1024, "rows": 8, "Hq": 12, "Hkv": 4,
         "hd": 64, "dtype": "fp16"},
        # one new token of each of many ragged sequences: the largest decode call
        {"name": "decode_large", "kind": "decode", "n": 128, "lo": 512, "hi": 8192, "rows": 1, "Hq": 32, "Hkv": 8,
         "hd": 128, "dtype": "bf16"},
        # a prompt group's K and V rows into their pages
        {"name": "append_prompts", "kind": "append", "n": 64, "lo": 128, "hi": 1900, "old": 0, "Hkv": 8, "hd": 128,
         "dtype": "bf16"},
        # eight candidates of each of four prompts, half of them dropped: latency
        {"name": "fork_candidates", "kind": "fork", "n": 4, "each": 8, "lo": 131, "hi": 893, "layers": 12, "Hkv": 12,
         "hd": 64, "n_pages": 1024, "dtype": "bf16"},
        # a cache that long serving has left scattered
        {"name": "compact_cache", "kind": "compact", "slots": 512, "width": 64, "live": 10007, "moves": 4001,
         "n_pages": 16384, "layers": 4, "Hkv": 8, "hd": 64, "dtype": "bf16"},
        # scores of one decode call's tokens of a few sequences: latency
        {"name": "score_small", "kind": "score", "rows": 8, "V": 50257, "top": 5, "tau": 1.0, "dtype": "fp32"},
        # scores of 512 sequences at k = 8
        {"name": "score_large", "kind": "score", "rows": 4096, "V": 50257, "top": 8, "tau": 0.8, "dtype": "bf16"},
        # the loss and its gradient over a training batch's tokens
        {"name": "grad_batch", "kind": "grad", "rows": 2048, "V": 50257, "tau": 1.0, "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    """A whole number from lo to hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["prompt", "prompt", "decode", "decode", "append", "fork", "compact", "score", "score", "grad"])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    hkv, hd = rng.choice([1, 2, 4, 8]), rng.choice([64, 128])
    hq = hkv * rng.choice([1, 2, 3, 4, 8])
    if kind == "prompt":
        hq = min(hq, 16 if hkv < 8 else 8)
        hi = _log(rng, 2, 8000)
        lo = max(1, int(hi * rng.uniform(0.05, 1.0)))
        # at most the listed case's scores, and as many tokens
        n = _log(rng, 1, max(1, min(64, int(2 * 8192 ** 2 * 16 / (hi * hi * hq)), 16384 // hi)))
        return {"kind": "prompt", "n": n, "lo": lo, "hi": hi, "Hq": hq // hkv * hkv, "Hkv": hkv, "hd": hd,
                "dtype": dtype, "fused": rng.random() < 0.5}
    if kind == "decode":
        hi = _log(rng, 1, 40000)
        lo = max(1, int(hi * rng.uniform(0.05, 1.0)))
        n = _log(rng, 1, max(1, min(512, int(2e9 / (hi * hkv * hd * 4)))))
        return {"kind": "decode", "n": n, "lo": lo, "hi": hi, "rows": rng.choice([1, 1, 1, 2, 3, 5, 8]), "Hq": hq,
                "Hkv": hkv, "hd": hd, "dtype": dtype}
    if kind == "append":
        hi = _log(rng, 1, 2000)
        return {"kind": "append", "n": _log(rng, 1, 64), "lo": max(1, int(hi * rng.uniform(0.1, 1.0))), "hi": hi,
                "old": rng.choice([0, 0, 5, 16, rng.randint(1, 700)]), "Hkv": hkv, "hd": hd, "dtype": dtype}
    if kind == "fork":
        layers, hi = rng.randint(1, 12), _log(rng, 3, 900)
        return {"kind": "fork", "n": _log(rng, 1, 6), "each": rng.randint(1, 8), "lo": max(1, int(hi * rng.uniform(0.1, 1.0))),
                "hi": hi, "layers": layers, "Hkv": hkv, "hd": hd, "n_pages": rng.randint(600, 1024), "dtype": dtype}
    if kind == "compact":
        n_pages, width = _log(rng, 300, 16384), rng.randint(20, 64)
        live = int(n_pages * rng.uniform(0.2, 0.6))
        return {"kind": "compact", "slots": max(2, live * 5 // (3 * width) + rng.randint(1, 100)), "width": width, "live": live,
                "moves": int(min(live, n_pages - live) * rng.uniform(0.0, 0.5)), "n_pages": n_pages,
                "layers": rng.randint(1, 4), "Hkv": rng.choice([1, 2, 4, 8]), "hd": 64, "dtype": dtype}
    V = _log(rng, 1000, 130000)
    dtype = rng.choice(["bf16", "fp16", "fp32"])
    if kind == "score":
        rows = _log(rng, 1, max(2, int(4096 * 50257 / (V * (2 if dtype == "fp32" else 1)))))
        return {"kind": "score", "rows": min(rows, 4096), "V": V, "top": rng.choice([0, 1, 5, 8, 20]),
                "tau": rng.choice([1.0, 0.7, 1.3]), "dtype": dtype}
    rows = _log(rng, 1, max(2, int(2048 * 50257 / (V * (2 if dtype == "fp32" else 1)))))
    return {"kind": "grad", "rows": min(rows, 2048), "V": V, "tau": rng.choice([1.0, 0.7, 1.3]), "dtype": dtype}


# ------------------------------------------------------------------ inputs

def _spread(n, lo, hi):
    """n lengths spread evenly over [lo, hi], the ends among them."""
    return [hi] if n == 1 else [lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _shuffled(g, values):
    v = torch.tensor(values, dtype=torch.int32, device=DEV)
    return v[torch.randperm(len(values), generator=g, device=DEV)]


def _starts(lens):
    return torch.cat([torch.zeros(1, dtype=torch.int32, device=DEV), lens.cumsum(0).to(torch.int32)])


def _normal(g, shape, dtype):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32 if dtype == "fp32" else TYPES[dtype])


def _cdiv(a, b):
    return -(-a // b)


class _State:
    pass


def prepare(case, seed):
    s, g = _State(), torch.Generator(device=DEV).manual_seed(seed & 0x7FFFFFFF)
    s.kind = case["kind"]
    if s.kind in ("score", "grad"):
        R, V = case["rows"], case["V"]
        s.logits = (_normal(g, (R, V), case["dtype"]) * 3).to(TYPES[case["dtype"]])
        if case["rows"] > 2:
            # a grammar's mask on one row: most of the vocabulary is closed
            s.logits[1, V // 50:] = -math.inf
        s.tokens = torch.randint(0, V, (R,), generator=g, device=DEV)
        if case["rows"] > 2:
            s.tokens[1] = 3
            s.tokens[2] = -1          # padding: no token
        s.tau, s.top = case["tau"], case.get("top", 0)
        s.g_logp = torch.randn(R, generator=g, device=DEV)
        s.g_entropy = torch.randn(R, generator=g, device=DEV) * 0.1
        return s
    Hkv, hd, dt = case["Hkv"], case["hd"], case["dtype"]
    if s.kind == "prompt":
        Hq, lens = case["Hq"], _spread(case["n"], case["lo"], case["hi"])
        T = sum(lens)
        s.cu, s.longest = _starts(_shuffled(g, lens)), max(lens)
        if case["fused"]:
            s.q, s.k, s.v = _normal(g, (T, Hq + 2 * Hkv, hd), dt).split([Hq, Hkv, Hkv], dim=1)
        else:
            s.q, s.k, s.v = (_normal(g, (T, h, hd), dt) for h in (Hq, Hkv, Hkv))
        return s
    if s.kind == "decode":
        lens, width = _spread(case["n"], case["lo"], case["hi"]), _cdiv(case["hi"], PAGE)
        s.lens = _shuffled(g, lens)
        need = (s.lens + PAGE - 1) // PAGE
        n_pages = sum(_cdiv(x, PAGE) for x in lens)
        s.pool = _normal(g, (n_pages, 2, Hkv, PAGE, hd), dt)
        s.table = _table(g, need, width, torch.randperm(n_pages, generator=g, device=DEV))
        s.q = _normal(g, (case["n"], case["rows"], case["Hq"], hd), dt)
        return s
    if s.kind == "append":
        lens, width = _spread(case["n"], case["lo"], case["hi"]), _cdiv(case["hi"] + case["old"], PAGE)
        n, old = case["n"], case["old"]
        n_pages = n * width + 7
        cnt = _shuffled(g, lens)
        s.cu, s.slots = _starts(cnt), torch.randperm(n, generator=g, device=DEV).to(torch.int32)
        s.new_lens = cnt + old
        s.pool = _normal(g, (1, n_pages, 2, Hkv, PAGE, hd), dt)
        used = torch.full((n,), _cdiv(old, PAGE), dtype=torch.int32, device=DEV)
        _book(s, n, width, n_pages, used, torch.full_like(used, old), torch.randperm(n_pages, generator=g, device=DEV))
        s.k, s.v = _normal(g, (sum(lens), 2 * Hkv, hd), dt).split([Hkv, Hkv], dim=1)
        return s
    if s.kind == "fork":
        n, each, n_pages = case["n"], case["each"], case["n_pages"]
        lens = _shuffled(g, _spread(n, case["lo"], case["hi"]))
        slots = n * (1 + each)
        place = torch.randperm(slots, generator=g, device=DEV)
        width = _cdiv(case["hi"], PAGE) + 4
        all_lens = torch.zeros(slots, dtype=torch.int32, device=DEV)
        all_lens[place[:n]] = lens
        s.src = place[:n].repeat_interleave(each).to(torch.int32)
        s.dst = place[n:].to(torch.int32)
        s.losers = s.dst[torch.randperm(n * each, generator=g, device=DEV)[: _cdiv(n * each, 2)]].contiguous()
        s.pool = _normal(g, (case["layers"], n_pages, 2, Hkv, PAGE, hd), dt)
        _book(s, slots, width, n_pages, (all_lens + PAGE - 1) // PAGE, all_lens,
              torch.randperm(n_pages, generator=g, device=DEV))
        return s
    # compact: `moves` of the live pages lie at or above the live count; a
    # third of the slots are forks that share their pages with another slot
    slots, width, n_pages, live, moves = (case[k] for k in ("slots", "width", "n_pages", "live", "moves"))
    s.pool = _normal(g, (case["layers"], n_pages, 2, Hkv, PAGE, hd), dt)
    low = torch.randperm(live, generator=g, device=DEV)[moves:]
    high = live + torch.randperm(n_pages - live, generator=g, device=DEV)[:moves]
    ids = torch.cat([low, high])[torch.randperm(live, generator=g, device=DEV)]
    first = slots - slots // 3
    need = torch.tensor([live // first + (1 if i < live % first else 0) for i in range(first)], dtype=torch.int32, device=DEV)
    need = torch.cat([need, torch.zeros(slots - first, dtype=torch.int32, device=DEV)])
    _book(s, slots, width, n_pages, need, need * PAGE, ids)
    ref, table, lens = _parts(s, s.book)
    share = torch.arange(slots - first, device=DEV) % first
    table[first:] = table[share]
    lens[first:] = lens[share]
    ref.index_add_(0, table[first:].clamp(min=0).flatten().long(), (table[first:] >= 0).flatten().to(torch.int32))
    return s


def _table(g, need, width, ids):
    """A page table whose rows take `need` pages each, in the order of `ids`."""
    at = torch.arange(width, device=DEV)[None] + (need.cumsum(0) - need)[:, None]
    return torch.where(torch.arange(width, device=DEV)[None] < need[:, None], ids[at.clamp(max=len(ids) - 1)], -1).to(torch.int32)


def _book(s, slots, width, n_pages, used, lens, ids):
    """The book of a cache in one array: references of each page, the page table, the lengths."""
    s.slots_n, s.width, s.n_pages = slots, width, n_pages
    s.book = torch.zeros(n_pages + slots * width + slots, dtype=torch.int32, device=DEV)
    ref, table, ln = _parts(s, s.book)
    table.copy_(_table(None, used, width, ids))
    ln.copy_(lens)
    ref.index_add_(0, table.clamp(min=0).flatten().long(), (table >= 0).flatten().to(torch.int32))


def _parts(s, book):
    ref, table, lens = book.split([s.n_pages, s.slots_n * s.width, s.slots_n])
    return ref, table.view(s.slots_n, s.width), lens


# ------------------------------------------------------------------ one pass

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2606_10820_gb300 import serving
    if s.kind == "prompt":
        return serving.prompt_attention(s.q, s.k, s.v, s.cu, s.longest)
    if s.kind == "decode":
        return serving.paged_attention(s.q, s.pool, s.table, s.lens)
    if s.kind == "score":
        return serving.token_scores(s.logits, s.tokens, top=s.top, tau=s.tau)
    if s.kind == "grad":
        return serving.token_scores_grad(s.logits, s.tokens, s.g_logp, s.g_entropy, tau=s.tau)
    # the book is changed in place: a pass works on a copy, as a scheduler
    # keeps the one that it may go back to
    ref, table, lens = _parts(s, s.book.clone())
    if s.kind == "append":
        serving.pages_grow(ref, table, lens, s.slots, s.new_lens)
        serving.pages_append(s.pool[0], s.k, s.v, s.cu, table, lens, s.slots)
    elif s.kind == "fork":
        serving.pages_fork(s.pool, ref, table, lens, s.src, s.dst)
        serving.pages_free(ref, table, lens, s.losers)
    else:
        serving.pages_compact(s.pool, ref, table)
    return {"ref": ref, "table": table, "lens": lens, "pool": s.pool.view(torch.int16)}


def _run_plain(s):
    if s.kind == "prompt":
        return _plain_prompt(s)
    if s.kind == "decode":
        return _plain_decode(s)
    if s.kind in ("score", "grad"):
        return _plain_score(s)
    ref, table, lens = _parts(s, s.book.clone())
    {"append": _plain_append, "fork": _plain_fork, "compact": _plain_compact}[s.kind](s, ref, table, lens)
    return {"ref": ref, "table": table, "lens": lens, "pool": s.pool.view(torch.int16)}


def _attend(q, k, v, seen):
    """softmax(q k^T / sqrt(hd)) v over the keys that are seen; no key seen: zeros.
    q: [sequences][kv heads][heads of the group][rows][hd]; k, v: [sequences][kv heads][keys][hd]"""
    sc = (q.flatten(2, 3) @ k.transpose(-1, -2)).div_(math.sqrt(q.shape[-1])).view(*q.shape[:-1], -1)
    sc.masked_fill_(~seen, -math.inf)
    p = sc.sub_(sc.amax(-1, keepdim=True).clamp(min=-3e38)).exp_()
    return (p.flatten(2, 3) @ v).view(q.shape) / p.sum(-1, keepdim=True).clamp(min=1e-30)


def _plain_prompt(s):
    T, Hq, hd = s.q.shape
    Hkv, L = s.k.shape[1], s.longest
    cu = s.cu.long()
    pos = torch.arange(L, device=DEV)
    at = (cu[:-1, None] + pos).clamp(max=T - 1)
    q = s.q.float()[at].view(-1, L, Hkv, Hq // Hkv, hd).permute(0, 2, 3, 1, 4)
    k, v = (x.float()[at].transpose(1, 2) for x in (s.k, s.v))
    out = _attend(q, k, v, pos[None] <= pos[:, None]).permute(0, 3, 1, 2, 4).reshape(-1, L, Hq, hd)
    t = torch.arange(T, device=DEV)
    seq = torch.searchsorted(cu, t, right=True) - 1
    return out[seq, t - cu[seq]].to(s.q.dtype)


def _plain_decode(s):
    n, rows, Hq, hd = s.q.shape
    Hkv, L = s.pool.shape[2], s.table.shape[1] * PAGE
    kv = s.pool[s.table.clamp(min=0).long()].float().permute(2, 0, 3, 1, 4, 5).reshape(2, n, Hkv, L, hd)
    q = s.q.float().view(n, rows, Hkv, Hq // Hkv, hd).permute(0, 2, 3, 1, 4)
    last = s.lens.long()[:, None] - rows + torch.arange(rows, device=DEV)
    seen = torch.arange(L, device=DEV) <= last[..., None]
    out = _attend(q, kv[0], kv[1], seen[:, None, None])
    return out.permute(0, 3, 1, 2, 4).reshape(n, rows, Hq, hd).to(s.q.dtype)


def _free_pages(ref, n):
    """The n lowest pages without references."""
    ids = torch.arange(len(ref), device=DEV)
    return torch.where(ref == 0, ids, len(ref)).sort().values[:n]


def _plain_append(s, ref, table, lens):
    slots, cols = s.slots.long(), torch.arange(s.width, device=DEV)
    have, need = _pages(lens[slots]), _pages(s.new_lens)
    new = (cols >= have[:, None]) & (cols < need[:, None])
    ids = _free_pages(ref, s.n_pages).to(torch.int32)
    rank = (new.flatten().cumsum(0) - 1).view(new.shape)
    table[slots] = torch.where(new, ids[rank.clamp(min=0)], table[slots])
    lens[slots] = s.new_lens
    ref.index_add_(0, table[slots].clamp(min=0).flatten().long(), new.flatten().to(torch.int32))
    t = torch.arange(len(s.k), device=DEV)
    seq = torch.searchsorted(s.cu.long(), t, right=True) - 1
    at = s.new_lens[seq] - (s.cu[seq + 1] - s.cu[seq]) + t - s.cu[seq]
    page = table[slots[seq], at // PAGE].long()
    s.pool[0][page, 0, :, at % PAGE] = s.k
    s.pool[0][page, 1, :, at % PAGE] = s.v


def _pages(lens):
    return (lens + PAGE - 1) // PAGE


def _plain_fork(s, ref, table, lens):
    src, dst, losers, cols = s.src.long(), s.dst.long(), s.losers.long(), torch.arange(s.width, device=DEV)
    ln, rows = lens[src], table[src]
    full, part = (ln // PAGE)[:, None], ln % PAGE > 0
    new = _free_pages(ref, len(src))[(part.cumsum(0) - 1).clamp(min=0)]
    child = torch.where(cols < full, rows, torch.where((cols == full) & part[:, None], new[:, None].to(torch.int32), -1))
    ref.index_add_(0, child.clamp(min=0).flatten().long(), (child >= 0).flatten().to(torch.int32))
    old = rows.gather(1, full.clamp(max=s.width - 1).long())[:, 0].long()
    s.pool[:, new[part]] = s.pool[:, old[part]]
    table[dst], lens[dst] = child, ln
    gone = table[losers]
    ref.index_add_(0, gone.clamp(min=0).flatten().long(), -(gone >= 0).flatten().to(torch.int32))
    table[losers], lens[losers] = -1, 0


def _plain_compact(s, ref, table, lens):
    ids, used = torch.arange(s.n_pages, device=DEV), ref > 0
    high = used & (ids >= used.sum())
    src = ids[high]
    dst = ids[~used][: len(src)]
    s.pool[:, dst] = s.pool[:, src]
    to = ids.to(torch.int32)
    to[src] = dst.to(torch.int32)
    table.copy_(torch.where(table >= 0, to[table.clamp(min=0).long()], -1))
    ref[dst] = ref[src]
    ref[src] = 0


def _plain_score(s):
    x = s.logits.float() / s.tau
    m = x.amax(-1, keepdim=True)
    e = (x - m).exp()
    z = e.sum(-1, keepdim=True)
    lp, p = x - m - z.log(), e / z
    plogp = torch.where(p > 0, p * lp, torch.zeros_like(p))
    H = -plogp.sum(-1)
    has = s.tokens >= 0
    at = s.tokens.clamp(min=0)[:, None]
    out = {"logp": torch.where(has, lp.gather(1, at)[:, 0], torch.zeros_like(H)), "entropy": H, "lse": (m + z.log())[:, 0]}
    if s.kind == "score":
        if s.top:
            v, i = x.sort(dim=-1, descending=True, stable=True)
            out["top_ids"] = i[:, : s.top].to(torch.int32)
            out["top_logp"] = v[:, : s.top] - out["lse"][:, None]
        return out
    gl = torch.where(has, s.g_logp, torch.zeros_like(s.g_logp))[:, None]
    d = -gl * p - s.g_entropy[:, None] * (plogp + p * H[:, None])
    d.scatter_add_(1, at, gl)
    out["grad"] = (d / s.tau).to(s.logits.dtype)
    return out


# ------------------------------------------------------------------ work

def work(case):
    """Each input read once, each output written once; products counted as two
    operations a multiply-add over the visible pairs."""
    kind = case["kind"]
    size = 4 if case["dtype"] == "fp32" else 2
    if kind in ("score", "grad"):
        R, V = case["rows"], case["V"]
        wide = R * V * size * (2 if kind == "grad" else 1)
        return {"bytes": wide + R * (8 + 12 + 8 * case.get("top", 0) + (8 if kind == "grad" else 0)), "flops": 6 * R * V}
    hkv, hd = case["Hkv"], case["hd"]
    if kind == "compact":
        page = 2 * hkv * PAGE * hd * size
        return {"bytes": 2 * case["moves"] * case["layers"] * page + 8 * (case["n_pages"] + case["slots"] * case["width"]),
                "flops": 0}
    lens = _spread(case["n"], case["lo"], case["hi"])
    if kind == "prompt":
        T, pairs = sum(lens), sum(x * (x + 1) // 2 for x in lens)
        return {"bytes": 2 * T * (case["Hq"] + hkv) * hd * size, "flops": 4 * hd * case["Hq"] * pairs}
    if kind == "decode":
        rows = case["rows"]
        pairs = sum(max(0, x - rows + i + 1) for x in lens for i in range(rows))
        return {"bytes": sum(lens) * hkv * hd * 2 * size + 2 * case["n"] * rows * case["Hq"] * hd * size
                + 4 * sum(_cdiv(x, PAGE) for x in lens), "flops": 4 * hd * case["Hq"] * pairs}
    if kind == "append":
        pages = sum(_cdiv(x + case["old"], PAGE) for x in lens)
        return {"bytes": 4 * sum(lens) * hkv * hd * size + 4 * (case["n"] * _cdiv(case["hi"] + case["old"], PAGE) + 2 * pages),
                "flops": 0}
    parts = sum(1 for x in lens if x % PAGE) * case["each"]
    page = 2 * hkv * PAGE * hd * size * case["layers"]
    return {"bytes": 2 * parts * page + 8 * (case["n_pages"] + case["n"] * (1 + case["each"]) * (_cdiv(case["hi"], PAGE) + 5)),
            "flops": 0}


# ------------------------------------------------------------------ 64 bits

def exact(case, seed):
    """The definitions in 64 bits, one sequence (or block of rows) at a time."""
    s = prepare(case, seed)
    if s.kind in ("append", "fork", "compact"):
        return None                  # copies and whole numbers only
    if s.kind in ("score", "grad"):
        blocks = [_exact_rows(s, i, min(i + 256, case["rows"])) for i in range(0, case["rows"], 256)]
        out = {k: torch.cat([b[k] for b in blocks]) for k in blocks[0]}
        if s.kind == "score" and s.top:
            out["top_ids"] = None
        return out
    if s.kind == "prompt":
        cu = s.cu.tolist()
        return torch.cat([_exact_seq(s.q[a:b], s.k[a:b], s.v[a:b]) for a, b in zip(cu, cu[1:])])
    out = []
    for b, length in enumerate(s.lens.tolist()):
        kv = s.pool[s.table[b, : _cdiv(length, PAGE)].long()].permute(1, 0, 3, 2, 4).flatten(1, 2)[:, :length]
        out.append(_exact_seq(s.q[b], kv[0], kv[1]))
    return torch.stack(out)


def _exact_seq(q, k, v):
    """The last len(q) rows of a causal sequence of len(k) tokens, head by head."""
    n, Hq, hd = q.shape
    out = torch.zeros((n, Hq, hd), dtype=torch.float64, device=q.device)
    first = len(k) - n
    for h in range(Hq):
        kh, vh = (x[:, h * k.shape[1] // Hq].double() for x in (k, v))
        for a in range(0, n, 2048):
            b = min(n, a + 2048)
            if first + b <= 0:
                continue
            w = q[a:b, h].double() @ kh[: first + b].T / math.sqrt(hd)
            hidden = torch.arange(first + b, device=q.device)[None] > first + torch.arange(a, b, device=q.device)[:, None]
            w = torch.exp(w.masked_fill(hidden, -math.inf) - w.masked_fill(hidden, -math.inf).amax(1, keepdim=True))
            out[a:b, h] = torch.nan_to_num((w / w.sum(1, keepdim=True)) @ vh[: first + b])
    return out


def _exact_rows(s, a, b):
    x = s.logits[a:b].double() / s.tau
    lse = torch.logsumexp(x, 1)
    lp = x - lse[:, None]
    p = lp.exp()
    H = -torch.special.xlogy(p, p).sum(1)
    tok, rows = s.tokens[a:b], torch.arange(b - a, device=x.device)
    logp = torch.where(tok >= 0, lp[rows, tok.clamp(min=0)], 0.0)
    out = {"logp": logp, "entropy": H, "lse": lse}
    if s.kind == "score":
        if s.top:
            out["top_logp"] = lp.topk(s.top, 1).values
        return out
    gl, gh = torch.where(tok >= 0, s.g_logp[a:b], 0.0).double(), s.g_entropy[a:b].double()
    d = -gl[:, None] * p - gh[:, None] * (torch.special.xlogy(p, p) + p * H[:, None])
    d[rows, tok.clamp(min=0)] += gl
    out["grad"] = d / s.tau
    return out

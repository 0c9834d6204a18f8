"""Performance cases of rotated heads, attention over a shared prefix and the
policy loss (include/kforcing_serving.h).

Five kinds of case, each a plain dict:

  rotate  rotate_heads: the norms of the query and key heads and their rotary positions
  append  rotate_append: the same for new tokens of a paged cache, whose K and V rows
          go to their pages in the same pass
  back    rotate_heads_grad: the gradients of the heads and of the norms' weights
  shared  shared_attention: the newest rows of groups of sequences that begin with the
          same tokens, over a paged cache
  policy  policy_loss: the clipped policy loss with its KL and entropy terms, and the
          gradient of the logits

Model shapes are those of ``synth.WORKLOADS`` (12 heads of 64, vocabulary
50257, 16-token pages, prompts of 128 to 896 tokens), with grouped heads, and
generic wider ones.  Lengths are spread evenly over [lo, hi] and shuffled by the
seed, so that every seed asks for the same work.
"""
import math

import torch

own = False
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
PAGE = 16
EPS = 1e-6


def listed():
    return [
        # one token of each of eight sequences, rotation alone: latency
        {"name": "rotate_decode", "kind": "rotate", "T": 8, "Hq": 12, "Hkv": 4, "hd": 64, "rot": 64, "far": 1024,
         "theta": 1e4, "norm": False, "neighbours": False, "dtype": "bf16"},
        # a training batch of long documents, q and k views of one projection's output
        {"name": "rotate_batch", "kind": "rotate", "T": 16411, "Hq": 32, "Hkv": 8, "hd": 128, "rot": 128, "far": 131072,
         "theta": 1e6, "norm": True, "neighbours": False, "dtype": "bf16"},
        # a joint decode step of the paged serving workload at k = 4: eight rows per sequence
        {"name": "append_joint", "kind": "append", "n": 256, "lo": 8, "hi": 8, "old": 1016, "Hq": 12, "Hkv": 4, "hd": 64,
         "rot": 64, "theta": 1e4, "norm": True, "neighbours": False, "dtype": "bf16"},
        # a group of prompts, half of each head rotated, neighbouring elements paired
        {"name": "append_prompts", "kind": "append", "n": 24, "lo": 131, "hi": 1900, "old": 0, "Hq": 32, "Hkv": 8, "hd": 128,
         "rot": 64, "theta": 5e5, "norm": True, "neighbours": True, "dtype": "fp16"},
        # a short ragged training step
        {"name": "back_short", "kind": "back", "T": 509, "Hq": 12, "Hkv": 4, "hd": 64, "rot": 64, "far": 1024, "theta": 1e4,
         "norm": True, "neighbours": False, "dtype": "fp16"},
        # a training batch
        {"name": "back_batch", "kind": "back", "T": 16384, "Hq": 32, "Hkv": 8, "hd": 128, "rot": 128, "far": 8192, "theta": 1e6,
         "norm": True, "neighbours": False, "dtype": "bf16"},
        # eight candidates of one prompt: latency
        {"name": "shared_few", "kind": "shared", "groups": 1, "each": 8, "lo": 517, "hi": 517, "own_lo": 1, "own_hi": 61,
         "rows": 1, "Hq": 12, "Hkv": 4, "hd": 64, "dtype": "bf16"},
        # joint steps of sixteen candidates of each of sixteen prompts of the serving workload
        {"name": "shared_joint", "kind": "shared", "groups": 16, "each": 16, "lo": 128, "hi": 896, "own_lo": 8, "own_hi": 136,
         "rows": 8, "Hq": 12, "Hkv": 4, "hd": 64, "dtype": "fp16"},
        # candidates of a few long prompts, all at different lengths
        {"name": "shared_groups", "kind": "shared", "groups": 8, "each": 16, "lo": 1003, "hi": 4099, "own_lo": 1, "own_hi": 700,
         "rows": 1, "Hq": 32, "Hkv": 8, "hd": 128, "dtype": "fp16"},
        # many answers about one long document
        {"name": "shared_document", "kind": "shared", "groups": 1, "each": 64, "lo": 32771, "hi": 32771, "own_lo": 1,
         "own_hi": 1024, "rows": 1, "Hq": 32, "Hkv": 8, "hd": 128, "dtype": "bf16"},
        # the tokens of a few answers
        {"name": "policy_few", "kind": "policy", "rows": 61, "V": 50257, "tau": 1.0, "kl": 0.05, "entropy": 0.01, "dtype": "fp32"},
        # the tokens of a rollout batch
        {"name": "policy_batch", "kind": "policy", "rows": 4096, "V": 50257, "tau": 0.8, "kl": 0.02, "entropy": 0.001,
         "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    """A whole number from lo to hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rotate", "append", "back", "shared", "shared", "policy"])
    if kind == "policy":
        V, dtype = _log(rng, 1000, 130000), rng.choice(["bf16", "fp16", "fp32"])
        rows = _log(rng, 1, max(2, int(4096 * 50257 / (V * (2 if dtype == "fp32" else 1)))))
        return {"kind": "policy", "rows": min(rows, 8192), "V": V, "tau": rng.choice([1.0, 0.7, 1.3]),
                "kl": rng.choice([0.0, 0.02, 0.1]), "entropy": rng.choice([0.0, 0.003]), "dtype": dtype}
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    hkv, hd = rng.choice([1, 2, 4, 8]), rng.choice([64, 128])
    hq = hkv * rng.choice([1, 2, 3, 4, 8])
    if kind == "shared":
        hq = min(hq, 32)
        hi = _log(rng, 20, 33000)
        own_hi = _log(rng, 8, 1024)
        # at most the listed document's scores, and its keys
        each = _log(rng, 2, max(2, min(64, int(64 * 33000 * 32 / ((hi + own_hi) * hq)))))
        groups = _log(rng, 1, max(1, min(64, int(64 * 33000 * 32 / ((hi + own_hi) * hq * each)), 65536 // (hi + each * own_hi))))
        return {"kind": "shared", "groups": groups, "each": each, "lo": max(16, int(hi * rng.uniform(0.1, 1.0))), "hi": hi,
                "own_lo": rng.choice([8, max(8, own_hi // 2)]), "own_hi": own_hi, "rows": rng.choice([1, 1, 1, 2, 3, 5, 8]),
                "Hq": hq // hkv * hkv, "Hkv": hkv, "hd": hd, "dtype": dtype}
    head = {"Hq": hq, "Hkv": hkv, "hd": hd, "rot": rng.choice([hd, hd, hd // 2]), "theta": rng.choice([1e4, 5e5]),
            "norm": rng.random() < 0.7, "neighbours": rng.random() < 0.3, "dtype": dtype}
    most = 16384 * 40 * 128 // ((hq + hkv) * hd)
    if kind == "append":
        hi = _log(rng, 1, 1900)
        n = _log(rng, 1, max(1, min(256, most // (2 * hi))))
        return {"kind": "append", "n": n, "lo": max(1, int(hi * rng.uniform(0.1, 1.0))), "hi": hi,
                "old": rng.choice([0, 0, 5, 16, rng.randint(1, 1000)]), **head}
    return {"kind": kind, "T": _log(rng, 1, min(40000, most)), "far": _log(rng, 100, 1000000), **head}


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


def _pages(lens):
    return (lens + PAGE - 1) // PAGE


def _table(need, width, ids):
    """A page table whose rows take `need` pages each, in the order of `ids`."""
    at = torch.arange(width, device=DEV)[None] + (need.cumsum(0) - need)[:, None]
    return torch.where(torch.arange(width, device=DEV)[None] < need[:, None], ids[at.clamp(max=len(ids) - 1)], -1).to(torch.int32)


class _State:
    pass


def prepare(case, seed):
    s, g = _State(), torch.Generator(device=DEV).manual_seed(seed & 0x7FFFFFFF)
    s.kind = case["kind"]
    if s.kind == "policy":
        return _prepare_policy(s, g, case)
    if s.kind == "shared":
        return _prepare_shared(s, g, case)
    Hq, Hkv, hd, dt = case["Hq"], case["Hkv"], case["hd"], case["dtype"]
    s.freq = case["theta"] ** (-2.0 * torch.arange(case["rot"] // 2, dtype=torch.float64, device=DEV) / case["rot"])
    s.eps, s.neighbours, s.q_weight, s.k_weight = None, case["neighbours"], None, None
    if case["norm"]:
        s.eps = EPS
        s.q_weight, s.k_weight = (1 + 0.2 * _normal(g, (hd,), dt) for _ in range(2))
    if s.kind == "append":
        lens, old, n = _spread(case["n"], case["lo"], case["hi"]), case["old"], case["n"]
        cnt = _shuffled(g, lens)
        s.starts, s.slots = _starts(cnt), torch.randperm(n, generator=g, device=DEV).to(torch.int32)
        width = _cdiv(case["hi"] + old, PAGE)
        s.lens = torch.zeros(n, dtype=torch.int32, device=DEV)
        s.lens[s.slots.long()] = cnt + old
        # (of the tokens that a sequence had before only the last page is in this pool's upper part)
        n_pages = sum(_cdiv(x + old, PAGE) for x in lens) + 3
        s.pool = _normal(g, (n_pages, 2, Hkv, PAGE, hd), dt)
        s.table = _table(_pages(s.lens), width, torch.randperm(n_pages, generator=g, device=DEV))
        s.q, s.k, s.v = _normal(g, (sum(lens), Hq + 2 * Hkv, hd), dt).split([Hq, Hkv, Hkv], dim=1)
        return s
    T = case["T"]
    s.q, s.k, _ = _normal(g, (T, Hq + 2 * Hkv, hd), dt).split([Hq, Hkv, Hkv], dim=1)
    s.pos = torch.randint(0, case["far"], (T,), generator=g, device=DEV, dtype=torch.int32)
    if s.kind == "back":
        s.dq, s.dk = _normal(g, (T, Hq, hd), dt) * 0.01, _normal(g, (T, Hkv, hd), dt) * 0.01
    return s


def _prepare_shared(s, g, case):
    n, each, Hkv, hd, dt = case["groups"], case["each"], case["Hkv"], case["hd"], case["dtype"]
    s.shared = _shuffled(g, _spread(n, case["lo"], case["hi"]))
    own_lens = _shuffled(g, _spread(n * each, max(case["own_lo"], case["rows"]), max(case["own_hi"], case["rows"])))
    s.groups = torch.arange(0, n * each + 1, each, dtype=torch.int32, device=DEV)
    pre = s.shared.repeat_interleave(each)
    s.lens = pre + own_lens
    # the full pages of a group's prefix are in all of its tables; what follows is each sequence's own, the
    # rest of the prefix copied to its first page (as a fork leaves it)
    full = s.shared // PAGE
    need = torch.cat([full, _pages(s.lens) - pre // PAGE])
    n_pages, width = int(need.sum()), int(_pages(s.lens).max())
    s.pool = _normal(g, (n_pages, 2, Hkv, PAGE, hd), dt)
    ids = _table(need, width, torch.randperm(n_pages, generator=g, device=DEV))
    group = torch.arange(n * each, device=DEV) // each
    col = torch.arange(width, device=DEV)[None]
    k = full.repeat_interleave(each)[:, None]
    s.table = torch.where(col < k, ids[group], ids[n:].gather(1, (col - k).clamp(min=0).long()))
    first = s.table.gather(1, k.long())[:, 0].long()
    rest = (pre % PAGE)[:, None] > torch.arange(PAGE, device=DEV)
    s.pool[first] = torch.where(rest[:, None, None, :, None], s.pool[first[group * each]], s.pool[first])
    s.q = _normal(g, (n * each, case["rows"], case["Hq"], hd), dt)
    # (what a scheduler knows of its own requests)
    s.host = (s.shared.tolist(), s.lens.tolist(), each)
    return s


def _prepare_policy(s, g, case):
    R, V, dt = case["rows"], case["V"], case["dtype"]
    s.logits = (_normal(g, (R, V), dt) * 3).to(TYPES[dt])
    if R > 2:
        # a grammar's mask on one row: most of the vocabulary is closed
        s.logits[1, V // 50:] = -math.inf
    s.tau, s.kl, s.entropy, s.clip = case["tau"], case["kl"], case["entropy"], (0.2, 0.28)
    s.tokens = torch.empty(R, dtype=torch.int64, device=DEV)
    lp = torch.empty(R, device=DEV)
    for a in range(0, R, 1024):
        x = s.logits[a:a + 1024].float() / s.tau
        u = torch.rand(x.shape, generator=g, device=DEV).clamp(1e-20, 1 - 1e-7)
        # tokens as the policy draws them, and their scores
        s.tokens[a:a + 1024] = (x - (-u.log()).log()).argmax(-1)
        lp[a:a + 1024] = x.gather(1, s.tokens[a:a + 1024, None])[:, 0] - x.logsumexp(-1)
    # the policy that drew them is a few steps old; ratios are kept off the clip's two ends, where the
    # gradient jumps and a last bit would choose the side
    step = torch.randn(R, generator=g, device=DEV) * 0.2
    for end in (math.log(1 - s.clip[0]), math.log(1 + s.clip[1])):
        step = torch.where((step - end).abs() < 1e-3, step + 2e-3, step)
    s.old_logp, s.ref_logp = lp - step, lp + torch.randn(R, generator=g, device=DEV) * 0.1
    s.advantage = torch.randn(R, generator=g, device=DEV)
    if R > 2:
        s.tokens[2] = -1              # padding: no token
    s.weight = torch.full((R,), 1.0 / R, device=DEV)
    if R > 5:
        s.weight[5] = 0.0             # a row that the loss leaves out
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2606_10820_gb300 import serving
    if s.kind == "policy":
        return serving.policy_loss(s.logits, s.tokens, s.old_logp, s.advantage, ref_logp=s.ref_logp, weight=s.weight, clip=s.clip,
                                   kl_weight=s.kl, entropy_weight=s.entropy, tau=s.tau)
    if s.kind == "shared":
        return serving.shared_attention(s.q, s.pool, s.table, s.lens, s.groups, s.shared)
    how = {"q_weight": s.q_weight, "k_weight": s.k_weight, "eps": s.eps, "neighbours": s.neighbours}
    if s.kind == "rotate":
        return serving.rotate_heads(s.q, s.k, s.pos, s.freq, **how)
    if s.kind == "append":
        return serving.rotate_append(s.q, s.k, s.v, s.pool, s.starts, s.table, s.lens, s.slots, s.freq, **how), s.pool
    grads = serving.rotate_heads_grad(s.dq, s.dk, s.q, s.k, s.pos, s.freq, **how)
    return [grads[x] for x in ("q", "k", "q_weight", "k_weight") if grads.get(x) is not None]


def _run_plain(s):
    if s.kind == "policy":
        return _plain_policy(s)
    if s.kind == "shared":
        return _plain_shared(s)
    if s.kind == "rotate":
        return tuple(_plain_rotate(x, s.pos, s, w).to(x.dtype) for x, w in ((s.q, s.q_weight), (s.k, s.k_weight)))
    if s.kind == "append":
        t = torch.arange(len(s.k), device=DEV)
        seq = torch.searchsorted(s.starts.long(), t, right=True) - 1
        slot = s.slots[seq].long()
        at = s.lens[slot] - s.starts[seq + 1] + t
        page = s.table[slot, at // PAGE].long()
        s.pool[page, 0, :, at % PAGE] = _plain_rotate(s.k, at, s, s.k_weight).to(s.k.dtype)
        s.pool[page, 1, :, at % PAGE] = s.v
        return _plain_rotate(s.q, at, s, s.q_weight).to(s.q.dtype), s.pool
    return _plain_back(s)


def _turned(x, cos, sin, neighbours):
    """The first 2 len(cos) elements of the heads, each pair turned by its angle."""
    half = cos.shape[-1]
    y = x.clone()
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if neighbours else (slice(0, half), slice(half, 2 * half))
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    return y


def _angles(s, pos):
    """Cosine and sine of each position's angles, from 64 bits: those of far positions are large."""
    angle = pos.double()[:, None, None] * s.freq
    return angle.cos().float(), angle.sin().float()


def _plain_rotate(x, pos, s, weight):
    x = x.float()
    if s.eps is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + s.eps)
        if weight is not None:
            x = x * weight.float()
    return _turned(x, *_angles(s, pos), s.neighbours)


def _plain_back(s):
    cos, sin = _angles(s, s.pos)
    dx, dw = [], []
    for g, x, w in ((s.dq, s.q, s.q_weight), (s.dk, s.k, s.k_weight)):
        g = _turned(g.float(), cos, -sin, s.neighbours)
        if s.eps is not None:
            r = torch.rsqrt(x.float().square().mean(-1, keepdim=True) + s.eps)
            xh = x.float() * r
            if w is not None:
                dw.append((g * xh).sum((0, 1), dtype=torch.float64).float())
                g = g * w.float()
            g = r * (g - xh * (g * xh).mean(-1, keepdim=True))
        dx.append(g.to(x.dtype))
    return dx + dw


def _plain_shared(s):
    B, rows, Hq, hd = s.q.shape
    Hkv = s.pool.shape[2]
    shared, lens, each = s.host
    out = []
    for i, pre in enumerate(shared):
        b0, b1 = i * each, (i + 1) * each
        q = s.q[b0:b1].float().view(each, rows, Hkv, Hq // Hkv, hd).permute(2, 0, 1, 3, 4)      # [Hkv, each, rows, G, hd]
        # the prefix once, for all rows of the group
        kv = s.pool[s.table[b0, : _cdiv(pre, PAGE)].long()].float().permute(1, 2, 0, 3, 4).flatten(2, 3)[:, :, :pre]
        score = (q.reshape(Hkv, -1, hd) @ kv[0].transpose(-1, -2)).view(Hkv, each, -1, pre)
        # each sequence's own keys
        cols = slice(pre // PAGE, _cdiv(max(lens[b0:b1]), PAGE))
        mine = s.pool[s.table[b0:b1, cols].clamp(min=0).long()].float().permute(2, 3, 0, 1, 4, 5).flatten(3, 4)
        pos = pre // PAGE * PAGE + torch.arange(mine.shape[3], device=DEV)
        last = s.lens[b0:b1, None] - rows + torch.arange(rows, device=DEV)
        seen = ((pos >= pre) & (pos <= last[..., None])).repeat_interleave(Hq // Hkv, 1)        # [each, rows x G, keys]
        tail = q.flatten(2, 3) @ mine[0].transpose(-1, -2)
        score = torch.cat([score, tail.masked_fill_(~seen, -math.inf)], -1).div_(math.sqrt(hd))
        p = score.sub_(score.amax(-1, keepdim=True)).exp_()
        o = (p[..., :pre].reshape(Hkv, -1, pre) @ kv[1]).view(Hkv, each, -1, hd) + p[..., pre:] @ mine[1]
        o = o / p.sum(-1, keepdim=True)
        out.append(o.view(Hkv, each, rows, -1, hd).permute(1, 2, 0, 3, 4).reshape(each, rows, Hq, hd))
    return torch.cat(out).to(s.q.dtype)


def _plain_policy(s):
    x = s.logits.float() / s.tau
    m = x.amax(-1, keepdim=True)
    e = (x - m).exp()
    z = e.sum(-1, keepdim=True, dtype=torch.float64)
    logz = z.log()
    lp, p = (x - m) - logz.float(), e / z.float()
    plogp = torch.where(p > 0, p * lp, torch.zeros_like(p))
    H = -plogp.sum(-1, dtype=torch.float64)
    has, at = s.tokens >= 0, s.tokens.clamp(min=0)[:, None]
    # each row's numbers in 64 bits: the ratio is compared with the clip's ends
    logp = torch.where(has, (x.gather(1, at) - m).double()[:, 0] - logz[:, 0], 0.0)
    adv, weight = s.advantage.double(), torch.where(has, s.weight, torch.zeros_like(s.weight)).double()
    ratio = torch.where(has, (logp - s.old_logp.double()).exp(), 1.0)
    clipped = ratio.clamp(1 - s.clip[0], 1 + s.clip[1])
    u = torch.where(has, s.ref_logp.double() - logp, 0.0)
    kl = u.exp() - 1 - u
    gain = torch.minimum(ratio * adv, clipped * adv)
    loss = weight * (s.kl * kl - gain - s.entropy * H)
    open_ = ratio * adv <= clipped * adv
    gl = (weight * (s.kl * (1 - u.exp()) - torch.where(open_, ratio * adv, 0.0))).float()[:, None]
    gh = (-weight * s.entropy).float()[:, None]
    d = -gl * p - gh * (plogp + p * H.float()[:, None])
    d.scatter_add_(1, at, gl)
    out = {"loss": loss, "logp": logp, "entropy": H, "ratio": ratio, "kl": kl}
    return {**{k: v.float() for k, v in out.items()}, "grad": (d / s.tau).to(s.logits.dtype)}


# ------------------------------------------------------------------ work

def work(case):
    """Each input read once, each output written once; products counted as two
    operations a multiply-add over the visible pairs."""
    kind = case["kind"]
    size = 4 if case["dtype"] == "fp32" else 2
    if kind == "policy":
        R, V = case["rows"], case["V"]
        return {"bytes": 2 * R * V * size + R * (8 + 4 * 4 + 4 * 5), "flops": 8 * R * V}
    hq, hkv, hd = case["Hq"], case["Hkv"], case["hd"]
    if kind == "shared":
        n, each, rows = case["groups"], case["each"], case["rows"]
        pre = sum(_spread(n, case["lo"], case["hi"]))
        mine = sum(_spread(n * each, max(case["own_lo"], rows), max(case["own_hi"], rows)))
        pairs = rows * (each * pre + mine) - n * each * rows * (rows - 1) // 2
        return {"bytes": (pre + mine) * hkv * hd * 2 * size + 2 * n * each * rows * hq * hd * size, "flops": 4 * hd * hq * pairs}
    if kind == "append":
        T = sum(_spread(case["n"], case["lo"], case["hi"]))
        return {"bytes": 2 * T * (hq + 2 * hkv) * hd * size, "flops": 6 * T * (hq + hkv) * hd}
    T = case["T"]
    if kind == "rotate":
        return {"bytes": 2 * T * (hq + hkv) * hd * size + 4 * T, "flops": 6 * T * (hq + hkv) * hd}
    # (without norms the gradient needs no heads)
    return {"bytes": (3 if case["norm"] else 2) * T * (hq + hkv) * hd * size + 4 * T, "flops": 12 * T * (hq + hkv) * hd}


# ------------------------------------------------------------------ 64 bits

def exact(case, seed):
    """The definitions in 64 bits, one sequence (or block of rows) at a time."""
    s = prepare(case, seed)
    if s.kind == "policy":
        blocks = [_exact_policy(s, i, min(i + 256, case["rows"])) for i in range(0, case["rows"], 256)]
        return {k: torch.cat([b[k] for b in blocks]) for k in blocks[0]}
    if s.kind == "shared":
        out = []
        for b, length in enumerate(s.lens.tolist()):
            kv = s.pool[s.table[b, : _cdiv(length, PAGE)].long()].permute(1, 0, 3, 2, 4).flatten(1, 2)[:, :length]
            out.append(_exact_rows(s.q[b], kv[0], kv[1]))
        return torch.stack(out)
    if s.kind == "rotate":
        return _exact_heads(s, s.q, s.pos, s.q_weight), _exact_heads(s, s.k, s.pos, s.k_weight)
    if s.kind == "append":
        pool, pos = s.pool.double(), []
        starts, slots, lens, table = s.starts.tolist(), s.slots.tolist(), s.lens.tolist(), s.table.long()
        for i, slot in enumerate(slots):
            count = starts[i + 1] - starts[i]
            pos.append(torch.arange(lens[slot] - count, lens[slot], device=DEV))
        pos = torch.cat(pos)
        k = _exact_heads(s, s.k, pos, s.k_weight)
        rows = torch.repeat_interleave(s.slots.long(), (s.starts[1:] - s.starts[:-1]).long())
        page = table[rows, pos // PAGE]
        for h in range(case["Hkv"]):
            pool[page, 0, h, pos % PAGE] = k[:, h]
            pool[page, 1, h, pos % PAGE] = s.v[:, h].double()
        return _exact_heads(s, s.q, pos, s.q_weight), pool
    # each pair of elements as a complex number: the rotation's transpose is its conjugate
    dx, dw = [], []
    for dy, x, w in ((s.dq, s.q, s.q_weight), (s.dk, s.k, s.k_weight)):
        d = _as_complex_turn(s, dy.double(), s.pos, -1)
        if s.eps is not None:
            x = x.double()
            norm = (x.pow(2).mean(-1, keepdim=True) + s.eps).sqrt()
            if w is not None:
                dw.append((d * x / norm).sum((0, 1)))
                d = d * w.double()
            d = d / norm - x * (d * x).mean(-1, keepdim=True) / norm ** 3
        dx.append(d)
    return dx + dw


def _as_complex_turn(s, x, pos, sign):
    rot = 2 * len(s.freq)
    head = x[..., :rot]
    pair = head.reshape(*head.shape[:-1], rot // 2, 2) if s.neighbours else head.reshape(*head.shape[:-1], 2, rot // 2).transpose(-1, -2)
    angle = sign * pos.double()[:, None] * s.freq[None]
    turned = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * torch.polar(torch.ones_like(angle), angle)[:, None])
    turned = turned if s.neighbours else turned.transpose(-1, -2)
    return torch.cat([turned.reshape(head.shape), x[..., rot:]], -1)


def _exact_heads(s, x, pos, weight):
    x = x.double()
    if s.eps is not None:
        x = x / (x.pow(2).mean(-1, keepdim=True) + s.eps).sqrt()
        if weight is not None:
            x = x * weight.double()
    return _as_complex_turn(s, x, pos, 1)


def _exact_rows(q, k, v):
    """The last len(q) rows of a causal sequence of len(k) tokens."""
    n, Hq, hd = q.shape
    Hkv = k.shape[1]
    qh = q.double().view(n, Hkv, Hq // Hkv, hd).permute(1, 0, 2, 3).reshape(Hkv, -1, hd)
    w = torch.bmm(qh, k.double().permute(1, 2, 0)) / math.sqrt(hd)
    last = (len(k) - n + torch.arange(n, device=q.device)).repeat_interleave(Hq // Hkv)
    hidden = torch.arange(len(k), device=q.device)[None] > last[:, None]
    p = torch.softmax(w.masked_fill(hidden, -math.inf), -1)
    o = torch.bmm(p, v.double().transpose(0, 1)).view(Hkv, n, Hq // Hkv, hd)
    return o.permute(1, 0, 2, 3).reshape(n, Hq, hd)


def _exact_policy(s, a, b):
    logprob = torch.log_softmax(s.logits[a:b].double() / s.tau, 1)
    p = logprob.exp()
    H = -torch.special.xlogy(p, p).sum(1)
    tok, rows = s.tokens[a:b], torch.arange(b - a, device=s.logits.device)
    out = {k: torch.zeros(b - a, dtype=torch.float64, device=p.device) for k in ("loss", "logp", "entropy", "ratio", "kl")}
    out["entropy"], out["ratio"] = H, out["ratio"] + 1
    has = tok >= 0
    lp = logprob[rows, tok.clamp(min=0)]
    r = torch.exp(lp - s.old_logp[a:b].double())
    u = s.ref_logp[a:b].double() - lp
    A, w = s.advantage[a:b].double(), s.weight[a:b].double() * has
    kl = torch.expm1(u) - u
    high, low = r > 1 + s.clip[1], r < 1 - s.clip[0]
    stopped = (high & (A > 0)) | (low & (A < 0))
    used = torch.where(A > 0, r.clamp(max=1 + s.clip[1]), r.clamp(min=1 - s.clip[0]))
    out["loss"] = w * (s.kl * kl - used * A - s.entropy * H)
    for k, v in (("logp", lp), ("ratio", r), ("kl", kl)):
        out[k] = torch.where(has, v, out[k])
    gl = w * (-s.kl * torch.expm1(u) - torch.where(stopped, 0.0, r * A))
    gh = -w * s.entropy
    d = -gl[:, None] * p - gh[:, None] * (torch.special.xlogy(p, p) + p * H[:, None])
    d[rows, tok.clamp(min=0)] += gl
    out["grad"] = d / s.tau
    return out

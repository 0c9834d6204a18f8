"""rotate_heads, rotate_append and rotate_heads_grad of heads that hold infinities: elements that are not rotated stay as they are,
whatever is beside them, and a pair is spoilt by its own elements alone (needs a GB300)."""
import math

import pytest

from test_gpu_rotate import cache, gen, make, near, sv, turn  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
HEADS = [(64, 16), (64, 32), (64, 48), (64, 0), (128, 64), (128, 112), (128, 16), (128, 0)]


def same_bits(a, b):
    return torch.equal(a.contiguous().view(torch.int16), b.contiguous().view(torch.int16))


def wild(x, rot, seed):
    """The elements past `rot` at the ends of the type, each one in many places: infinities, -0, the largest and the least."""
    f = torch.finfo(x.dtype)
    least = 2.0 ** -24 if x.dtype == torch.float16 else f.tiny
    some = torch.tensor([math.inf, -math.inf, -0.0, f.max, -f.max, least, 1.5, 0.0], device="cuda").to(x.dtype)
    at = torch.randint(0, len(some), x[..., rot:].shape, generator=gen(seed), device="cuda")
    x[..., rot:] = some[at]
    return x


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("hd,rot", HEADS)
def test_what_is_not_rotated_stays(sv, dtype, neighbours, hd, rot):  # noqa: F811
    q, k, v, pos, freq, _ = make(67, 7, 3, hd, rot, dtype, seed=rot)
    q, k = wild(q.clone(), rot, 1), wild(k.clone(), rot, 2)
    for got in (sv.rotate_heads(q, k, pos, freq, neighbours=neighbours),
                tuple(sv.rotate_heads_grad(q, k, q, k, pos, -freq, neighbours=neighbours)[x] for x in "qk")):
        for y, x in zip(got, (q, k)):
            assert same_bits(y[..., rot:], x[..., rot:])
            near(y[..., :rot], x[..., :rot], pos, freq, neighbours)
    # and on the way to the pages: 40 and 27 tokens of two sequences
    pool, starts, table, lens, which = cache([40, 27], [40, 27], [1, 0], 3, hd, 16, dtype, gen(3))
    at = torch.cat([torch.arange(40, device="cuda"), torch.arange(27, device="cuda")])
    y = sv.rotate_append(q, k, v, pool, starts, table, lens, which, freq, neighbours=neighbours)
    sv.status()
    slot = torch.tensor([1] * 40 + [0] * 27, device="cuda")
    held = pool[table[slot, at // 16].long(), 0, :, at % 16]
    for z, x in ((y, q), (held, k)):
        assert same_bits(z[..., rot:], x[..., rot:])
        near(z[..., :rot], x[..., :rot], at.int(), freq, neighbours)


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("hd,rot", [h for h in HEADS if h[1]])
@pytest.mark.parametrize("norm", [False, True])
def test_an_infinity_spoils_its_pair(sv, neighbours, hd, rot, norm):  # noqa: F811
    """One infinity a head, everywhere once.  Without norms only its pair (or, past them, nothing) is touched.  With norms the
    head's other elements are divided by infinity: zeros, and the pair of the infinity is no number."""
    q, k, _, _, freq, _ = make(hd, 2, 1, hd, rot, torch.bfloat16, seed=7)
    q, pos = q.clone(), torch.full((hd,), 3, dtype=torch.int32, device="cuda")
    at = torch.arange(hd, device="cuda")
    q[at, 0, at] = math.inf
    n = rot // 2
    other = torch.where(at >= rot, at, torch.where(at % 2 == 0, at + 1, at - 1) if neighbours else torch.where(at < n, at + n, at - n))
    pair = torch.zeros(hd, hd, dtype=torch.bool, device="cuda")
    pair[at, at] = pair[at, other] = True
    got = sv.rotate_heads(q, k, pos, freq, neighbours=neighbours, eps=1e-6 if norm else None)[0]
    spoilt = ~torch.isfinite(got[:, 0])
    assert torch.isfinite(got[:, 1]).all()
    if norm:
        assert spoilt.equal(pair) and (got[:, 0][~pair] == 0).all()
    else:
        # (3 freq is no multiple of a quarter turn: neither product of the pair is 0 times infinity)
        assert spoilt.equal(pair)
        clean = q.clone()
        clean[at, 0, at] = 0
        want = sv.rotate_heads(clean, k, pos, freq, neighbours=neighbours)[0]
        assert same_bits(got[:, 0][~pair], want[:, 0][~pair])

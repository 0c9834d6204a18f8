"""Steps that keep a part of their rows, over the book's pages: room ahead, lengths of the step's own,
rows that were not kept overwritten by the next step's (needs a GB300)."""
import pytest

from test_gpu_paged_attention import check, sv  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("Hq,Hkv,hd", [(6, 2, 64), (4, 2, 128)])
def test_kept_rows_stay_and_others_go(sv, Hq, Hkv, hd):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(hd)
    kept, rows, slots = [14, 1, 40], 5, i32([2, 0, 1])
    book = sv.new_book(40, 3, 8)
    pool = torch.full((40, 2, Hkv, 16, hd), float("nan"), device="cuda", dtype=torch.bfloat16)
    new = lambda n: torch.randn(n, 2 * Hkv, hd, generator=g, device="cuda").bfloat16()  # noqa: E731
    starts = lambda n: i32([sum(n[:i]) for i in range(len(n) + 1)])                      # noqa: E731

    def lens_of(at):          # by slot
        out = torch.zeros(3, dtype=torch.int32, device="cuda")
        out[slots.long()] = i32(at)
        return out

    truth = [new(n) for n in kept]
    sv.pages_grow(*book, slots, i32([n + rows for n in kept]))
    k, v = torch.cat(truth).split(Hkv, 1)
    sv.pages_append(pool, k, v, starts(kept), book[1], lens_of(kept), slots)
    for accepted in ([1, 5, 3], [4, 1, 5], [2, 2, 1], [5, 5, 5]):
        at = [n + rows for n in kept]
        sv.pages_grow(*book, slots, i32(at))
        step = [new(rows) for _ in kept]
        k, v = torch.cat(step).split(Hkv, 1)
        sv.pages_append(pool, k, v, starts([rows] * 3), book[1], lens_of(at), slots)
        q = torch.randn(3, rows, Hq, hd, generator=g, device="cuda").bfloat16()
        check(sv, q, pool, book[1][slots.long()].contiguous(), i32(at))
        kept = [n + a for n, a in zip(kept, accepted)]
        truth = [torch.cat([x, y[:a]]) for x, y, a in zip(truth, step, accepted)]
        for i, s in enumerate(slots.tolist()):
            pages = book[1][s, : -(-kept[i] // 16)].long()
            got = pool[pages].permute(1, 0, 3, 2, 4).flatten(1, 2)[:, : kept[i]]
            assert torch.equal(got[0], truth[i][:, :Hkv]) and torch.equal(got[1], truth[i][:, Hkv:])
    sv.status()

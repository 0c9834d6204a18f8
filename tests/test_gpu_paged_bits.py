"""paged_attention's bits: the same lengths, table width and pool size give the same ones, wherever the pages
lie; another width or pool size may take other kernels and stays within the operator's tolerance (needs a GB300)."""
import pytest

from test_gpu_paged_attention import check, make, sv  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("lens,rows,Hq,Hkv,hd,spare", [
    ([900, 17, 333], 8, 8, 2, 128, 9000), ([900, 17, 333], 8, 8, 2, 128, 5), ([3000, 1, 700], 8, 12, 4, 64, 5), ([40, 100], 1, 4, 2, 64, 5),
    ([20011], 1, 16, 2, 128, 5)])
def test_same_bits_wherever_the_pages_lie(sv, lens, rows, Hq, Hkv, hd, spare):  # noqa: F811
    q, pool, table, n = make(lens, rows, Hq, Hkv, hd, seed=9, spare=spare)
    want = check(sv, q, pool, table, n)
    for _ in range(3):
        perm = torch.randperm(len(pool), device="cuda")
        moved = torch.where(table >= 0, torch.argsort(perm)[table.clamp(min=0).long()].to(torch.int32), -1)
        assert torch.equal(want, sv.paged_attention(q, pool[perm].contiguous(), moved, n))


def test_wider_tables_and_pools_stay_within_the_tolerance(sv):  # noqa: F811
    q, pool, table, n = make([150, 33, 97], 8, 32, 4, 128, seed=3)
    for more in (0, 40, 3000):
        wide = torch.cat([table, torch.full((3, more), -1, dtype=torch.int32, device="cuda")], 1)
        check(sv, q, pool, wide, n)
        check(sv, q, torch.cat([pool, torch.zeros(more, *pool.shape[1:], dtype=pool.dtype, device="cuda")]), wide, n)

"""shared_attention at a size past what its own kernels count in: the rows of paged attention, to the bit (needs a GB300)."""
import pytest

from test_gpu_shared_attention import i32, make, sv  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def test_a_very_wide_table(sv):  # noqa: F811
    q, pool, table, lens, starts, shared = make([(40, [41 + i % 30 for i in range(200)]), (17, [20] * 56)], 1, 8, 8, 64, seed=1)
    wide = torch.full((256, 530000), -1, dtype=torch.int32, device="cuda")      # 0.5 GB
    wide[:, : table.shape[1]] = table
    got = sv.shared_attention(q, pool, wide, lens, starts, shared)
    sv.status()
    assert torch.equal(got, sv.paged_attention(q, pool, wide, lens)) and torch.isfinite(got).all()

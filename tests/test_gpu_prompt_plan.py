"""Calls of more than 128 prompts, whose items a block of its own lists, again and again: every row
is written every time (needs a GB300).  An output row of one token is its V row."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def test_every_row_of_many_prompts_every_time():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__ as g
    g.build()
    from paper_2606_10820_gb300 import serving as sv
    n = 1900
    q, k, v = (torch.randn(n, h, 64, device="cuda").bfloat16() for h in (2, 1, 1))
    starts = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    bad = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(300):
        out = sv.prompt_attention(q, k, v, starts, 1, out=torch.full_like(q, float("nan")))
        bad += (out != v.expand_as(out)).sum()
    sv.status()
    assert int(bad) == 0

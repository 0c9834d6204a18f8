"""Choices of the serving operators' host code by bounds that a caller may give loosely, without a GPU."""
import pytest

from host_calls import launches
from test_serving_host import OK, lib, prompt  # noqa: F401


def grid(lib, **kw):  # noqa: F811
    assert prompt(lib, **kw) == OK
    return launches(lib)[-1].grid[0]


@pytest.mark.parametrize("hd", [64, 128])
def test_a_loose_longest_keeps_the_pairs_of_a_full_grid(lib, hd):  # noqa: F811
    """64 prompts of 512 tokens: two heads an item, half as many CTAs, whether `longest` is theirs or the model's."""
    many = dict(hd=hd, n=64, T=64 * 512, Hq=32, Hkv=8, q_row=32 * hd, out_row=32 * hd, k_row=8 * hd, v_row=8 * hd,
                q_head=hd, k_head=hd, v_head=hd, out_head=hd)
    lib.fake_clear()
    pairs = grid(lib, longest=512, **many)
    assert pairs == (64 * 512 // 128 + 64) * 16
    for longest in (600, 4096, 131072, 524288):
        assert grid(lib, longest=longest, **many) == pairs


def test_one_long_prompt_of_few_heads_takes_single_sub_tiles(lib):  # noqa: F811
    one = dict(n=1, T=4096, Hq=8, Hkv=2)
    lib.fake_clear()
    assert grid(lib, longest=4096, **one) == grid(lib, longest=524288, **one) == (4096 // 128 + 1) * 8

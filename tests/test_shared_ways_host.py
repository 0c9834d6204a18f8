"""The kernels that shared_attention's sizes choose are those that shared_ways.py says, without a GPU; and its cases choose what they are listed under."""
import random

import pytest

import shared_ways
from host_calls import launches
from test_more_operators_host import _fresh, lib, serving_lib, shared  # noqa: F401
from test_serving_host import OK

KERNELS = {"paged": "paged", "rows": "rows", "tiles": "prefix"}


def chosen(lib, B, rows, Hq, Hkv, hd, n_pages, page, width, n):  # noqa: F811
    assert shared(lib, B=B, rows=rows, Hq=Hq, Hkv=Hkv, hd=hd, q_seq=rows * Hq * hd, q_row=Hq * hd, q_head=hd, n_pages=n_pages, page=page, width=width, n=n) == OK
    first = launches(lib)[0].kernel.split("k_")[1].split("<")[0]
    return next(w for w, k in KERNELS.items() if k == first)


def test_the_rule(lib):  # noqa: F811
    rng, seen = random.Random(1), {w: 0 for w in KERNELS}

    def some(lo, hi):
        return max(lo, min(hi, int(round(2 ** rng.uniform(0, 30) % (hi + 1)))))

    for _ in range(3000):
        Hkv = rng.choice([1, 2, 3, 4, 8])
        sizes = (some(1, 600), rng.choice([1, 1, 2, 3, 5, 8, 100]), Hkv * rng.choice([1, 2, 3, 4, 8]), Hkv, rng.choice([64, 128]), some(1, 60000),
                 rng.choice([16, 32, 48, 128]), some(1, 3000), some(1, 200))
        way = shared_ways.way_of(*sizes)
        seen[way] += 1
        assert chosen(lib, *sizes) == way, sizes
    assert min(seen.values()) > 200, seen


@pytest.mark.parametrize("way", KERNELS)
def test_the_cases(lib, way):  # noqa: F811
    for case in shared_ways.CASES[way]:
        assert shared_ways.way_of(*shared_ways.sizes_of(case)) == way == chosen(lib, *shared_ways.sizes_of(case)), (way, case[1:], shared_ways.sizes_of(case))

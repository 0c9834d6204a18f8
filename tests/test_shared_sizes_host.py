"""shared_attention takes every size that paged attention takes, without a GPU."""
import pytest

from host_calls import launches
from test_more_operators_host import _fresh, lib, refused, serving_lib, shared  # noqa: F401
from test_serving_host import OK, P


@pytest.mark.parametrize("size", [dict(B=4096, n=2, width=1 << 20), dict(B=300, n=2, width=1 << 20, Hq=64, Hkv=8), dict(B=1 << 20, rows=16, Hq=128, Hkv=128, n=3, width=4, hd=64),
                                  dict(B=(1 << 25), n=(1 << 24) + 1, width=2, Hq=1, Hkv=1), dict(B=1 << 25, n=2, width=3, Hq=8, Hkv=8)])
def test_sizes_past_the_own_kernels_counts(lib, size):  # noqa: F811
    call = dict(n_pages=1 << 30, **size)
    assert shared(lib, **call) == OK
    assert [x.kernel.split("k_")[1].split("<")[0] for x in launches(lib)][0] == "paged"
    a = dict(rows=1, Hq=8, Hkv=2, hd=128)
    a.update(size)
    assert lib.kf_op_shared_attention_work(a["B"], a["rows"], a["Hq"], a["Hkv"], a["hd"], 1 << 30, 16, a["width"], a["n"]) == \
        lib.kf_op_paged_attention_work(a["B"], a["rows"], a["Hq"], a["Hkv"], a["hd"], 16, a["width"])
    # what paged attention refuses, this one does
    assert refused(lib, "kf_op_shared_attention", shared(lib, **{**call, "width": 1 << 27, "work": P}))


def test_sizes_just_below_keep_their_kernels(lib):  # noqa: F811
    assert shared(lib, B=1000, n=2, width=1 << 18, n_pages=1 << 30) == OK
    assert "k_prefix" in launches(lib)[0].kernel

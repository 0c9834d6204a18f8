"""Outputs of kf_op_rotate_heads whose heads would lie over each other, without a GPU: refused exactly where two heads share an element."""
import random

import pytest

from host_calls import launches
from test_more_operators_host import _fresh, lib, refused, rotate, serving_lib  # noqa: F401
from test_serving_host import OK, P


def meet(T, H, row, head, hd):
    """By the elements themselves."""
    seen = set()
    for t in range(T):
        for h in range(H):
            at = range(t * row + h * head, t * row + h * head + hd)
            if not seen.isdisjoint(at):
                return True
            seen.update(at)
    return False


def far(T, H, row, head):
    return dict(T=T, Hq=H, Hkv=H, oq_row=row, oq_head=head, ok_row=1 << 20, ok_head=1 << 14)


@pytest.mark.parametrize("bad", [dict(oq_row=64), dict(oq_row=128), dict(oq_row=192), dict(oq_row=248), dict(ok_row=64), dict(ok_row=120),
                                 dict(T=2, oq_row=64, oq_head=64), dict(T=1 << 30, Hq=4096, q_row=1 << 20, oq_row=1 << 17, oq_head=64),
                                 dict(oq_row=64, oq_head=512), dict(oq=P, ok=P, ok_row=512, oq_row=512, k=4 * P),
                                 dict(oq=2 * P, ok=2 * P)])
def test_refused(lib, bad):  # noqa: F811
    assert refused(lib, "kf_op_rotate_heads", rotate(lib, **bad)) and not launches(lib)


@pytest.mark.parametrize("fine", [dict(oq_row=256), dict(oq_row=1 << 20, oq_head=1 << 10), dict(T=1, oq_row=64), dict(T=1, oq_row=0),
                                  dict(Hq=1, oq_row=64, oq_head=0), dict(oq_row=64, oq_head=64 * 9), dict(T=2, oq_row=192, oq_head=128, Hq=2),
                                  dict(T=1 << 30, Hq=2, Hkv=1, oq_row=64, oq_head=64 << 30)])
def test_taken(lib, fine):  # noqa: F811
    assert rotate(lib, **fine) == OK and len(launches(lib)) == 1


def test_every_layout_of_few_heads(lib):  # noqa: F811
    rng = random.Random(3)
    seen = {True: 0, False: 0}
    for _ in range(400):
        T, H, row, head = rng.randint(1, 6), rng.randint(1, 6), 8 * rng.randint(0, 60), 8 * rng.randint(0, 60)
        want = meet(T, H, row, head, 64)
        seen[want] += 1
        assert (rotate(lib, **far(T, H, row, head)) != OK) == want, (T, H, row, head)
        launches(lib)
    assert min(seen.values()) > 50

"""Host code of the rotated heads, of the attention over shared prefixes and of the policy loss, without a GPU: what they
refuse before any CUDA call, and which kernels their sizes choose."""
import ctypes

import pytest

from host_calls import launches
from test_serving_host import F32, I32, I64, OK, P, VP, lib as serving_lib, refused  # noqa: F401


@pytest.fixture(scope="module")
def lib(serving_lib):  # noqa: F811
    rows = [VP, I64, I64]
    turn = [VP, I32, I32, F32, VP, VP]
    serving_lib.kf_op_rotate_heads.argtypes = [I32, I64] + [I32] * 3 + rows * 2 + [VP] + turn + rows * 2 + [VP]
    serving_lib.kf_op_rotate_append.argtypes = [I32, I32, VP, VP, I64] + [I32] * 3 + rows * 3 + turn + [VP, VP, I32, I32, VP, I32, I32, VP, VP]
    serving_lib.kf_op_rotate_heads_grad.argtypes = [I32, I64] + [I32] * 3 + rows * 4 + [VP] + turn + [VP] * 6
    serving_lib.kf_op_rotate_heads_grad_work.argtypes, serving_lib.kf_op_rotate_heads_grad_work.restype = [I64, I32, I32, I32], I64
    serving_lib.kf_op_shared_attention.argtypes = [I32] * 6 + [VP] + [I64] * 3 + [VP, I64, I32, VP, I32, VP, I32, VP, VP, F32] + [VP] * 3
    serving_lib.kf_op_shared_attention_work.argtypes, serving_lib.kf_op_shared_attention_work.restype = [I32] * 5 + [I64, I32, I32, I32], I64
    serving_lib.kf_op_policy_loss.argtypes = [I32, I64, I32, VP, I64, VP, ctypes.c_double] + [VP] * 4 + [F32] * 4 + [VP] * 6 + [I64, VP]
    return serving_lib


@pytest.fixture(autouse=True)
def _fresh(lib):
    lib.fake_clear()


def rotate(lib, **kw):
    a = dict(type=1, T=9, Hq=4, Hkv=2, hd=64, q=P, q_row=512, q_head=64, k=P, k_row=512, k_head=64, pos=P, freq=P, n=32, nb=0, eps=1e-6,
             wq=P, wk=P, oq=P, oq_row=256, oq_head=64, ok=P, ok_row=128, ok_head=64, stream=None)
    a.update({"oq": 2 * P, "ok": 3 * P})
    a.update(kw)
    return lib.kf_op_rotate_heads(*a.values())


@pytest.mark.parametrize("bad", [dict(type=0), dict(type=3), dict(hd=96), dict(T=-1), dict(T=1 << 31), dict(Hq=0), dict(Hkv=0), dict(Hq=5000),
                                 dict(n=-8), dict(n=12), dict(n=40), dict(eps=float("nan")), dict(eps=float("inf")), dict(eps=-1.0), dict(wq=P + 2),
                                 dict(freq=None), dict(freq=P + 4), dict(pos=None), dict(pos=P + 2), dict(q=None), dict(q=P + 8), dict(k=None),
                                 dict(q_row=510), dict(k_head=-64), dict(oq=None), dict(ok=3 * P + 4), dict(oq_row=1 << 38), dict(oq=P),
                                 dict(ok=P, ok_row=128), dict(oq_row=0), dict(oq_head=32), dict(ok_head=0), dict(ok_row=8)])
def test_rotate_refusals(lib, bad):
    assert refused(lib, "kf_op_rotate_heads", rotate(lib, **bad))


def test_rotate_kernels(lib):
    def one(**kw):
        assert rotate(lib, **kw) == OK
        got = launches(lib)
        assert len(got) == 1
        return got[0]

    assert "k_rotate" in one().kernel and one(T=1 << 16).grid[0] == one(T=1 << 16, eps=-1.0, wq=None, wk=None).grid[0]
    # few tokens: the passes over the heads are split over warps; the heads of a pass stay together
    assert one(T=1, Hq=32, Hkv=8, hd=128, q_row=8192, k_row=8192, oq_head=128, ok_head=128).grid[0] * 4 >= 10
    assert rotate(lib, T=0, q=None, k=None, oq=None, ok=None, pos=None) == OK and not launches(lib)
    assert rotate(lib, n=0, freq=None) == OK
    # over the input itself
    assert rotate(lib, oq=P, oq_row=512, ok=P, ok_row=512) == OK


def append(lib, **kw):
    a = dict(type=1, n=3, which=P, starts=P, T=9, Hq=4, Hkv=2, hd=64, q=P, q_row=512, q_head=64, k=P, k_row=512, k_head=64, v=P, v_row=512,
             v_head=64, freq=P, nf=32, nb=1, eps=-1.0, wq=None, wk=None, oq=P, pool=P, n_pages=10, page=16, table=P, slots=3, width=4, lens=P,
             stream=None)
    a.update(kw)
    return lib.kf_op_rotate_append(*a.values())


@pytest.mark.parametrize("bad", [dict(type=0), dict(hd=32), dict(n=-1), dict(n=0), dict(n_pages=0), dict(slots=0), dict(width=-1), dict(page=0),
                                 dict(page=1 << 21), dict(width=1 << 28), dict(which=None), dict(starts=None), dict(pool=None), dict(pool=P + 8),
                                 dict(lens=None), dict(table=None), dict(v=None), dict(v_row=4), dict(oq=None), dict(oq=P + 2), dict(wq=P),
                                 dict(starts=P + 1)])
def test_append_refusals(lib, bad):
    assert refused(lib, "kf_op_rotate_append", append(lib, **bad))


def back(lib, **kw):
    a = dict(type=2, T=9, Hq=4, Hkv=2, hd=64, dq=P, dq_row=256, dq_head=64, dk=P, dk_row=128, dk_head=64, q=P, q_row=512, q_head=64, k=P, k_row=512,
             k_head=64, pos=P, freq=P, n=32, nb=0, eps=1e-6, wq=P, wk=P, gq=P, gk=P, gwq=P, gwk=P, work=P, stream=None)
    a.update(kw)
    return lib.kf_op_rotate_heads_grad(*a.values())


@pytest.mark.parametrize("bad", [dict(type=0), dict(T=-1), dict(dq=None), dict(dk=P + 8), dict(dk_row=100), dict(q=None), dict(k=None), dict(gq=None),
                                 dict(gk=P + 4), dict(pos=None), dict(wq=None), dict(gwk=P + 2), dict(work=None), dict(work=P + 16), dict(n=4)])
def test_back_refusals(lib, bad):
    assert refused(lib, "kf_op_rotate_heads_grad", back(lib, **bad))


def test_back_kernels(lib):
    def names(**kw):
        assert back(lib, **kw) == OK
        return [(x.kernel.split("k_")[1].split("<")[0], x.dependent) for x in launches(lib)]

    assert names() == [("back", False), ("join", True)]
    assert names(gwq=None, gwk=None, work=None) == [("back", False)]
    # without norms: the rotation back, of dq and dk alone
    assert names(eps=-1.0, wq=None, wk=None, gwq=None, gwk=None, q=None, k=None, work=None) == [("rotate", False)]
    for T in (1, 500, 100000):
        need = lib.kf_op_rotate_heads_grad_work(T, 4, 2, 64)
        assert back(lib, T=T) == OK and launches(lib)[0].grid[0] * 2 * 64 * 4 <= need
    assert lib.kf_op_rotate_heads_grad_work(0, 4, 2, 64) == 0


def shared(lib, **kw):
    a = dict(type=1, B=16, rows=1, Hq=8, Hkv=2, hd=128, q=P, q_seq=1024, q_row=1024, q_head=128, pool=P, n_pages=20000, page=16, table=P, width=1000,
             lens=P, n=2, groups=P, shared=P, scale=0.1, out=P, work=P, stream=None)
    a.update(kw)
    return lib.kf_op_shared_attention(*a.values())


@pytest.mark.parametrize("bad", [dict(type=0), dict(hd=32), dict(B=-1), dict(rows=0), dict(Hq=9), dict(page=8), dict(page=24), dict(width=-1),
                                 dict(n_pages=-1), dict(n_pages=1 << 31), dict(scale=-1.0), dict(scale=float("nan")), dict(q=None), dict(lens=None),
                                 dict(table=None), dict(pool=None), dict(out=P + 4), dict(q_head=100), dict(work=None), dict(work=P + 64), dict(n=-1),
                                 dict(n=0), dict(groups=None), dict(shared=None), dict(groups=P + 2)])
@pytest.mark.parametrize("width", [100, 1000])
def test_shared_refusals(lib, bad, width):
    assert refused(lib, "kf_op_shared_attention", shared(lib, **{"width": width, **bad}))


def test_shared_kernels(lib):
    def names(**kw):
        assert shared(lib, **kw) == OK
        return [(x.kernel.split("k_")[1].split("<")[0], x.dependent) for x in launches(lib)]

    # what reads the prefixes: tcgen05, tiles of few rows, or paged attention, by the reads that the table and the pool allow for
    assert names(B=64, Hq=32, Hkv=8, width=2000) == [("prefix", False), ("rows", True), ("add", True)]
    assert names(width=1000) == [("rows", False), ("add", True)]
    assert [x[0] for x in names(width=100)] == ["paged", "join"] == [x[0] for x in names(n_pages=100)]
    # nothing that is shared: paged attention
    assert [x[0] for x in names(n=16)] == ["paged", "join"] and [x[0] for x in names(n_pages=0, pool=None)] == ["paged", "join"]
    assert shared(lib, B=0, n=0) == OK and not launches(lib)
    assert lib.kf_op_shared_attention_work(16, 1, 8, 2, 128, 20000, 16, 1000, 2) > 2 * 16 * 8 * 128 * 4
    assert lib.kf_op_shared_attention_work(16, 1, 8, 2, 128, 20000, 16, 100, 2) == lib.kf_op_paged_attention_work(16, 1, 8, 2, 128, 16, 100)
    assert lib.kf_op_shared_attention_work(0, 1, 8, 2, 128, 20000, 16, 600, 2) == 0
    # sizes at their ends
    assert lib.kf_op_shared_attention_work(1 << 16, 1, 8, 2, 128, 1 << 30, 16, 1 << 10, 1 << 15) > 0
    assert lib.kf_op_shared_attention_work(1 << 20, 64, 64, 2, 128, 1 << 30, 16, 1 << 20, 2) == 0


def policy(lib, **kw):
    a = dict(type=0, R=9, V=100, logits=P, stride=100, tokens=P, tau=1.0, old=P, adv=P, ref=P, weight=P, low=0.2, high=0.2, klw=0.1, hw=0.1, loss=P,
             logp=P, entropy=P, ratio=P, kl=P, grad=2 * P, grad_stride=100, stream=None)
    a.update(kw)
    return lib.kf_op_policy_loss(*a.values())


@pytest.mark.parametrize("bad", [dict(type=3), dict(R=-1), dict(V=0), dict(V=1 << 20), dict(stride=99), dict(logits=None), dict(logits=P + 2),
                                 dict(tokens=None), dict(tokens=P + 4), dict(tau=0.0), dict(tau=float("nan")), dict(tau=1e-40), dict(tau=float("inf")),
                                 dict(old=None), dict(adv=None), dict(adv=P + 2), dict(ref=None), dict(low=-0.1), dict(low=1.5), dict(low=float("nan")),
                                 dict(high=-0.1), dict(high=float("nan")), dict(klw=float("inf")), dict(hw=float("nan")), dict(loss=None), dict(kl=None),
                                 dict(grad=None), dict(grad_stride=50), dict(grad=P, grad_stride=200)])
def test_policy_refusals(lib, bad):
    assert refused(lib, "kf_op_policy_loss", policy(lib, **bad))


def test_policy_kernels(lib):
    def one(**kw):
        assert policy(lib, **kw) == OK
        got = launches(lib)
        assert len(got) == 1 and "k_scores_grad" in got[0].kernel
        return got[0]

    assert one(ref=None, kl=None, klw=0.0, weight=None, high=float("inf")).cluster == 1
    assert one(R=1, V=50257, stride=50257, grad_stride=50257).cluster > 1
    assert policy(lib, R=0) == OK and not launches(lib)

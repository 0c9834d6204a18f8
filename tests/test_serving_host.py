"""Host code of the serving operators, without a GPU (host_calls.py): what they
refuse before any CUDA call, and which kernels their sizes choose."""
import ctypes

import pytest

import host_calls
from host_calls import launches

OK, E_ARG = 0, -1
P = 1 << 20     # an aligned device address that nothing reads
I32, I64, F32, VP = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_void_p


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    lib = host_calls.load(str(tmp_path_factory.mktemp("host")))
    lib.kf_op_prompt_attention.argtypes = [I32, I32, I64] + [I32] * 4 + [VP, I64, I64] * 4 + [VP, F32, VP, VP]
    lib.kf_op_prompt_attention_work.argtypes, lib.kf_op_prompt_attention_work.restype = [I32, I64], I64
    lib.kf_op_paged_attention.argtypes = [I32] * 6 + [VP] + [I64] * 3 + [VP, I64, I32, VP, I32, VP, F32] + [VP] * 3
    lib.kf_op_paged_attention_work.argtypes, lib.kf_op_paged_attention_work.restype = [I32] * 7, I64
    lib.kf_op_pages_grow.argtypes = [I32, VP, VP, VP, I32, VP, I32, I32, VP, I32, VP, VP]
    lib.kf_op_pages_compact.argtypes = [VP, I32, VP, I32, I32, VP, I32, I64, VP, VP, VP]
    lib.kf_op_pages_append.argtypes = [I32, VP, VP, I64, I32, I32, VP, I64, I64, VP, I64, I64, VP, I32, I32, VP, I32, I32, VP, VP]
    lib.kf_op_token_scores.argtypes = [I32, I64, I32, VP, I64, VP, F32, I32] + [VP] * 6
    lib.kf_op_token_scores_grad.argtypes = [I32, I64, I32, VP, I64, VP, F32] + [VP] * 6 + [I64, VP]
    lib.kf_last_error.argtypes, lib.kf_last_error.restype = [VP], ctypes.c_char_p
    return lib


@pytest.fixture(autouse=True)
def _fresh(lib):
    lib.fake_clear()


def refused(lib, name, rc):
    return rc == E_ARG and lib.kf_last_error(None).decode().startswith(name + ": ") and not launches(lib)


def prompt(lib, **kw):
    a = dict(type=1, n=3, T=300, longest=200, Hq=8, Hkv=2, hd=64, q=P, q_row=512, q_head=64, k=P, k_row=128, k_head=64, v=P, v_row=128,
             v_head=64, out=P, out_row=512, out_head=64, starts=P, scale=0.125, work=P, stream=None)
    a.update(kw)
    return lib.kf_op_prompt_attention(*a.values())


@pytest.mark.parametrize("bad", [dict(type=0), dict(type=3), dict(hd=96), dict(Hq=7), dict(Hkv=0), dict(n=-1), dict(T=-1), dict(T=1 << 31),
                                 dict(longest=-1), dict(longest=524289), dict(scale=0.0), dict(scale=float("nan")), dict(scale=float("inf")),
                                 dict(q=None), dict(q=P + 2), dict(k_row=130), dict(v_head=60), dict(out=P + 8), dict(starts=P + 1),
                                 dict(n=0), dict(out_row=-512), dict(n=200, work=None), dict(n=200, work=P + 16)])
def test_prompt_refusals(lib, bad):
    assert refused(lib, "kf_op_prompt_attention", prompt(lib, **bad))


def test_prompt_kernels(lib):
    # up to 128 sequences without a plan and without scratch
    assert lib.kf_op_prompt_attention_work(128, 1000) == 0 and prompt(lib, n=128, work=None) == OK
    assert [x.kernel.split("<")[0].split("::")[-1] for x in launches(lib)] == ["k_prompt"]
    need = lib.kf_op_prompt_attention_work(129, 1000)
    assert need >= 256 + 16 * (129 + 1000 // 128) and prompt(lib, n=129, T=1000) == OK
    got = launches(lib)
    assert len(got) == 2 and "k_plan" in got[0].kernel and not got[0].dependent and "k_prompt" in got[1].kernel and got[1].dependent
    assert prompt(lib, n=0, T=0) == OK and not launches(lib)


def paged(lib, **kw):
    a = dict(type=2, B=4, rows=1, Hq=8, Hkv=2, hd=128, q=P, q_seq=1024, q_row=1024, q_head=128, pool=P, n_pages=100, page=16, table=P,
             width=64, lens=P, scale=0.1, out=P, work=P, stream=None)
    a.update(kw)
    return lib.kf_op_paged_attention(*a.values())


@pytest.mark.parametrize("bad", [dict(type=0), dict(hd=32), dict(B=-1), dict(rows=0), dict(Hq=9), dict(page=8), dict(page=24), dict(page=8192),
                                 dict(width=-1), dict(width=1 << 30), dict(n_pages=-1), dict(scale=-1.0), dict(q=None), dict(lens=None),
                                 dict(table=None), dict(pool=None), dict(out=P + 4), dict(q_head=100), dict(work=None), dict(work=P + 64)])
def test_paged_refusals(lib, bad):
    assert refused(lib, "kf_op_paged_attention", paged(lib, **bad))


def test_paged_kernels(lib):
    def kernels(**kw):
        assert paged(lib, **kw) == OK
        return [x.kernel.split("k_")[1].split("(")[0] for x in launches(lib)]

    assert [x.split("<")[0] for x in kernels(width=2000)] == ["paged", "join"]
    # a few short sequences: a CTA per segment, no scratch
    assert lib.kf_op_paged_attention_work(4, 1, 8, 2, 128, 16, 16) == 0
    assert [x.split("<")[0] for x in kernels(width=16, work=None)] == ["paged"]
    assert lib.kf_op_paged_attention_work(4, 1, 8, 2, 128, 16, 17) > 0
    # 32 query rows a pass at head_dim 64 only
    assert kernels(hd=64, rows=4, Hq=16)[0].endswith("64, 2>") and kernels(hd=64)[0].endswith("64, 1>")
    assert kernels(rows=8)[0].endswith("128, 1>")
    # two tiles that take turns: an even number of them over a cache past the L2
    large = dict(width=4096, n_pages=20000)
    assert kernels(rows=8, **large)[0].endswith("128, 2>") and kernels(rows=16, **large)[0].endswith("128, 2>")
    assert kernels(rows=4, **large)[0].endswith("128, 1>") and kernels(rows=12, **large)[0].endswith("128, 1>")
    assert paged(lib, B=0) == OK and not launches(lib)


def grow(lib, **kw):
    a = dict(n=2, which=P, new=P, ref=P, n_pages=100, table=P, slots=5, width=7, lens=P, page=16, work=P, stream=None)
    a.update(kw)
    return lib.kf_op_pages_grow(*a.values())


@pytest.mark.parametrize("bad", [dict(n=-1), dict(n=6), dict(n_pages=0), dict(slots=0), dict(width=-1), dict(page=0), dict(width=1 << 30),
                                 dict(slots=1 << 20, width=1 << 12), dict(ref=None), dict(table=None), dict(work=None), dict(which=None),
                                 dict(lens=None), dict(which=P + 2), dict(work=P + 4)])
def test_book_refusals(lib, bad):
    assert refused(lib, "kf_op_pages_grow", grow(lib, **bad))


def test_book_teams(lib):
    """One CTA for a small book, a cluster for a large one; moves are a dependent launch."""
    assert grow(lib) == OK and launches(lib)[0].grid[0] == 1
    assert grow(lib, n_pages=1 << 20) == OK
    assert launches(lib)[0].grid[0] == 8
    for bytes_ in (8, 24, 0, 1 << 31):
        assert refused(lib, "kf_op_pages_compact", lib.kf_op_pages_compact(P, 100, P, 5, 7, P, 2, bytes_, None, P, None))
    assert lib.kf_op_pages_compact(P, 100, P, 5, 7, P, 2, 4096, None, P, None) == OK
    got = launches(lib)
    assert "k_compact" in got[0].kernel and "k_move" in got[1].kernel and got[1].dependent


def test_append_refusals(lib):
    def append(**kw):
        a = dict(n=2, which=P, starts=P, T=10, Hkv=2, hd=64, k=P, k_row=128, k_head=64, v=P, v_row=128, v_head=64, pool=P, n_pages=9, page=16,
                 table=P, slots=3, width=4, lens=P, stream=None)
        a.update(kw)
        return lib.kf_op_pages_append(*a.values())

    for bad in (dict(n=-1), dict(T=-1), dict(hd=12), dict(Hkv=0), dict(k=None), dict(k=P + 8), dict(k_row=100), dict(v_head=4), dict(page=0),
                dict(table=None), dict(lens=P + 2)):
        assert refused(lib, "kf_op_pages_append", append(**bad)), bad
    assert append(T=0) == OK and not launches(lib)
    assert append() == OK and len(launches(lib)) == 1


def scores(lib, with_grad=False, **kw):
    a = dict(type=1, R=5, V=50257, logits=P, stride=50257, tokens=P, tau=1.0)
    a.update(dict(g_logp=None, g_entropy=None, logp=P, entropy=P, lse=P, grad=P, grad_stride=50257, stream=None) if with_grad else
             dict(top=3, logp=P, entropy=P, lse=P, top_ids=P, top_logp=P, stream=None))
    a.update(kw)
    return (lib.kf_op_token_scores_grad if with_grad else lib.kf_op_token_scores)(*a.values())


@pytest.mark.parametrize("bad", [dict(type=3), dict(R=-1), dict(V=0), dict(V=600000), dict(stride=50256), dict(tau=0.0), dict(tau=-1.0),
                                 dict(tau=float("nan")), dict(tau=1e-45), dict(tau=float("inf")), dict(logits=None), dict(logits=P + 1),
                                 dict(tokens=None), dict(tokens=P + 4)])
def test_score_refusals(lib, bad):
    for grad in (False, True):
        assert refused(lib, "kf_op_token_scores_grad" if grad else "kf_op_token_scores", scores(lib, grad, **bad))


def test_more_score_refusals(lib):
    for bad in (dict(top=-1), dict(top=65), dict(top_ids=None), dict(V=2, top=3)):
        assert refused(lib, "kf_op_token_scores", scores(lib, **bad))
    for bad in (dict(grad=None), dict(grad=P + 1), dict(grad_stride=50256), dict(grad_stride=50264)):
        assert refused(lib, "kf_op_token_scores_grad", scores(lib, True, **bad))
    assert scores(lib, R=0) == OK and not launches(lib)


def test_score_kernels(lib):
    def shape(grad=False, **kw):
        assert scores(lib, grad, **kw) == OK
        got = launches(lib)
        assert len(got) == 1
        return got[0].threads, got[0].cluster

    assert shape(R=4096, V=1000, stride=1000)[0] == 64 and shape(R=64, V=1000, stride=1000)[0] == 256 and shape(R=4096)[0] == 256
    assert shape(R=1)[1] > 1 and shape(R=4096)[1] <= 1
    assert shape(True, R=4096, V=1000, stride=1000, grad_stride=1000)[0] == 64
    assert shape(True, R=64, V=1000, stride=1000, grad_stride=1000)[0] == 512
    assert shape(True, R=4096)[0] == 512 and shape(True, R=4096, type=0)[1] == 2      # 201 KB a row: two CTAs

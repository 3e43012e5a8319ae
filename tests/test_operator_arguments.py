"""Refusals of the calls around a product: the packed product with an activation and a residual, the paged cache, beam search.  All of them are
answered on the host, before anything is launched; the pointers here are never followed."""
import ctypes

import pytest

vp, ll = ctypes.c_void_p, ctypes.c_longlong
OK, INVALID, UNSUPPORTED, ALIGNMENT, WORKSPACE = 0, -1, -2, -3, -4
FAKE, ODD = 0x10000, 0x10004


@pytest.fixture(scope="module")
def lib():
    from paper_1802_00150_b200 import build
    lib = ctypes.CDLL(build.build())
    return lib


def call(function, good, **changed):
    """The call with `good` arguments, some changed by name; good is an ordered dict."""
    args = dict(good)
    assert set(changed) <= set(args)
    args.update(changed)
    function.argtypes = [vp if isinstance(good[n], vp) or good[n] is None else type(good[n]) if isinstance(good[n], (ctypes._SimpleCData, ctypes.Array)) else ctypes.c_int
                         for n in args]
    return function(*[a if not isinstance(a, str) else None for a in args.values()])


def pointer(at=FAKE):
    return vp(at)


PRODUCT = dict(Wcodes=pointer(), Walpha=pointer(), m=8, n=128, k_w=2, xcodes=pointer(), xbeta=pointer(), batch=0, k_a=2, bias=pointer(0),
               activation=1, residual=pointer(0), ldr=0, y=pointer(), ldy=8, stream=pointer(0))


@pytest.mark.parametrize("changed, status", [
    ({}, OK),                                                                   # no vectors: nothing to do
    ({"m": 0}, OK),
    ({"activation": 5}, OK),
    ({"activation": 6}, UNSUPPORTED),
    ({"activation": -1}, UNSUPPORTED),
    ({"residual": pointer(), "ldr": 7}, INVALID),
    ({"residual": pointer(), "ldr": 8}, OK),
    ({"residual": pointer(FAKE), "ldr": 9, "batch": 2}, INVALID),               # y with another stride
    ({"Wcodes": pointer(0)}, INVALID),
    ({"y": pointer(0)}, INVALID),
    ({"ldy": 7}, INVALID),
    ({"n": 0}, INVALID),
    ({"batch": -1}, INVALID),
    ({"k_w": 5}, UNSUPPORTED),
    ({"k_a": 0}, UNSUPPORTED),
    ({"xcodes": pointer(ODD)}, ALIGNMENT),
])
def test_product_with_activation(lib, changed, status):
    assert call(lib.amq_binary_gemm_act, PRODUCT, **changed) == status


VIEW = dict(pages=4, page_size=16, heads=2, d=64, k=4, table=pointer(), ld_table=3, max_pages=3, lengths=pointer())
CACHE = dict(cache_kcodes=pointer(), cache_kcoeffs=pointer(), cache_vcodes=pointer(), cache_vcoeffs=pointer())
APPEND = dict(kcodes=pointer(), kcoeffs=pointer(), vcodes=pointer(), vcoeffs=pointer(), **CACHE, **VIEW, batch=2, count=1, stream=pointer(0))

VIEW_REFUSALS = [
    ({"pages": -1}, INVALID), ({"page_size": 0}, INVALID), ({"heads": 0}, INVALID), ({"d": 0}, INVALID), ({"max_pages": -1}, INVALID),
    ({"ld_table": 2}, INVALID), ({"k": 0}, UNSUPPORTED), ({"k": 5}, UNSUPPORTED), ({"d": 129}, UNSUPPORTED),
    ({"max_pages": 1 << 16, "ld_table": 1 << 16, "page_size": 1 << 16}, UNSUPPORTED), ({"lengths": pointer(0)}, INVALID), ({"table": pointer(0)}, INVALID),
    ({"cache_kcodes": pointer(0)}, INVALID), ({"cache_vcoeffs": pointer(0)}, INVALID), ({"cache_kcodes": pointer(ODD)}, ALIGNMENT),
    ({"cache_vcodes": pointer(ODD)}, ALIGNMENT), ({"batch": -1}, INVALID), ({"batch": 0}, OK),
]


@pytest.mark.parametrize("changed, status", VIEW_REFUSALS + [
    ({"count": 0}, OK), ({"count": -1}, INVALID), ({"max_pages": 0}, OK), ({"kcodes": pointer(0)}, INVALID), ({"vcoeffs": pointer(0)}, INVALID),
    ({"kcodes": pointer(ODD)}, ALIGNMENT), ({"vcodes": pointer(ODD)}, ALIGNMENT), ({"batch": 1 << 20, "count": 1 << 20}, UNSUPPORTED),
])
def test_cache_append(lib, changed, status):
    assert call(lib.amq_cache_append, APPEND, **changed) == status


ATTENTION = dict(q=pointer(), q_batch=ll(256), q_token=ll(256), q_head=ll(64), **CACHE, **VIEW, batch=2, q_len=1, q_heads=4, scale=ctypes.c_float(0.1),
                 out=pointer(), workspace=pointer(), workspace_bytes=ctypes.c_size_t(1 << 40), stream=pointer(0))


@pytest.mark.parametrize("changed, status", VIEW_REFUSALS + [
    ({"q_len": 0}, OK), ({"q_len": -1}, INVALID), ({"q_heads": 3}, INVALID), ({"q_heads": 0}, INVALID), ({"q": pointer(0)}, INVALID),
    ({"out": pointer(0)}, INVALID), ({"batch": 1 << 20, "q_len": 1 << 12}, UNSUPPORTED),
])
def test_cache_attention(lib, changed, status):
    assert call(lib.amq_cache_attention, ATTENTION, **changed) == status


SELECT = dict(logits=pointer(), ld=100, vocab=100, scores=pointer(), finished=pointer(), eos=2, batch=2, beams=4, scores_out=pointer(),
              parents=pointer(), tokens=pointer(), finished_out=pointer(0), stream=pointer(0))


@pytest.mark.parametrize("changed, status", [
    ({"batch": 0}, OK), ({"batch": -1}, INVALID), ({"beams": 0}, INVALID), ({"beams": 33}, UNSUPPORTED), ({"vocab": 0}, INVALID), ({"ld": 99}, INVALID),
    ({"eos": 100}, INVALID), ({"eos": -2}, INVALID), ({"eos": -1}, INVALID), ({"logits": pointer(0)}, INVALID), ({"scores": pointer(0)}, INVALID),
    ({"scores_out": pointer(0)}, INVALID), ({"parents": pointer(0)}, INVALID), ({"tokens": pointer(0)}, INVALID),
    ({"vocab": 1 << 30, "ld": 1 << 30}, UNSUPPORTED), ({"batch": 1 << 29}, UNSUPPORTED),
])
def test_beam_select(lib, changed, status):
    assert call(lib.amq_beam_select, SELECT, **changed) == status


def reorder(lib, src=(FAKE, FAKE), dst=(FAKE, FAKE), row=(64, 64), from_=(64, 64), to=(64, 64), count=None, parents=FAKE, batch=1, beams=4):
    pointers = lambda v: (vp * len(v))(*v)  # noqa: E731
    sizes = lambda v: (ctypes.c_size_t * len(v))(*v)  # noqa: E731
    lib.amq_beam_reorder.argtypes = [vp] * 5 + [ctypes.c_int, vp, ctypes.c_int, ctypes.c_int, vp]
    return lib.amq_beam_reorder(pointers(src), pointers(dst), sizes(row), sizes(from_), sizes(to), len(src) if count is None else count, parents, batch, beams, None)


def test_beam_reorder(lib):
    assert reorder(lib, count=0) == OK
    assert reorder(lib) == INVALID                                  # one state twice, in place
    assert reorder(lib, dst=(2 * FAKE, 2 * FAKE)) == INVALID
    assert reorder(lib, dst=(2 * FAKE, FAKE)) == INVALID            # (the second is read by the first's threads)
    assert reorder(lib, dst=(FAKE, 2 * FAKE)) == INVALID
    assert reorder(lib, batch=0) == OK
    assert reorder(lib, row=(0, 0)) == OK
    assert reorder(lib, count=-1) == INVALID
    assert reorder(lib, batch=-1) == INVALID
    assert reorder(lib, beams=0) == INVALID
    assert reorder(lib, beams=33) == UNSUPPORTED
    assert reorder(lib, count=9) == UNSUPPORTED
    assert reorder(lib, parents=None) == INVALID
    assert reorder(lib, src=(FAKE, None)) == INVALID
    assert reorder(lib, from_=(64, 60)) == INVALID
    assert reorder(lib, to=(60, 64)) == INVALID
    assert reorder(lib, to=(128, 64)) == INVALID                    # in place at another stride
    assert reorder(lib, dst=(FAKE, FAKE + 0x1002)) == ALIGNMENT
    assert reorder(lib, row=(62, 64)) == ALIGNMENT
    lib.amq_beam_reorder.argtypes = [vp] * 5 + [ctypes.c_int, vp, ctypes.c_int, ctypes.c_int, vp]
    assert lib.amq_beam_reorder(None, None, None, None, None, 1, FAKE, 1, 4, None) == INVALID

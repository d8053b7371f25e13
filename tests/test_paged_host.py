"""Paged cache and residual verification: structure layouts and the refusals that need no device."""
import ctypes as C
import os
import re

import pytest

import paper_2604_17701_b200 as wisv
from paper_2604_17701_b200 import build, paged

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, ESHAPE, EALIGN = -1, -2, -3


@pytest.fixture(scope="module")
def lib():
    build.build()
    return paged._lib()


def test_struct_layouts_match_the_header():
    header = open(os.path.join(ROOT, "include", "wisv.h")).read()
    for struct, cls in (("wisv_cache_config", paged._CacheConfig), ("wisv_pages", paged._Pages),
                        ("wisv_layout", paged._Layout), ("wisv_append", paged._Append),
                        ("wisv_attend", paged._Attend), ("wisv_residual", paged._Residual)):
        body = re.search(r"typedef struct \{([^}]*)\} %s;" % struct, header).group(1)
        body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
        fields = []
        for decl in body.split(";"):
            kind = C.c_void_p if "*" in decl else C.c_int64 if "int64_t" in decl else \
                C.c_float if "float" in decl else C.c_int32
            decl = re.sub(r"\b(const|void|float|int32_t|int64_t)\b|\*", "", decl)
            fields += [(n.strip(), kind) for n in decl.split(",") if n.strip()]
        assert fields == list(cls._fields_), struct


def test_status_bits_and_limits_match_the_workloads():
    header = open(os.path.join(ROOT, "include", "wisv.h")).read()
    bits = dict(re.findall(r"#define (WISV_ST_[A-Z_]+)\s+(\d+)", header))
    assert len(set(bits.values())) == len(bits) and bits["WISV_ST_NO_PAGES"] == "32" and bits["WISV_ST_NO_MASS"] == "64"
    # 2^18 weights of at most 2^44 stay below 2^63
    assert int(re.search(r"#define WISV_STATIC_MAX_V\s+(\d+)", header).group(1)) * 2 ** 44 < 2 ** 63


GOOD = dict(n_heads=32, n_kv_heads=8, head_dim=128, page_size=16, n_pages=64, max_requests=4, max_blocks=32, dtype=1)


@pytest.mark.parametrize("change, code", [
    (dict(dtype=0), EINVAL), (dict(dtype=3), EINVAL), (dict(n_heads=30), ESHAPE), (dict(n_kv_heads=0), ESHAPE),
    (dict(n_heads=0), ESHAPE), (dict(n_heads=65, n_kv_heads=1), ESHAPE), (dict(head_dim=96), ESHAPE),
    (dict(page_size=8), ESHAPE), (dict(page_size=48), ESHAPE), (dict(page_size=512), ESHAPE), (dict(n_pages=0), ESHAPE),
    (dict(max_requests=0), ESHAPE), (dict(max_requests=4097), ESHAPE), (dict(max_blocks=0), ESHAPE),
    (dict(max_blocks=1 << 28), ESHAPE), (dict(n_pages=1 << 28), ESHAPE)])
def test_cache_create_refuses(lib, change, code):
    h = C.c_void_p(1)
    cfg = paged._CacheConfig(**{**GOOD, **change})
    assert lib.wisv_cache_create(C.byref(cfg), C.byref(h)) == code
    assert h.value is None


def test_null_arguments(lib):
    h = C.c_void_p()
    assert lib.wisv_cache_create(None, C.byref(h)) == EINVAL
    assert lib.wisv_cache_create(C.byref(paged._CacheConfig(**GOOD)), None) == EINVAL
    assert lib.wisv_cache_destroy(None) == EINVAL
    assert lib.wisv_cache_extend(None, None, 1, 1, None, 1, None, None) == EINVAL
    assert lib.wisv_cache_commit(None, None, 1, None, None, None) == EINVAL
    assert lib.wisv_cache_append(None, None, None) == EINVAL
    assert lib.wisv_cache_attend(None, None, None) == EINVAL
    assert lib.wisv_cache_error(None, None, None) == EINVAL
    assert lib.wisv_verify_residual(None, None) == EINVAL
    assert lib.wisv_cache_launch_count(None) == 0


def _residual(**kw):
    base = dict(B=2, K=4, k_off=None, T_total=8, V=1000, target_probs=4096, target_stride=1000, target_dtype=0,
                draft_tokens=4096, draft_probs=4096, draft_stride=1000, draft_dtype=0, draft_ids=None, n_top=0,
                uniforms=4096, u_draw=4096, accept_in=None, accept_len=4096, token=4096, mass=None, status=None)
    return paged._Residual(**{**base, **kw})


@pytest.mark.parametrize("change, code", [
    (dict(target_probs=None), EINVAL), (dict(u_draw=None), EINVAL), (dict(accept_len=None), EINVAL), (dict(token=None), EINVAL),
    (dict(target_dtype=3), EINVAL), (dict(draft_dtype=7), EINVAL), (dict(uniforms=None), EINVAL),
    (dict(draft_tokens=None), EINVAL), (dict(draft_probs=None, draft_ids=4096, n_top=4), EINVAL),
    (dict(B=0), ESHAPE), (dict(V=0), ESHAPE), (dict(V=262145, target_stride=262145), ESHAPE), (dict(target_stride=999), ESHAPE),
    (dict(draft_stride=999), ESHAPE), (dict(K=65, T_total=130), ESHAPE), (dict(T_total=7), ESHAPE), (dict(T_total=-1), ESHAPE),
    (dict(draft_ids=4096, n_top=0), ESHAPE), (dict(draft_ids=4096, n_top=257), ESHAPE),
    (dict(target_probs=4098), EALIGN), (dict(draft_probs=4097, draft_dtype=1), EALIGN)])
def test_verify_residual_refuses(lib, change, code):
    assert lib.wisv_verify_residual(C.byref(_residual(**change)), None) == code


def test_binding_needs_a_cuda_device():
    with pytest.raises(ValueError):
        wisv.PagedCache(**{**GOOD, "device": "cpu"})


@pytest.mark.parametrize("i, name", list(enumerate(n for n, _ in paged._Pages._fields_)))
def test_bookkeeping_arrays_cannot_be_replaced(i, name):
    """The library holds their addresses: another tensor in the attribute would give the calls different tables."""
    cache = object.__new__(wisv.PagedCache)
    cache._owned = tuple(range(5))
    assert getattr(cache, name) == i                               # the order of the block of addresses
    setattr(cache, name, cache._owned[i])                          # as `+=` does after its work in place
    with pytest.raises(AttributeError):
        setattr(cache, name, None)

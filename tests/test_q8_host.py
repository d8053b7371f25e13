"""The 8-bit paged cache: structure layouts and the refusals that need no device."""
import ctypes as C
import os
import re

import pytest
import torch

import paper_2604_17701_b200 as wisv
from paper_2604_17701_b200 import build, paged

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL = -1


def test_struct_layouts_match_the_header():
    header = open(os.path.join(ROOT, "include", "wisv.h")).read()
    for struct, cls in (("wisv_q8_pages", paged._Q8Pages), ("wisv_q8_append", paged._Q8Append), ("wisv_q8_read", paged._Q8Read),
                        ("wisv_q8_attend", paged._Q8Attend)):
        body = re.search(r"typedef struct \{([^}]*)\} %s;" % struct, header).group(1)
        body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
        fields = []
        for decl in body.split(";"):
            kind = C.c_void_p if "*" in decl else C.c_int64 if "int64_t" in decl else C.c_float if "float" in decl else C.c_int32
            decl = re.sub(r"\b(const|void|float|int32_t|int64_t)\b|\*", "", decl)
            fields += [(n.strip(), kind) for n in decl.split(",") if n.strip()]
        assert fields == list(cls._fields_), struct


def test_null_arguments():
    build.build()
    lib = paged._lib()
    for name in ("wisv_cache_append_q8", "wisv_cache_read_q8", "wisv_cache_attend_q8"):
        assert getattr(lib, name)(None, None, None, None) == EINVAL


def test_pools_live_on_a_cuda_device():
    codes = torch.zeros((3, 16, 2, 64), dtype=torch.uint8).view(torch.float8_e4m3fn)
    scales = torch.zeros((3, 2, 16)).transpose(1, 2)
    with pytest.raises(ValueError):
        wisv.QuantPages(codes, codes, scales, scales)

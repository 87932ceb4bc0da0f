"""Host-only checks of pages of 4 bits: what the calls refuse, and the plain form that the GPU tests compare with."""
import numpy as np
import pytest
import torch

import pages_plain as P
from test_pages_cpu import calls, good, held, lib  # noqa: F401


def test_shapes(lib):  # noqa: F811
    four = lib.LRQK_PAGE_E2M1
    for kw in (dict(), dict(kv_dtype=1), dict(page=1, max_pages=1000), dict(n_pages=1 << 24)):
        assert lib.lrqk_validate_pages(good(lib, page_dtype=four, **kw)) == 0, kw
        assert lib.lrqk_pages_workspace_bytes(good(lib, page_dtype=four, **kw)) > 0, kw
    assert lib.lrqk_validate_pages(good(lib, page_dtype=four, n_pages=(1 << 24) + 1)) == -2     # 64 GiB of rows
    for t in (5, 6, 7, 9, 16):
        assert lib.lrqk_validate_pages(good(lib, page_dtype=t)) == -1


def test_header(lib):  # noqa: F811
    import os
    import re
    text = open(os.path.join(os.path.dirname(lib.__file__), "..", "include", "lrqk.h")).read()
    assert int(re.search(r"LRQK_PAGE_E2M1 = (\d)", text).group(1)) == lib.LRQK_PAGE_E2M1


def test_scales_are_needed(lib):  # noqa: F811
    import ctypes as C
    A, raw = 0x10000, lib.load_library()
    s, no_scale = good(lib, page_dtype=lib.LRQK_PAGE_E2M1), lib.Pages(0x10000, 0x10000, None, None, A, A, A)
    assert raw.lrqk_pages_append(C.byref(s), C.byref(no_scale), A, A, None) == -1
    assert raw.lrqk_chunk_attend(C.byref(s), C.byref(no_scale), A, A, A, 1 << 40, None) == -1
    assert raw.lrqk_pages_read(C.byref(s), C.byref(no_scale), 0, A, A, None) == -1


def test_pools(lib, monkeypatch):  # noqa: F811
    """Rows of 64 bytes, as uint8 or float4_e2m1fn_x2; shorter pools, scales and other types are errors."""
    s, u8 = good(lib, page_dtype=lib.LRQK_PAGE_E2M1), torch.uint8
    pool = lambda n=64, t=u8: dict(K=torch.zeros(200, 4, 16, n, dtype=t), V=torch.zeros(200, 4, 16, n, dtype=t))  # noqa: E731
    for kw in (pool(), dict(K=pool()["K"].view(torch.float4_e2m1fn_x2), V=pool()["V"].view(torch.float4_e2m1fn_x2)), pool(128)):
        for f in list(calls(lib, s, held(lib, monkeypatch, **kw)))[:2]:
            with pytest.raises(lib.LrqkError):
                f()
    for kw in (pool(63), dict(pool(), V=torch.zeros(199, 4, 16, 64, dtype=u8)), dict(pool(), K_scale=torch.zeros(200, 4, 16, 3, dtype=u8))):
        for f in calls(lib, s, held(lib, monkeypatch, **kw)):
            with pytest.raises(ValueError):
                f()
    for t in (torch.int8, torch.bfloat16, torch.float32):
        for f in calls(lib, s, held(lib, monkeypatch, **pool(128, t))):
            with pytest.raises(TypeError):
                f()
    four = dict(K=pool()["K"].view(torch.float4_e2m1fn_x2), V=pool()["V"].view(torch.float4_e2m1fn_x2))
    for t in (2, 3):                         # 8-bit rows
        for f in calls(lib, good(lib, page_dtype=t), held(lib, monkeypatch, **four)):
            with pytest.raises(TypeError):
                f()


def test_plain_form():
    """Codes, ties and scales by hand."""
    x = np.zeros((1, 128))
    x[0, :14] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.26, -0.74, 0.3, 6.0, -6.0, 5.1, 4.9]
    x[0, 32] = 6.5                           # 6.5 > 6: steps of 1
    x[0, 64] = 2.0 ** -120                   # the smallest scale
    code, byte = P.quantise(x, "e2m1")
    assert byte.tolist() == [[127, 128, 17, 17]]
    v = P.values(code, byte, "e2m1")[0]
    assert v[:14].tolist() == [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, -0.5, -0.5, 0.5, 6.0, -6.0, 6.0, 4.0]
    assert v[32] == 6.0 and v[64] == 0.0     # 3.25 of 2 -> 3 of 2; 2^-10 of 2^-110 -> 0
    assert code[0, 0] == 0x20 and code[0, 1] == 0x42
    x[0, 5] = np.nan
    code, byte = P.quantise(x, "e2m1")
    assert byte[0, 0] == 255 and np.isnan(P.values(code, byte, "e2m1")[0, :32]).all()

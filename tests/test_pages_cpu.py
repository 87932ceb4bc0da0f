"""Host-only checks of the paged cache's entry points: what they refuse, before any device work."""
import ctypes as C

import pytest
import torch


@pytest.fixture(scope="module")
def lib():
    import paper_2510_23649_amd as L
    from paper_2510_23649_amd import build as B
    if not B.is_built():
        B.build(verbose=False)
    return L


def good(lib, **kw):
    base = dict(B=2, Hq=28, Hkv=4, T=7, n_max=4, l_max=1000, page=16, n_pages=200, max_pages=63)
    base.update(kw)
    return lib.PagesShape.make(**base)


def test_shape_limits(lib):
    assert lib.lrqk_validate_pages(good(lib)) == 0
    for kw in (dict(page=1, max_pages=1000), dict(page=1024, max_pages=1), dict(l_cap=1000), dict(l_cap=2000),
               dict(Hq=32, Hkv=4), dict(page_dtype=2), dict(page_dtype=3), dict(kv_dtype=1, page_dtype=1),
               dict(kv_dtype=1, page_dtype=2), dict(scale=-1.0), dict(scale=0.0), dict(l_max=1), dict(n_max=100000),
               dict(n_pages=1 << 22), dict(n_pages=1 << 23, page_dtype=2)):
        assert lib.lrqk_validate_pages(good(lib, **kw)) == 0, kw
        assert lib.lrqk_pages_workspace_bytes(good(lib, **kw)) > 0, kw
    for kw in (dict(B=0), dict(Hq=30), dict(Hq=36), dict(Hkv=0), dict(d=64), dict(T=0), dict(T=1 << 24), dict(n_max=0),
               dict(l_max=0), dict(l_max=1 << 24), dict(max_pages=62), dict(page=0), dict(page=24), dict(page=2048),
               dict(page=-16), dict(n_pages=0), dict(l_cap=999), dict(l_cap=-1), dict(l_cap=1 << 24), dict(B=3000),
               dict(n_pages=(1 << 22) + 1), dict(n_pages=(1 << 23) + 1, page_dtype=2), dict(n_pages=(1 << 31) - 1),
               dict(scale=float("nan")), dict(scale=float("inf")), dict(T=(1 << 24) - 1, Hq=256, Hkv=32)):
        assert lib.lrqk_validate_pages(good(lib, **kw)) == -2, kw
        assert lib.lrqk_pages_workspace_bytes(good(lib, **kw)) == 0, kw
    for kw in (dict(kv_dtype=2), dict(kv_dtype=-1), dict(page_dtype=4), dict(page_dtype=-1),
               dict(kv_dtype=0, page_dtype=1), dict(kv_dtype=1, page_dtype=0)):
        assert lib.lrqk_validate_pages(good(lib, **kw)) == -1, kw
    assert lib.load_library().lrqk_validate_pages(None) == -1


def test_pointers_and_workspace(lib):
    raw, A = lib.load_library(), 0x10000     # an aligned fake address, never dereferenced here
    s, s8, bad = good(lib), good(lib, page_dtype=2), good(lib, page=24)
    full = lib.Pages(*([A] * 7))
    no_scale = lib.Pages(A, A, None, None, A, A, A)
    for fn, tail in ((raw.lrqk_pages_append, (A, A, None)), (raw.lrqk_pages_read, (0, A, A, None)),
                     (raw.lrqk_chunk_attend, (A, A, A, 1 << 40, None))):
        assert fn(None, C.byref(full), *tail) == -1
        assert fn(C.byref(bad), C.byref(full), *tail) == -2
        assert fn(C.byref(s), None, *tail) == -1
        assert fn(C.byref(s8), C.byref(no_scale), *tail) == -1
        for i in (0, 1, 4, 5, 6):
            for v in (None, A + 4):
                f = [A] * 7
                f[i] = v
                assert fn(C.byref(s), C.byref(lib.Pages(*f)), *tail) == -1, (fn, i)
        f = [A] * 7
        f[3] = A + 8
        assert fn(C.byref(s8), C.byref(lib.Pages(*f)), *tail) == -1
    p = C.byref(full)
    for args in ((None, A, None), (A, None, None), (A + 2, A, None), (A, A + 8, None)):
        assert raw.lrqk_pages_append(C.byref(s), p, *args) == -1
    for args in ((-1, A, A, None), (0, None, None, None), (0, A + 4, A, None), (0, A, A + 8, None)):
        assert raw.lrqk_pages_read(C.byref(s), p, *args) == -1
    assert raw.lrqk_pages_read(C.byref(s), p, 1000, A, A, None) == 0        # no such position: nothing to do
    big = 1 << 40
    for args in ((None, A, A, big), (A, None, A, big), (A, A, None, big), (A + 4, A, A, big), (A, A + 4, A, big),
                 (A, A, A + 16, big)):
        assert raw.lrqk_chunk_attend(C.byref(s), p, *args, None) == -1
    assert raw.lrqk_chunk_attend(C.byref(s), p, A, A, A, lib.lrqk_pages_workspace_bytes(s) - 1, None) == -4


def test_binding_matches_the_header(lib):
    import os
    import re
    text = open(os.path.join(os.path.dirname(lib.__file__), "..", "include", "lrqk.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = lambda n: [x for d in re.search(r"typedef struct %s \{(.*?)\} %s;" % (n, n), text, re.S).group(1).split(";")  # noqa: E731
                       for x in re.findall(r"(\w+)\s*(?:,|$)", d.strip())]
    assert names("lrqk_pages_shape") == [n for n, _ in lib.PagesShape._fields_]
    assert names("lrqk_pages") == [n for n, _ in lib.Pages._fields_]
    for n in ("BF16", "F32", "E4M3", "I8"):
        assert int(re.search(r"LRQK_PAGE_%s = (\d)" % n, text).group(1)) == getattr(lib, "LRQK_PAGE_" + n)


def test_binding_refuses_what_is_no_device_tensor(lib):
    """Wrong types, strides, sizes and places are Python errors, not reads of other memory."""
    x = torch.zeros(4, 2, 16, 128, dtype=torch.bfloat16)
    i = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        lib.make_pages(K=x, V=x, table=i, start=i, kv_len=i)                 # host memory
    with pytest.raises(TypeError):
        lib.make_pages(K=x, V=x.float(), table=i, start=i, kv_len=i)
    with pytest.raises(TypeError):
        lib.make_pages(K=x.half(), V=x.half(), table=i, start=i, kv_len=i)
    s, p = good(lib), lib.Pages(*([0x10000] * 7))
    rows = torch.zeros(7, 28, 128, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        lib.lrqk_pages_append(s, p, rows.float(), rows, stream=0)
    with pytest.raises(ValueError):
        lib.lrqk_pages_append(s, p, rows[:0], rows, stream=0)
    with pytest.raises(ValueError):
        lib.lrqk_chunk_attend(s, p, rows[:6], rows, rows, stream=0)
    with pytest.raises(ValueError):
        lib.lrqk_chunk_attend(s, p, rows, rows, rows, stream=0)              # host memory
    with pytest.raises(ValueError):
        lib.lrqk_pages_read(s, p, 0, torch.zeros(2, 4, 1000, 128, dtype=torch.bfloat16), None, stream=0)  # not pinned


def held(lib, monkeypatch, **kw):
    """Pages whose tensors fit good(lib, page_dtype=2), but for what is given; in host memory, taken for a device's."""
    from paper_2510_23649_amd import binding
    t = dict(K=torch.zeros(200, 4, 16, 128, dtype=torch.uint8), V=torch.zeros(200, 4, 16, 128, dtype=torch.uint8),
             K_scale=torch.zeros(200, 4, 16, 4, dtype=torch.uint8), V_scale=torch.zeros(200, 4, 16, 4, dtype=torch.uint8),
             table=torch.zeros(2, 63, dtype=torch.int32), start=torch.zeros(3, dtype=torch.int32),
             kv_len=torch.zeros(2, dtype=torch.int32))
    t.update(kw)
    monkeypatch.setattr(binding, "_dev", lambda x, dtype=None: None if x is None else 0x10000)
    monkeypatch.setattr(binding, "_raw_stream", lambda *a: 0)
    return lib.make_pages(**t)


def calls(lib, s, p):
    """Every call on pages p, as it begins: what it would pass on to the library is not there."""
    for f in (lambda: lib.lrqk_pages_append(s, p, None, None), lambda: lib.lrqk_pages_read(s, p, 0, None, None),
              lambda: lib.lrqk_chunk_attend(s, p, None, torch.zeros(1), torch.zeros(1))):
        yield f


def test_pages_that_do_not_hold_the_shape(lib, monkeypatch):
    """Pools, scales and tables of other types and sizes than the shape says: errors, and nothing launched."""
    u8, i32 = torch.uint8, torch.int32
    short = {"K": torch.zeros(199, 4, 16, 128, dtype=u8), "V": torch.zeros(200, 4, 16, 127, dtype=u8),
             "K_scale": torch.zeros(200, 4, 16, 3, dtype=u8), "V_scale": torch.zeros(0, dtype=u8),
             "table": torch.zeros(1, 125, dtype=i32), "start": torch.zeros(2, dtype=i32), "kv_len": torch.zeros(1, dtype=i32)}
    s = good(lib, page_dtype=2)
    for name, t in short.items():
        for f in calls(lib, s, held(lib, monkeypatch, **{name: t})):
            with pytest.raises(ValueError, match=name):
                f()
    p = held(lib, monkeypatch)
    for kw in (dict(n_pages=201), dict(B=3), dict(max_pages=64), dict(max_pages=200, page=8), dict(Hkv=8, Hq=32), dict(page=32)):
        for f in calls(lib, good(lib, **{"page_dtype": 2, **kw}), p):
            with pytest.raises(ValueError):
                f()
    # the table's rows lie max_pages entries apart
    wide = held(lib, monkeypatch, table=torch.zeros(2, 70, dtype=i32))
    for f in calls(lib, s, wide):
        with pytest.raises(ValueError, match="table"):
            f()


def test_pages_of_another_type_than_the_shape_says(lib, monkeypatch):
    pool = lambda t: dict(K=torch.zeros(200, 4, 16, 128, dtype=t), V=torch.zeros(200, 4, 16, 128, dtype=t))  # noqa: E731
    for t, kw in ((torch.float32, dict(page_dtype=0)), (torch.bfloat16, dict(kv_dtype=1, page_dtype=1)),
                  (torch.bfloat16, dict(page_dtype=2)), (torch.float32, dict(kv_dtype=1, page_dtype=3)),
                  (torch.uint8, dict(page_dtype=0)), (torch.uint8, dict(kv_dtype=1, page_dtype=1))):
        for f in calls(lib, good(lib, **kw), held(lib, monkeypatch, **pool(t))):
            with pytest.raises(TypeError):
                f()


def test_pages_that_hold_the_shape(lib, monkeypatch):
    """What fits goes on to the library, which refuses the pointers that are not there; a bad shape is its to refuse."""
    u8 = torch.uint8
    fits = [(good(lib, page_dtype=2), {}), (good(lib, page_dtype=3), {}), (good(lib, n_pages=100, page_dtype=2), {}),
            (good(lib, B=1, page_dtype=2), {}), (good(lib, B=1, max_pages=126, page_dtype=2), {}),
            (good(lib, page_dtype=2), dict(K=torch.zeros(200, 4, 16, 128, dtype=torch.int8), V=torch.zeros(200, 4, 16, 128, dtype=torch.int8))),
            (good(lib, page_dtype=2), dict(K=torch.zeros(200, 4, 16, 128).to(torch.float8_e4m3fn), V=torch.zeros(200, 4, 16, 128).to(torch.float8_e4m3fn))),
            (good(lib, page_dtype=2), dict(table=torch.zeros(126, dtype=torch.int32))),
            (good(lib, page_dtype=2), dict(K=torch.zeros(200 * 4 * 16 * 128, dtype=u8))),
            (good(lib), dict(K=torch.zeros(200, 4, 16, 128, dtype=torch.bfloat16), V=torch.zeros(200, 4, 16, 128, dtype=torch.bfloat16), K_scale=None, V_scale=None)),
            (good(lib, page_dtype=2), dict(K_scale=None, V_scale=None))]
    for s, kw in fits:
        p = held(lib, monkeypatch, **kw)
        for _ in range(2):                   # found, and found again
            for f in list(calls(lib, s, p))[:2]:
                with pytest.raises(lib.LrqkError) as e:
                    f()
                assert e.value.status == -1
    p = held(lib, monkeypatch)
    for f in list(calls(lib, good(lib, page=24, n_pages=1 << 20, page_dtype=2), p))[:2]:
        with pytest.raises(lib.LrqkError) as e:
            f()
        assert e.value.status == -2
    # another shape after one that fits
    lib_s, bad = good(lib, page_dtype=2), good(lib, page_dtype=2, n_pages=300)
    for s, err in ((lib_s, lib.LrqkError), (bad, ValueError), (lib_s, lib.LrqkError)):
        with pytest.raises(err):
            lib.lrqk_pages_append(s, p, None, None)


def test_what_was_found_to_fit_is_found_again(lib, monkeypatch):
    """Another number of tokens or another length means the same pages; each of what says how much they hold does not."""
    from paper_2510_23649_amd import binding
    p, s = held(lib, monkeypatch), good(lib, page_dtype=2)
    binding._hold(p, s)
    looked = []
    monkeypatch.setattr(binding, "lrqk_validate_pages", lambda x: looked.append(1) or -1)
    for kw in ({}, dict(T=100, n_max=90), dict(l_max=700, l_cap=800), dict(Hq=8, scale=2.0)):
        binding._hold(p, good(lib, page_dtype=2, **kw))
    assert not looked
    for kw in (dict(B=1), dict(Hkv=2), dict(d=64), dict(page=8), dict(n_pages=100), dict(max_pages=64), dict(page_dtype=3)):
        binding._hold(p, good(lib, **{"page_dtype": 2, **kw}))
        assert looked.pop()

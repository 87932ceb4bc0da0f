"""Host-only checks of rotary positions and of the tables made on the device: the table of a rope, and what the calls refuse."""
import ctypes as C
import os
import re

import numpy as np
import pytest
import torch

import tables_plain as X
from test_pages_cpu import good, held, lib  # noqa: F401

A = 0x10000                                  # an aligned fake address, never dereferenced here


def test_structures_and_constants_match_the_header(lib):  # noqa: F811
    text = open(os.path.join(os.path.dirname(lib.__file__), "..", "include", "lrqk.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = lambda n: [x for d in re.search(r"typedef struct %s \{(.*?)\} %s;" % (n, n), text, re.S).group(1).split(";")  # noqa: E731
                       for x in re.findall(r"(\w+)\s*(?:,|$)", d.strip())]
    from paper_2510_23649_amd import binding
    for c, py in (("lrqk_rope", lib.Rope), ("lrqk_rotate_shape", binding.RotateShape), ("lrqk_new_rows", binding.NewRows),
                  ("lrqk_pages_tables", lib.PagesTables)):
        assert names(c) == [n for n, _ in py._fields_], c
    for n in ("ROPE_HALVES", "ROPE_PAIRS", "ROPE_PLAIN", "ROPE_LINEAR", "ROPE_BASE", "ROPE_BANDS", "ROPE_RAMP", "ADVANCE_OK",
              "ADVANCE_LONG", "ADVANCE_SHARED", "ADVANCE_PAGES", "ADVANCE_ROWS"):
        assert int(re.search(r"LRQK_%s = (\d)" % n, text).group(1)) == getattr(lib, "LRQK_" + n)


@pytest.mark.parametrize("scaling", range(5))
def test_turns(lib, scaling):  # noqa: F811
    """Against float64: a frequency is off by 2^-50 of itself there, and by 2^-65 turns here."""
    for rot in (2, 4, 20, 64, 96, 128):
        for kw in (dict(base=10000.0, factor=8.0, low=1.0, high=4.0, l_orig=8192), dict(base=500000.0, factor=40.0, low=1.0, high=32.0, l_orig=4096),
                   dict(base=1.5, factor=0.5, low=0.25, high=1.0, l_orig=1), dict(base=1e6, factor=1.0, low=2.0, high=3.0, l_orig=1 << 20)):
            turns, amplitude = lib.lrqk_rope_turns(rot, scaling, **kw)
            f, a = X.frequencies(rot, scaling, **kw)
            got = np.array([(int(x) & (1 << 64) - 1) / 2.0 ** 64 for x in turns])
            assert len(got) == rot // 2 and abs(amplitude - a) <= 2.0 ** -23 * a
            assert (np.abs(got - f / (2 * np.pi)) <= 2.0 ** -48 * f + 2.0 ** -64).all()


def test_turns_refused(lib):  # noqa: F811
    raw, buf, a = lib.load_library(), (C.c_uint64 * 64)(), C.c_float()
    call = lambda rot=64, kind=3, base=1e4, factor=2.0, low=1.0, high=4.0, l=100, out=buf: raw.lrqk_rope_turns(rot, kind, base, factor, low, high, l, out, C.byref(a))  # noqa: E731,E741
    nan, inf = float("nan"), float("inf")
    assert call() == 0 and raw.lrqk_rope_turns(64, 0, 1e4, nan, nan, nan, -1, buf, None) == 0
    for kw in (dict(rot=0), dict(rot=3), dict(rot=130), dict(rot=-2)):
        assert call(**kw) == -2, kw
    for kw in (dict(out=None), dict(kind=-1), dict(kind=5), dict(base=1.0), dict(base=nan), dict(base=inf), dict(base=-3.0), dict(factor=0.0),
               dict(factor=nan), dict(factor=inf), dict(low=0.0), dict(low=4.0), dict(low=nan), dict(high=nan), dict(high=inf), dict(l=0)):
        assert call(**kw) == -1, kw
    with pytest.raises(lib.LrqkError):
        lib.lrqk_rope_turns(7, base=1e4)
    with pytest.raises(lib.LrqkError):
        lib.lrqk_rope_turns(0, base=1e4)


def test_rotate_refused(lib):  # noqa: F811
    from paper_2510_23649_amd.binding import RotateShape
    raw = lib.load_library()

    def call(rope=None, q=A, q_out=2 * A, k=3 * A, k_out=4 * A, pos=A, **kw):
        s = RotateShape(**dict(dict(T=4, Hq=8, Hkv=2, d=128, q_type=0, q_out_type=1, k_type=0), **kw))
        r = dict(dict(layout=0, rot=128, back=0, amplitude=1.0, turns=A), **(rope or {}))
        return raw.lrqk_rotate(C.byref(s), C.byref(lib.Rope(**r)), pos, q, q_out, k, k_out, None)

    for rope in (dict(rot=0), dict(rot=5), dict(rot=130), dict(amplitude=float("nan")), dict(amplitude=float("inf"))):
        assert call(rope) == -2, rope
    for rope in (dict(turns=None), dict(turns=A + 8), dict(layout=2), dict(layout=-1), dict(back=2), dict(back=-1)):
        assert call(rope) == -1, rope
    for kw in (dict(T=0), dict(T=1 << 24), dict(d=64), dict(Hq=0), dict(Hkv=1025), dict(Hq=-1), dict(q_stride=1023), dict(q_stride=1028),
               dict(q_out_stride=1026), dict(k_stride=255), dict(k_out_stride=260), dict(k_stride=-256)):
        assert call(**kw) == -2, kw
    for kw in (dict(pos=None), dict(pos=A + 4), dict(q=None), dict(q_out=None), dict(k=None), dict(k_out=None), dict(q=A + 8), dict(k_out=A + 2),
               dict(q_type=2), dict(q_out_type=-1), dict(k_type=3), dict(q=None, q_out=None, k=None, k_out=None),
               dict(q_out=A), dict(q_out=A, q_out_type=0, q_stride=2048), dict(k_out=3 * A, k_out_stride=512)):
        assert call(**kw) == -1, kw
    s = RotateShape(T=4, Hq=8, Hkv=2, d=128)
    r = lib.Rope(0, 128, 0, 1.0, A)
    assert raw.lrqk_rotate(None, C.byref(r), A, A, 2 * A, None, None, None) == -1
    assert raw.lrqk_rotate(C.byref(s), None, A, A, 2 * A, None, None, None) == -1


def test_rotate_append_refused(lib):  # noqa: F811
    from paper_2510_23649_amd.binding import NewRows
    raw, s = lib.load_library(), good(lib)
    full, rope = lib.Pages(*([A] * 7)), lib.Rope(0, 128, 0, 1.0, A)

    def call(shape=s, pages=full, rope=rope, **kw):
        n = NewRows(**dict(dict(q=A, k=2 * A, v=3 * A, q_out=4 * A), **kw))
        return raw.lrqk_pages_rotate_append(C.byref(shape), C.byref(pages), C.byref(rope), C.byref(n), None)

    assert call(shape=good(lib, page=24)) == -2 and call(rope=lib.Rope(0, 7, 0, 1.0, A)) == -2 and call(rope=lib.Rope(3, 8, 0, 1.0, A)) == -1
    for kw in (dict(k=None), dict(v=None), dict(q=None), dict(q_out=None), dict(k=A + 8), dict(v=A + 4), dict(q=A + 4), dict(q_out=A + 2),
               dict(pos=A), dict(slot=A), dict(pos=A, slot=A + 4), dict(pos=A + 8, slot=A), dict(q_out=A, q_stride=28 * 128 + 8)):
        assert call(**kw) == -1, kw
    for kw in (dict(q_stride=28 * 128 - 8), dict(k_stride=4 * 128 + 4), dict(v_stride=-512)):
        assert call(**kw) == -2, kw
    for i in (0, 1, 4, 5, 6):
        for x in (None, A + 4):
            f = [A] * 7
            f[i] = x
            assert call(pages=lib.Pages(*f)) == -1
            if i < 2:                        # with positions and slots given, the tables are not looked at
                assert call(pages=lib.Pages(*f), pos=A, slot=A) == -1
    n = NewRows(q=A, k=A, v=A, q_out=2 * A)
    assert raw.lrqk_pages_rotate_append(None, C.byref(full), C.byref(rope), C.byref(n), None) == -1
    assert raw.lrqk_pages_rotate_append(C.byref(s), None, C.byref(rope), C.byref(n), None) == -1
    assert raw.lrqk_pages_rotate_append(C.byref(s), C.byref(full), None, C.byref(n), None) == -1
    assert raw.lrqk_pages_rotate_append(C.byref(s), C.byref(full), C.byref(rope), None, None) == -1


def test_advance_refused(lib):  # noqa: F811
    raw, s = lib.load_library(), good(lib)
    big = 1 << 40
    names = [n for n, _ in lib.PagesTables._fields_]
    call = lambda t, keep=A, n=A, ws=A, size=big, shape=s: raw.lrqk_pages_advance(C.byref(shape), C.byref(t), keep, n, ws, size, None)  # noqa: E731
    for i, name in enumerate(names):
        for x in (None, A + 4):
            if x is None and name in ("seq", "pos", "slot"):
                continue
            f = [A] * 8
            f[i] = x
            assert call(lib.PagesTables(*f)) == -1, name
            if name in ("refs", "table", "kv_len"):
                assert raw.lrqk_pages_tables_init(C.byref(s), C.byref(lib.PagesTables(*f)), None) == -1
    t = lib.PagesTables(*([A] * 8))
    for kw in (dict(keep=A + 4), dict(n=None), dict(n=A + 8), dict(ws=None), dict(ws=A + 16)):
        assert call(t, **kw) == -1, kw
    assert call(t, size=lib.lrqk_pages_advance_workspace_bytes(s) - 1) == -4
    assert call(t, shape=good(lib, page=24)) == -2 and lib.lrqk_pages_advance_workspace_bytes(good(lib, page=24)) == 0
    assert lib.lrqk_pages_advance_workspace_bytes(good(lib, B=2340)) >= 4 * 4 * 2341
    assert raw.lrqk_pages_advance(C.byref(s), None, A, A, A, big, None) == -1
    assert raw.lrqk_pages_advance(None, C.byref(t), A, A, A, big, None) == -1
    assert raw.lrqk_pages_tables_init(C.byref(s), None, None) == -1 and raw.lrqk_pages_tables_init(None, C.byref(t), None) == -1


def test_binding_refuses(lib, monkeypatch):  # noqa: F811
    """Wrong types, sizes and strides are Python errors, not reads of other memory."""
    from paper_2510_23649_amd import binding
    turns = torch.zeros(64, dtype=torch.int64)
    with pytest.raises(ValueError):
        lib.make_rope(turns=turns, rot=128)                  # host memory
    monkeypatch.setattr(binding, "_dev", lambda x, dtype=None: None if x is None else A)
    monkeypatch.setattr(binding, "_here", lambda *a: 0)
    with pytest.raises(ValueError):
        lib.make_rope(turns=turns[:63], rot=128)
    with pytest.raises(TypeError):
        lib.make_rope(turns=turns.float(), rot=128)
    rope = lib.make_rope(turns=turns, rot=128)
    x = torch.zeros(4, 8, 128)
    with pytest.raises(ValueError):
        lib.lrqk_rotate(rope, torch.zeros(4, dtype=torch.int32), x, x)       # host memory

    class Fake(torch.Tensor):                # a host tensor that says it is a device's
        is_cuda = True

    fake = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt).as_subclass(Fake)  # noqa: E731
    pos = torch.zeros(4, dtype=torch.int32)
    q, k = fake(4, 8, 128), fake(4, 2, 128)
    bad = [(ValueError, dict(q=q)), (ValueError, dict(q_out=q)), (ValueError, dict(k=k)), (ValueError, dict(q=q, q_out=q, k=k)),
           (ValueError, dict(q=q, q_out=fake(4, 7, 128))), (ValueError, dict(q=q, q_out=fake(3, 8, 128))), (ValueError, dict(q=fake(4, 8, 64), q_out=q)),
           (ValueError, dict(q=q.transpose(0, 1), q_out=q)), (ValueError, dict(q=fake(8, 4, 128).transpose(0, 1), q_out=q)),
           (ValueError, dict(q=fake(4, 8, 256)[..., ::2], q_out=q)), (ValueError, dict(q=fake(1, 8, 128).expand(4, 8, 128), q_out=q)),
           (TypeError, dict(q=fake(4, 8, 128, dt=torch.float16), q_out=q)), (ValueError, dict(k=k, k_out=fake(4, 2, 128, dt=torch.float32)))]
    for err, kw in bad:
        with pytest.raises(err):
            lib.lrqk_rotate(rope, pos, **kw)
    with pytest.raises(lib.LrqkError):       # nothing to turn
        lib.lrqk_rotate(rope, pos)
    s = good(lib, page_dtype=2)
    p = held(lib, monkeypatch)
    q, k = fake(7, 28, 128), fake(7, 4, 128)
    monkeypatch.setattr(binding, "_fits", lambda *a, **kw: A)
    go = lambda **kw: lib.lrqk_pages_rotate_append(s, p, rope, **dict(dict(q=q, k_new=k, v_new=k, q_out=q), **kw))  # noqa: E731
    for err, kw in ((ValueError, dict(q=None)), (ValueError, dict(q_out=None)), (ValueError, dict(q=fake(7, 27, 128))), (ValueError, dict(v_new=fake(7, 5, 128))),
                    (ValueError, dict(k_new=fake(6, 4, 128))), (TypeError, dict(v_new=fake(7, 4, 128, dt=torch.float32))), (ValueError, dict(pos=pos)),
                    (ValueError, dict(slot=pos)), (ValueError, dict(pos=pos, slot=pos))):
        with pytest.raises(err):
            go(**kw)


def test_binding_refuses_tables(lib, monkeypatch):  # noqa: F811
    from paper_2510_23649_amd import binding
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    t = dict(refs=i32(200), table=i32(2, 63), kv_len=i32(2), start=i32(3), status=i32(2), seq=i32(7), pos=i32(7), slot=i32(7))
    with pytest.raises(ValueError):
        lib.make_pages_tables(**t)                           # host memory
    monkeypatch.setattr(binding, "_dev", lambda x, dtype=None: None if x is None else A)
    monkeypatch.setattr(binding, "_raw_stream", lambda *a: 0)
    s, ws = good(lib), torch.zeros(16, dtype=torch.uint8)
    go = lambda **kw: lib.lrqk_pages_advance(s, lib.make_pages_tables(**dict(t, **kw)), None, i32(2), ws)  # noqa: E731
    with pytest.raises(lib.LrqkError) as e:  # fits: the library says that the workspace is too small
        go()
    assert e.value.status == -4
    for name, x in (("refs", i32(199)), ("table", i32(2, 62)), ("table", i32(2, 70)), ("kv_len", i32(1)), ("start", i32(2)), ("status", i32(1)),
                    ("seq", i32(6)), ("pos", i32(0)), ("slot", i32(6))):
        with pytest.raises(ValueError):
            go(**{name: x})
    with pytest.raises(ValueError):
        lib.lrqk_pages_advance(s, lib.make_pages_tables(**t), i32(1), i32(2), ws)
    with pytest.raises(ValueError):
        lib.lrqk_pages_advance(s, lib.make_pages_tables(**t), None, i32(1), ws)


def test_plain_advance():
    """The plain form by hand."""
    refs, table, ln = np.zeros(6, np.int32), np.full((2, 4), -1, np.int32), np.zeros(2, np.int32)
    w = X.advance(refs, table, ln, None, [5, 3], page=4, n_max=9, l_max=16, T=9)
    assert w["table"].tolist() == [[0, 1, -1, -1], [2, -1, -1, -1]] and w["start"].tolist() == [0, 5, 8] and w["refs"].tolist() == [1, 1, 1, 0, 0, 0]
    assert w["slot"].tolist() == [0, 1, 2, 3, 4, 8, 9, 10, -1] and w["pos"].tolist() == [0, 1, 2, 3, 4, 0, 1, 2, -1]
    w = X.advance(w["refs"], w["table"], w["kv_len"], [4, 3], [0, 6], page=4, n_max=9, l_max=16, T=9)
    assert w["table"].tolist() == [[0, -1, -1, -1], [2, 1, 3, -1]] and w["kv_len"].tolist() == [4, 9] and w["seq"].tolist() == [1] * 6 + [-1] * 3
    w = X.advance(w["refs"], w["table"], w["kv_len"], [4, 9], [9, 1], page=4, n_max=9, l_max=16, T=9)
    assert w["status"].tolist() == [X.PAGES, X.ROWS]         # 3 pages of 2 that are free; 9 + 1 rows of 9

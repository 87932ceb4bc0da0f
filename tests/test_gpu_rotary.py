"""GPU tests of rotary positions: lrqk_rotate against float64, lrqk_pages_rotate_append against lrqk_rotate and
lrqk_pages_append bit for bit.  A turned element may be off by

  8 2^-24 amplitude (|x_u| + |x_v|)

(cosine and sine are off by at most 3.2 2^-24: 1.7 from the angle, whose conversion, constant and product are rounded, 1.5 from
the series; the amplitude's product adds 1, the two products and their sum 2: 6 to 7 in all) and by half a step of its type."""
import numpy as np
import pytest
import torch

import paper_2510_23649_amd as L
import pages_plain as P
import tables_plain as X
import test_gpu_pages as base
from test_gpu_pages import DEV, D, MARK, Case

pytestmark = pytest.mark.gpu
base.PAGE["e2m1"] = L.LRQK_PAGE_E2M1
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
B16, F32 = torch.bfloat16, torch.float32


def rope_of(rot, scaling=X.PLAIN, layout=0, back=False, amplitude=None, **kw):
    kw = dict(dict(base=10000.0), **kw)
    turns, a = L.lrqk_rope_turns(rot, scaling, **kw)
    f, want = X.frequencies(rot, scaling, **kw)
    assert abs(a - want) < 1e-6
    a = a if amplitude is None else amplitude
    return L.make_rope(turns=turns.to(DEV), rot=rot, layout=layout, amplitude=a, back=back), f, float(np.float32(a))


def check(got, x, pos, f, amplitude, pairs, back):
    """got: the output; x: the input, both [T,H,128]."""
    y, mass = X.turned(x.double().cpu().numpy(), pos.cpu().numpy(), f, amplitude, pairs, back)
    g = got.double().cpu().numpy()
    rot = 2 * len(f)
    if got.dtype == x.dtype:                 # what is not turned stays as it is
        assert torch.equal(got[..., rot:].contiguous().view(torch.uint8), x[..., rot:].contiguous().view(torch.uint8))
    nan = np.isnan(y)
    assert np.array_equal(np.isnan(g), nan)
    inf = np.isinf(y)
    assert np.array_equal(g[inf], y[inf])
    fine = np.isfinite(y)
    far = np.abs(np.where(fine, g - np.where(fine, y, 0), 0))
    tol = 8 * 2.0 ** -24 * abs(amplitude) * mass + HALF[got.dtype] * np.abs(y) * (1 + 2.0 ** -20) + 1e-37
    bad = fine & ~(far <= np.where(fine, tol, 0))
    assert not bad.any(), f"off by {far[bad].max()} at {np.argwhere(bad)[0]}"


def packed(T, Hq, Hkv, dt, g, pad=0):
    """q, k, v as parts of one projection's rows."""
    x = torch.randn(T, Hq + 2 * Hkv + pad, D, generator=g).to(dt).to(DEV)
    return x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:Hq + 2 * Hkv], x


def test_the_bound_notices_a_wrong_turn():
    """The comparison itself, on the host: a sine of the wrong sign, a pair of the other layout, a position off by one."""
    g = np.random.default_rng(0)
    x, pos = g.standard_normal((3, 2, D)), np.array([1, 5, 100])
    f, _ = X.frequencies(64, X.PLAIN, 10000.0)
    y, _ = X.turned(x, pos, f, 1.0, False, False)
    xt, pt = torch.from_numpy(x).float(), torch.from_numpy(pos)
    x = xt.double().numpy()
    good = torch.from_numpy(X.turned(x, pos, f, 1.0, False, False)[0]).float()
    check(good, xt, pt, f, 1.0, False, False)
    for other in (X.turned(x, pos, f, 1.0, False, True), X.turned(x, pos, f, 1.0, True, False), X.turned(x, pos + 1, f, 1.0, False, False),
                  X.turned(x, pos, f, 1.00001, False, False)):
        with pytest.raises(AssertionError):
            check(torch.from_numpy(other[0]).float(), xt, pt, f, 1.0, False, False)


@pytest.mark.parametrize("layout", [0, 1], ids=["halves", "pairs"])
@pytest.mark.parametrize("rot", [2, 4, 6, 16, 20, 32, 48, 62, 64, 96, 110, 112, 126, 128])
def test_parts_of_a_head(rot, layout):
    g = torch.Generator().manual_seed(rot)
    for i, (qi, qo, kt) in enumerate([(B16, B16, B16), (F32, F32, F32), (B16, F32, B16), (F32, B16, F32), (F32, F32, B16), (B16, B16, F32)]):
        T, Hq, Hkv = [(1, 8, 2), (5, 7, 7), (70, 3, 1), (33, 28, 4), (2, 1, 9), (400, 5, 6)][i]
        rope, f, a = rope_of(rot, layout=layout, back=bool(i % 2), amplitude=[1.0, 1.25][i // 3])
        pos = torch.randint(0, 5000, (T,), generator=g, dtype=torch.int32).to(DEV)
        q, k = torch.randn(T, Hq, D, generator=g).to(qi).to(DEV), torch.randn(T, Hkv, D, generator=g).to(kt).to(DEV)
        qo_, ko = torch.full((T, Hq, D), MARK, dtype=qo, device=DEV), torch.full((T, Hkv, D), MARK, dtype=kt, device=DEV)
        L.lrqk_rotate(rope, pos, q, qo_, k, ko)
        check(qo_, q, pos, f, a, layout, bool(i % 2))
        check(ko, k, pos, f, a, layout, bool(i % 2))


@pytest.mark.parametrize("scaling", [X.PLAIN, X.LINEAR, X.BASE, X.BANDS, X.RAMP])
@pytest.mark.parametrize("layout,rot", [(0, 128), (1, 64), (0, 34)])
def test_scaled_for_long_contexts(layout, rot, scaling):
    g = torch.Generator().manual_seed(1)
    rope, f, a = rope_of(rot, scaling, layout, base=500000.0, factor=8.0, low=1.0, high=32.0, l_orig=4096)
    pos = torch.tensor([0, 1, 4095, 32767, 131071, 1 << 20, (1 << 24) - 1], dtype=torch.int32).to(DEV)
    q, out = torch.randn(7, 4, D, generator=g).to(DEV), torch.empty(7, 4, D, device=DEV)
    L.lrqk_rotate(rope, pos, q, out)
    check(out, q, pos, f, a, layout, False)


def test_far_and_negative_positions():
    """Up to 2^24 positions the reference's own angle is off by less than 2^-29; beyond, pairs whose frequency is a power of two
    over 2 pi turns are compared: angles that float64 has exactly."""
    g = torch.Generator().manual_seed(2)
    rope, f, a = rope_of(128)
    pos = torch.tensor([-1, -7, -4096, -(1 << 24), 0, 3], dtype=torch.int32).to(DEV)
    q, out = torch.randn(6, 2, D, generator=g).to(DEV), torch.empty(6, 2, D, device=DEV)
    L.lrqk_rotate(rope, pos, q, out)
    check(out, q, pos, f, a, 0, False)
    # turns of 2^-j, exactly
    turns = torch.tensor([1 << (63 - j) if j else -(1 << 63) for j in range(64)], dtype=torch.int64)
    rope = L.make_rope(turns=turns.to(DEV), rot=128)
    pos = torch.tensor([-(1 << 31), (1 << 31) - 1, 123456789, -987654321, 1, 0], dtype=torch.int32)
    L.lrqk_rotate(rope, pos.to(DEV), q, out)
    step = np.array([2.0 ** -(j + 1) for j in range(64)])
    frac = np.array([[(int(p) * (1 << (63 - j))) % (1 << 64) / 2.0 ** 64 for j in range(64)] for p in pos])
    x = q.double().cpu().numpy()
    c, s = np.cos(2 * np.pi * frac)[:, None], np.sin(2 * np.pi * frac)[:, None]
    y = np.concatenate([x[..., :64] * c - x[..., 64:] * s, x[..., 64:] * c + x[..., :64] * s], -1)
    mass = np.tile(np.abs(x[..., :64]) + np.abs(x[..., 64:]), 2)
    assert step[0] == 0.5 and (np.abs(out.double().cpu().numpy() - y) <= 8 * 2.0 ** -24 * mass + 2.0 ** -24 * np.abs(y)).all()


@pytest.mark.parametrize("dt", [B16, F32])
def test_strides(dt):
    """q and k as parts of one projection's rows, outputs with rows between them that nothing may touch."""
    g = torch.Generator().manual_seed(3)
    for T in (1, 2, 65, 600):
        q, k, _, whole = packed(T, 6, 3, dt, g, pad=1)
        keep = whole.clone()
        rope, f, a = rope_of(128, layout=T % 2)
        pos = torch.randint(0, 100000, (T,), generator=g, dtype=torch.int32).to(DEV)
        out = torch.full((T, 12, D), MARK, dtype=dt, device=DEV)
        L.lrqk_rotate(rope, pos, q, out[:, 1:7], k, out[:, 8:11])
        check(out[:, 1:7], q, pos, f, a, T % 2, False)
        check(out[:, 8:11], k, pos, f, a, T % 2, False)
        assert torch.equal(whole, keep) and (out[:, [0, 7, 11]] == MARK).all()


@pytest.mark.parametrize("dt", [B16, F32])
@pytest.mark.parametrize("rot,layout", [(128, 0), (128, 1), (20, 0), (52, 0), (126, 0), (64, 0)])
def test_in_place(rot, layout, dt):
    g = torch.Generator().manual_seed(4)
    for T in (1, 300, 3000):
        q, k, v, whole = packed(T, 8, 2, dt, g)
        q0, k0, v0 = q.clone(), k.clone(), v.clone()
        rope, f, a = rope_of(rot, layout=layout)
        pos = torch.randint(0, 100000, (T,), generator=g, dtype=torch.int32).to(DEV)
        L.lrqk_rotate(rope, pos, q, q, k, k)
        check(q, q0, pos, f, a, layout, False)
        check(k, k0, pos, f, a, layout, False)
        assert torch.equal(v, v0)


@pytest.mark.parametrize("dt", [B16, F32])
def test_many_heads_and_many_tokens(dt):
    g = torch.Generator().manual_seed(11)
    for T, Hq, Hkv in ((2, 1024, 1), (3, 1, 1023), (9000, 2, 1)):
        rope, f, a = rope_of(128, layout=T % 2)
        pos = torch.randint(0, 100000, (T,), generator=g, dtype=torch.int32).to(DEV)
        q, k = torch.randn(T, Hq, D, generator=g).to(dt).to(DEV), torch.randn(T, Hkv, D, generator=g).to(dt).to(DEV)
        qo, ko = torch.full_like(q, MARK), torch.full_like(k, MARK)
        L.lrqk_rotate(rope, pos, q, qo, k, ko)
        check(qo, q, pos, f, a, T % 2, False)
        check(ko, k, pos, f, a, T % 2, False)


def test_one_of_both():
    g = torch.Generator().manual_seed(5)
    rope, f, a = rope_of(128)
    pos = torch.arange(9, dtype=torch.int32, device=DEV)
    for dt in (B16, F32):
        x, out = torch.randn(9, 5, D, generator=g).to(dt).to(DEV), torch.empty(9, 5, D, dtype=dt, device=DEV)
        L.lrqk_rotate(rope, pos, q=x, q_out=out)
        check(out, x, pos, f, a, 0, False)
        out2 = torch.empty_like(out)
        L.lrqk_rotate(rope, pos, k=x, k_out=out2)
        assert torch.equal(out, out2)


@pytest.mark.parametrize("dt", [B16, F32])
@pytest.mark.parametrize("rot,layout", [(128, 0), (128, 1), (40, 0), (44, 0), (42, 1)])
def test_what_is_no_number_stays_in_its_pair(rot, layout, dt):
    g = torch.Generator().manual_seed(6)
    rope, f, a = rope_of(rot, layout=layout)
    pos = torch.randint(1, 1000, (12,), generator=g, dtype=torch.int32).to(DEV)
    x = torch.randn(12, 4, D, generator=g).to(dt)
    bad = [float("nan"), float("inf"), -float("inf"), 3.0e38]
    for t in range(12):
        x[t, t % 4, [0, rot - 1, rot // 2, 127, 5, 1][t % 6]] = bad[t % 4]
    x = x.to(DEV)
    out = torch.empty_like(x)
    L.lrqk_rotate(rope, pos, x, out)
    y, _ = X.turned(x.double().cpu().numpy(), pos.cpu().numpy(), f, a, layout, False)
    big = float(torch.finfo(dt).max)
    assert np.abs(y[np.isfinite(y)]).max() < 4.5e38
    near = np.isfinite(y) & (np.abs(y) > big * 0.99)         # beyond the type, or next to it
    got = out.double().cpu().numpy()
    assert np.array_equal(np.isnan(got[~near]), np.isnan(y[~near]))
    fine = np.isfinite(y) & (np.abs(y) < 1e30)
    want = torch.from_numpy(np.where(fine, y, 0.0))
    tol = 8 * 2.0 ** -24 * np.abs(X.turned(x.double().cpu().numpy(), pos.cpu().numpy(), f, a, layout, False)[1]) + HALF[dt] * np.abs(want.numpy()) * 1.001
    assert (np.abs(np.where(fine, got, 0) - want.numpy()) <= np.where(fine & np.isfinite(tol), tol, np.inf)).all()


@pytest.mark.parametrize("rot,layout", [(128, 0), (64, 1), (12, 0)])
def test_back_is_the_gradient(rot, layout):
    """Against differences: the map is linear, so (f(x + h e) - f(x)) / h is its column, off by the bound of two results over h;
    and <f(x), g> = <x, back(g)>."""
    g = torch.Generator().manual_seed(7)
    T, h = 3, 64.0
    fwd, f, a = rope_of(rot, layout=layout, amplitude=1.5)
    bwd, _, _ = rope_of(rot, layout=layout, amplitude=1.5, back=True)
    pos = torch.tensor([1, 1000, 70000], dtype=torch.int32, device=DEV)
    x = torch.randn(T, 1, D, generator=g).to(DEV)
    grad = torch.randn(T, 1, D, generator=g).to(DEV)
    got, y0 = torch.empty_like(x), torch.empty_like(x)
    L.lrqk_rotate(bwd, pos, grad, got)
    L.lrqk_rotate(fwd, pos, x, y0)
    check(got, grad, pos, f, a, layout, True)
    # all 128 columns at once: heads are independent
    moved = x.repeat(1, D, 1) + h * torch.eye(D, device=DEV)
    y1 = torch.empty_like(moved)
    L.lrqk_rotate(fwd, pos, moved, y1)
    col = (y1.double() - y0.double()) / h                    # [T, D (moved), D (result)]
    num = (col * grad.double()).sum(-1)
    tol = 2 * 9 * 2.0 ** -24 * 1.5 * (2 * h + 20) / h * grad.double().abs().sum(-1)
    assert ((num - got.double()[:, 0]).abs() <= tol).all()
    lhs, rhs = (y0.double() * grad.double()).sum(), (x.double() * got.double()).sum()
    assert float((lhs - rhs).abs()) <= 2 * 9 * 2.0 ** -24 * 1.5 * float((2 * x.double().abs() * 2 * grad.double().abs().amax()).sum())


def test_back_undoes_it():
    g = torch.Generator().manual_seed(8)
    fwd, f, _ = rope_of(96)
    bwd, _, _ = rope_of(96, back=True)
    x = torch.randn(50, 8, D, generator=g).to(DEV)
    pos = torch.randint(0, 1 << 24, (50,), generator=g, dtype=torch.int32).to(DEV)
    y, z = torch.empty_like(x), torch.empty_like(x)
    L.lrqk_rotate(fwd, pos, x, y)
    L.lrqk_rotate(bwd, pos, y, z)
    _, mass = X.turned(x.double().cpu().numpy(), pos.cpu().numpy(), f, 1.0, False, False)
    assert ((z - x).abs().cpu().numpy() <= 2 * 9 * 2.0 ** -24 * np.sqrt(2) * 2 * mass + 1e-37).all()


# ---- turned and appended -----------------------------------------------------------------------------------
KINDS = [("bf16", "bf16"), ("f32", "f32"), ("bf16", "e4m3"), ("bf16", "i8"), ("f32", "e4m3"), ("f32", "i8"), ("bf16", "e2m1"), ("f32", "e2m1")]


def both(c, rope, maps, q_in_place=False, no_q=False):
    """The one call and the two, on pools that hold the same; everything has to be the same bits."""
    g = torch.Generator().manual_seed(99)
    dt = P.TYPE[c.kv]
    q, k, v, whole = packed(c.T, c.Hq, c.Hkv, dt, g)
    if q_in_place:
        q = q.contiguous()
    n = np.diff(c.start)
    seq = np.repeat(np.arange(c.B), n)
    pos = np.full(c.T, -1, np.int32)
    slot = np.full(c.T, -1, np.int32)
    for t, b in zip(range(int(c.start[0]), int(c.start[-1])), seq):
        pos[t] = c.len[b] - n[b] + (t - c.start[b])
        at = c.where(int(b), int(pos[t]))
        slot[t] = -1 if at is None else at[0] * c.page + at[1]
    dpos, dslot = torch.from_numpy(pos).to(DEV), torch.from_numpy(slot).to(DEV)
    mark = lambda: torch.full((c.T, c.Hq, D), MARK, dtype=dt, device=DEV)  # noqa: E731
    # the two calls, as dense rows
    q1, k1 = mark(), torch.empty(c.T, c.Hkv, D, dtype=dt, device=DEV)
    L.lrqk_rotate(rope, dpos, q, q1, k, k1)
    q1[torch.from_numpy(pos < 0).to(DEV)] = q[torch.from_numpy(pos < 0).to(DEV)] if q_in_place else MARK
    want = {x: c.d[x].clone() for x in "KV"}, {x: None if c.ds[x] is None else c.ds[x].clone() for x in "KV"}
    pg = L.make_pages(K=want[0]["K"], V=want[0]["V"], K_scale=want[1]["K"], V_scale=want[1]["V"], table=c.dtable, start=c.dstart, kv_len=c.dlen)
    L.lrqk_pages_append(c.shape, pg, k1, v.contiguous())
    # the one
    q2 = q if q_in_place else mark()
    L.lrqk_pages_rotate_append(c.shape, c.pg, rope, None if no_q else q, k, v, None if no_q else q2, **(dict(pos=dpos, slot=dslot) if maps else {}))
    bits = lambda x: x.contiguous().view(torch.uint8)  # noqa: E731
    if not no_q:
        assert torch.equal(bits(q2), bits(q1))
    for x in "KV":
        assert torch.equal(bits(c.d[x]), bits(want[0][x])), x
        assert c.ds[x] is None or torch.equal(c.ds[x], want[1][x]), x


@pytest.mark.parametrize("kv,pages", KINDS)
@pytest.mark.parametrize("maps", [False, True], ids=["tables", "maps"])
@pytest.mark.parametrize("seqs", [[(1, 1)], [(1, 40), (1, 7), (1, 16)], [(70, 100), (0, 9), (33, 33), (5, 3)]], ids=["one", "step", "chunk"])
def test_one_call_is_the_two(seqs, maps, kv, pages):
    for i, (page, Hkv, G) in enumerate([(16, 2, 4), (1, 3, 1), (256, 5, 3), (64, 8, 2)]):
        rope, _, _ = rope_of([128, 64, 20, 96][i], layout=i % 2, amplitude=1.2)
        c = Case(seqs, Hkv, G, page, kv, pages, seed=20 + i, front=2, back=3, holes=0.1 if len(seqs) > 2 else 0.0).to_device()
        both(c, rope, maps, q_in_place=i == 2, no_q=i == 3)


@pytest.mark.parametrize("maps", [False, True], ids=["tables", "maps"])
def test_positions_that_do_not_exist(maps):
    """Below 0: nothing is written.  From l_max on: q is turned, k and v have no place."""
    for seqs, l_max in (([(10, 4), (3, 0), (40, 20), (1, 0)], None), ([(20, 150), (3, 90), (1, 400)], 100)):
        for kv, pages in (("bf16", "e2m1"), ("f32", "f32")):
            c = Case(seqs, 2, 4, 16, kv, pages, seed=3, l_max=l_max).to_device()
            both(c, rope_of(128)[0], maps)


@pytest.mark.parametrize("kv,pages", [("bf16", "e2m1"), ("f32", "f32")])
def test_many_heads_of_pages(kv, pages):
    for maps in (False, True):
        c = Case([(3, 20), (1, 9)], 33, 8, 16, kv, pages, seed=31).to_device()
        both(c, rope_of(62, layout=0)[0], maps)


def test_many_sequences_and_tokens():
    rng = np.random.default_rng(14)
    c = Case([(int(rng.integers(0, 40)), int(rng.integers(40, 160))) for _ in range(150)], 2, 2, 16, "bf16", "e2m1", seed=14).to_device()
    both(c, rope_of(128)[0], False)


def test_slots_that_are_no_rows():
    """Slots outside the pool drop k and v and nothing else; no address comes of them."""
    c = Case([(6, 6)], 2, 2, 16, "bf16", "bf16", seed=1).to_device()
    rope, f, a = rope_of(128)
    g = torch.Generator().manual_seed(1)
    q, k, v, _ = packed(6, 4, 2, B16, g)
    keep = {x: c.d[x].clone() for x in "KV"}
    pos = torch.tensor([0, 1, 2, 3, -1, -5], dtype=torch.int32, device=DEV)
    slot = torch.tensor([-1, c.n_pages * 16, (1 << 31) - 1, -(1 << 31), 3, 4], dtype=torch.int32, device=DEV)
    out = torch.full((6, 4, D), MARK, dtype=B16, device=DEV)
    L.lrqk_pages_rotate_append(c.shape, c.pg, rope, q, k, v, out, pos=pos, slot=slot)
    assert all(torch.equal(c.d[x].view(torch.int16), keep[x].view(torch.int16)) for x in "KV")
    check(out[:4], q[:4], pos[:4], f, a, 0, False)
    assert (out[4:] == MARK).all()


def test_streams_and_graphs():
    """On another stream, and captured: a replay follows the positions, rows and slots that the memory holds."""
    g = torch.Generator().manual_seed(9)
    c = Case([(1, 300), (1, 300), (1, 300)], 2, 4, 16, "bf16", "e2m1", seed=4).to_device()
    rope, f, a = rope_of(128)
    q, k, v, whole = packed(3, 8, 2, B16, g)
    out, out2 = (torch.zeros(3, 8, D, dtype=B16, device=DEV) for _ in range(2))
    ko = torch.zeros(3, 2, D, dtype=B16, device=DEV)
    pos, slot = (torch.zeros(3, dtype=torch.int32, device=DEV) for _ in range(2))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.lrqk_rotate(rope, pos, q, out2, k, ko)
        L.lrqk_pages_rotate_append(c.shape, c.pg, rope, q, k, v, out, pos=pos, slot=slot)
    s = torch.cuda.Stream()
    for i in range(4):
        whole.copy_(torch.randn(whole.shape, generator=g).to(B16))
        pos.copy_(torch.randint(0, 300, (3,), generator=g).to(torch.int32))
        slot.copy_(torch.randperm(c.n_pages * 16, generator=g)[:3].to(torch.int32))
        before = {x: c.d[x].clone() for x in "KV"}, {x: c.ds[x].clone() for x in "KV"}
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), out2.clone(), {x: c.d[x].clone() for x in "KV"}, {x: c.ds[x].clone() for x in "KV"}
        for x in "KV":
            c.d[x].copy_(before[0][x])
            c.ds[x].copy_(before[1][x])
        out.zero_()
        torch.cuda.synchronize()
        L.lrqk_pages_rotate_append(c.shape, c.pg, rope, q, k, v, out, pos=pos, slot=slot, stream=s)
        s.synchronize()
        assert torch.equal(got[0], out) and torch.equal(got[1], out)
        assert all(torch.equal(got[2][x], c.d[x]) and torch.equal(got[3][x], c.ds[x]) for x in "KV")
        check(out, q, pos, f, a, 0, False)


def test_a_decode_step_at_its_position():
    """q and k of a decode step turned into what the factor update and the decode step take: q in fp32 out of bf16 rows; with every position
    selected the step is the attention over pages that hold keys turned the same way."""
    Hkv, G, l, r = 2, 4, 200, 32
    Hq, w, ksel = Hkv * G, 16, l - 16
    g = torch.Generator().manual_seed(10)
    rope, f, a = rope_of(128, X.BANDS, factor=4.0, l_orig=64)
    q, k, v, _ = packed(l, Hq, Hkv, B16, g)
    pos = torch.arange(l, dtype=torch.int32, device=DEV)
    q32, k_t = torch.empty(l, Hq, D, device=DEV), torch.empty(l, Hkv, D, dtype=B16, device=DEV)
    L.lrqk_rotate(rope, pos, q, q32, k, k_t)
    check(q32, q, pos, f, a, 0, False)
    Kp, Vp = (torch.empty((1, Hkv, l, D), dtype=B16).pin_memory() for _ in range(2))
    Kp.copy_(k_t.permute(1, 0, 2)[None])
    Vp.copy_(v.permute(1, 0, 2)[None])
    torch.cuda.synchronize()
    shp = L.Shape.make(B=1, Hq=Hq, Hkv=Hkv, l=l, r=r, k=ksel, w=w, C_slots=ksel)
    A_K = torch.randn(1, Hkv, l, r, generator=g).to(DEV)
    buf, plan = L.LayerBuffers(shp, A_K, Kp, Vp), L.Plan(shp)
    out1 = torch.zeros(1, Hq, D, device=DEV)
    L.lrqk_decode_step(plan, shp, 0, buf.struct, torch.randn(1, Hq, r, generator=g).to(DEV), q32[-1:].contiguous(), out1,
                       L.LRQK_FETCH_DIRECT | L.LRQK_SELECT_FRESH)
    torch.cuda.synchronize()
    qd, Kd, Vd = q32[-1].double().cpu(), k_t.double().cpu(), v.double().cpu()
    for h in range(Hq):
        s = (Kd[:, h // G] @ qd[h]) * float(np.float32(D ** -0.5))
        p = torch.softmax(s, 0)
        y, mass = p @ Vd[:, h // G], p @ Vd[:, h // G].abs()
        slack = 2 * (float((Kd[:, h // G].abs() @ qd[h].abs()).max()) * D ** -0.5 * 130 + 3 * float(s.abs().max()) + 4) * 2.0 ** -24
        assert ((out1[0, h].double().cpu() - y).abs() <= 2.0 ** -24 * y.abs() + mass * (slack + 2 * l * 2.0 ** -24)).all()
    plan.close()

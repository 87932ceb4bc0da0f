"""GPU tests of the paged cache at the ends of the number range: rows near the largest finite numbers, scores that are
huge, of the lowest value or of -infinity, infinities that only some tokens see, contexts of 128K.  Cases, plain
forms and bounds are those of tests/test_gpu_pages.py unless a test says otherwise."""
import numpy as np
import pytest
import torch

import paper_2510_23649_amd as L
import pages_plain as P
from test_gpu_pages import DEV, D, MARK, Case, exact_on_device

pytestmark = pytest.mark.gpu
E8 = [("bf16", "e4m3"), ("bf16", "i8"), ("f32", "e4m3"), ("f32", "i8")]
# (new tokens, length) of the first sequence, with three heads a group: one row a wavefront, 33 to 64 rows, more
WAYS = {"one": (1, 40), "thin": (9, 75), "pair": (14, 75), "tile": (70, 150)}
BIGGEST = {"bf16": float(torch.finfo(torch.bfloat16).max), "f32": float(torch.finfo(torch.float32).max)}


# ---- rows written in 8 bits --------------------------------------------------------------------------
def quantise(x, pages):
    """P.quantise, but that no finite element becomes 2^128, which neither bf16 nor fp32 holds: the next lower code."""
    code, byte = P.quantise(x, pages)
    top = np.repeat(byte == (247 if pages == "e4m3" else 249), 32, axis=-1)
    if pages == "e4m3":                      # 256 * 2^120 -> 240 * 2^120
        code = np.where(top & ((code & 0x7F) == 0x78), code - 1, code)
    else:                                    # 64 * 2^122 -> 63 * 2^122
        code = np.where(top & (code == 64), 63, np.where(top & (code == 192), 193, code))
    return code.astype(np.uint8), byte


def special_blocks(kv, pages, g):
    """Blocks of 32 elements at which a scale or a rounding can go wrong, as rows of 128 (four blocks a row)."""
    top, dt, big = P.TOP[pages], P.TYPE[kv], BIGGEST[kv]
    up = lambda x, to: float(torch.nextafter(torch.tensor(x, dtype=dt), torch.tensor(to, dtype=dt)))  # noqa: E731
    rnd = lambda: torch.randn(32, generator=g, dtype=torch.float64)  # noqa: E731
    one = lambda v, i=9: rnd().index_fill_(0, torch.tensor(i), v)  # noqa: E731
    steps = torch.arange(32, dtype=torch.float64)
    blocks = [torch.zeros(32), -torch.zeros(32), torch.full((32,), 3.0e38), torch.full((32,), 1.0e-30), torch.full((32,), 1.0e-40),
              torch.linspace(-top, top, 32), one(up(top, big), 0), one(-up(top, big)), one(up(top, 0.0)), one(top * 2.0 ** -110),
              torch.full((32,), -top * 2.0 ** -112), (steps * 0.5 + 0.25).index_fill_(0, torch.tensor(31), top),
              (steps + 0.5).index_fill_(0, torch.tensor(31), -top), one(float("nan"), 3), one(float("inf")), one(-float("inf")),
              # the largest finite numbers, and those around the last one that rounds down to a code whose value is finite
              torch.full((32,), big), -torch.full((32,), big), one(big), one(-big, 31), one(up(big, 0.0)),
              torch.linspace(-1.0, 1.0, 32, dtype=torch.float64) * big, torch.linspace(0.9, 1.0, 32, dtype=torch.float64) * big,
              one(247.0 * 2.0 ** 120), one(248.0 * 2.0 ** 120), one(-249.0 * 2.0 ** 120), one(1.75 * 2.0 ** 127),
              one(up(1.75 * 2.0 ** 127, big)), one(127.0 * 2.0 ** 121), one(up(127.0 * 2.0 ** 121, big)), one(-2.0 ** 127)]
    blocks += [rnd() for _ in range(-len(blocks) % 4)]
    return torch.stack([b.to(torch.float64) for b in blocks]).view(-1, 128).to(dt)


@pytest.mark.parametrize("kv,pages", E8)
@pytest.mark.parametrize("page,Hkv", [(16, 1), (4, 2), (64, 3)])
def test_special_blocks_are_written_and_read(page, Hkv, kv, pages):
    """Every special block in K and in V of tokens that belong to a sequence and have a page; finite elements stay finite."""
    x = special_blocks(kv, pages, torch.Generator().manual_seed(7))
    n = -(-x.shape[0] // Hkv)
    c = Case([(n, n + 5), (1, 3)], Hkv, 2, page, kv, pages, seed=60, front=2, back=3)
    x = torch.cat([x, x[:n * Hkv - x.shape[0]]])
    c.k_new[2:2 + n] = x.view(n, Hkv, D)
    c.v_new[2:2 + n] = x.flip(0).view(n, Hkv, D)
    assert all(c.where(0, 5 + i) is not None for i in range(n)) and int(c.start[0]) == 2 and int(c.start[1]) == 2 + n
    c.to_device()
    L.lrqk_pages_append(c.shape, c.pg, c.k_new.to(DEV), c.v_new.to(DEV))
    out = {a: torch.full((2, Hkv, n + 5, D), MARK, dtype=P.TYPE[kv], device=DEV) for a in "KV"}
    L.lrqk_pages_read(c.shape, c.pg, 0, out["K"], out["V"])
    for name, new in (("K", c.k_new), ("V", c.v_new)):
        code, byte = quantise(new[2:2 + n].double().numpy(), pages)
        at = [c.where(0, 5 + i) for i in range(n)]
        pg, off = [a[0] for a in at], [a[1] for a in at]
        assert np.array_equal(c.ds[name].cpu().numpy()[pg, :, off], byte), f"{name}: scales"
        assert np.array_equal(c.d[name].cpu().numpy()[pg, :, off], code), f"{name}: codes"
        got = out[name][0, :, 5:].transpose(0, 1).double().cpu().numpy()
        assert np.array_equal(got, P.values(code, byte, pages), equal_nan=True), f"{name}: values"
        fine = np.isfinite(new[2:2 + n].double().numpy().reshape(n, Hkv, 4, 32)).all(-1)
        assert np.isfinite(got.reshape(n, Hkv, 4, 32)).all(-1)[fine].all(), f"{name}: a finite element is read as an infinity"


# ---- infinities in V ---------------------------------------------------------------------------------
@pytest.mark.parametrize("kv,pages", E8)
@pytest.mark.parametrize("way", WAYS)
def test_codes_too_large_for_the_type(way, kv, pages):
    """A pool from elsewhere may hold codes whose value exceeds bf16 and fp32: infinities for the tokens that see them."""
    n, ln = WAYS[way]
    c = Case([(n, ln), (2, 40)], 1, 3, 16, kv, pages, seed=61)
    for p, d, minus in ((ln - 1, 5, False), (ln - max(1, n // 2), 40, True), (ln - n, 70, False), (2, 100, True)):
        pg, o = c.where(0, p)
        c.pool["V"][pg, 0, o, d // 32 * 32:d // 32 * 32 + 32] = 0
        c.pool["V"][pg, 0, o, d] = (0x7E if pages == "e4m3" else 0x7F) if not minus else (0xFE if pages == "e4m3" else 0x81)
        c.sc["V"][pg, 0, o, d // 32] = 254
    rows = c.rows

    def as_held(name, b):
        x, there = rows(name, b)
        return np.where(np.abs(x) > BIGGEST["f32"], np.copysign(np.inf, x), x), there

    c.rows = as_held
    c.to_device()
    c.check_attend(c.attend())


@pytest.mark.parametrize("kv", ["bf16", "f32"])
@pytest.mark.parametrize("way", WAYS)
def test_infinities_reach_the_tokens_that_see_them(way, kv):
    """Infinities and NaN in V rows of later tokens and of earlier ones, in K rows of later ones, for every shape of workgroup."""
    n, ln = WAYS[way]
    c = Case([(n, ln), (2, 40)], 2, 3, 16, kv, kv, seed=62)
    for j, p in enumerate((ln - 1, ln - max(1, n // 2), ln - n, 1)):
        pg, o = c.where(0, p)
        c.pool["V"][pg, j % 2, o, 5 + j] = [float("inf"), float("-inf"), float("nan"), float("inf")][j]
        if j == 0 and n > 1:
            c.pool["K"][pg, 1, o, 3] = float("nan")
    c.to_device()
    c.check_attend(c.attend())


@pytest.mark.parametrize("kv", ["bf16", "f32"])
@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("v", [0.0, float("inf"), float("nan")], ids=["finite", "inf", "nan"])
def test_scores_of_minus_infinity_alone(v, way, kv):
    """Tokens that see only scores of -infinity get zeros, whatever the rows of V hold."""
    n, ln = WAYS[way]
    c = Case([(n, ln), (1, 1)], 1, 3, 16, kv, kv, seed=63)
    c.q[..., 0], c.q[..., 1:] = 1.0, 0.0
    c.pool["K"][..., 0] = -float("inf")
    for p, d in ((ln - 1, 3), (ln - n, 60), (2, 127)):
        pg, o = c.where(0, p)
        c.pool["V"][pg, 0, o, d] = v
    c.to_device()
    assert (c.attend() == 0).all()


# ---- scores --------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kv", ["bf16", "f32"])
@pytest.mark.parametrize("way", WAYS)
def test_lowest_scores_beside_ordinary_ones(way, kv):
    n, ln = WAYS[way]
    c = Case([(n, ln), (1, 35)], 1, 3, 16, kv, kv, seed=64)
    c.q[..., 0] = 1.0
    for b, p, v in ((0, 7, -3.0e38), (0, ln - n, -float("inf")), (0, ln - n // 2 - 1, -3.0e38), (0, 33, -float("inf")), (1, 0, -3.0e38),
                    (1, 34, -float("inf"))):
        pg, o = c.where(b, p)
        c.pool["K"][pg, :, o, 1:] = 0.0
        c.pool["K"][pg, :, o, 0] = v
    c.to_device()
    c.check_attend(c.attend())


LONG = dict(WAYS, one_in_pieces=(1, 3000), pair_in_pieces=(14, 3000), tile_in_pieces=(50, 3000))


@pytest.mark.parametrize("kv", ["bf16", "f32"])
@pytest.mark.parametrize("way", LONG)
def test_huge_scores_all_alike(way, kv):
    """Scores are q . K = v exactly and all alike, so that every weight is exactly 1 and the output the mean of what is
    seen: off by its own rounding, those of the two sums over L positions and two for the quotient."""
    n, ln = LONG[way]
    c = Case([(n, ln)], 1, 3, 16, kv, kv, seed=65)
    c.q[..., 0], c.q[..., 1:] = 1.0, 0.0
    c.pool["K"][:] = 0.0
    V, _ = c.rows("V", 0)
    many = np.arange(ln - n, ln)[:, None] + 1.0
    y, mass = (np.cumsum(x, 0)[ln - n:, None] / many[:, None] for x in (V[0], np.abs(V[0])))
    tol = (2.0 ** -8 if kv == "bf16" else 2.0 ** -24) * np.abs(y) + mass * (2 * ln + 2) * 2.0 ** -24
    c.to_device()
    for v in (-3.0e38, 3.0e38, -1.0e30, 1.0e12, -5.0e9, 1.0e6):
        c.d["K"][..., 0] = v
        got = c.attend().double().cpu().numpy()
        assert (np.abs(got - y) <= tol).all(), (v, np.abs(got - y).max())


@pytest.mark.parametrize("kv", ["bf16", "f32"])
@pytest.mark.parametrize("way", LONG)
@pytest.mark.parametrize("order", ["grows", "falls", "mixed"])
def test_huge_scores_far_apart(order, way, kv):
    """Scores that are multiples of a large power of two, exactly: all weight on the largest, whose row of V is the output.
    (Scores differ by 2^22 sqrt(1 / 128) at least: what the others count for is 0.)  Its weight w need not be 1, since the
    maximum that it is taken at is rounded: y = fl(fl(w V) fl(1 / w)) has three roundings in fp32, (1 + 2^-24)^3 - 1 < 3.001 2^-24;
    in bf16 fl(w V) of two bf16 numbers is exact and the output's rounding takes the other two back: nothing is off."""
    n, ln = LONG[way]
    first = ln - n
    c = Case([(n, ln)], 1, 3, 16, kv, kv, seed=66)
    c.q[..., 0], c.q[..., 1:] = 1.0, 0.0
    c.pool["K"][:] = 0.0
    V, _ = c.rows("V", 0)
    m = np.zeros(ln)                         # 1 .. 240 (8 bits: exact in bf16) at some positions, 0 at the others
    some = np.linspace(0, ln - 1, min(ln, 240)).astype(np.int64)
    m[some] = np.arange(1, len(some) + 1)
    if order == "falls":
        m = m[::-1].copy()
    elif order == "mixed":
        m[some] = np.random.default_rng(67).permutation(m[some])
    best = np.array([int(np.argmax(m[:i + 1])) for i in range(first, ln)])
    assert all((np.delete(m[:i + 1], j) < m[j]).all() for i, j in zip(range(first, ln), best)), "one largest score a token"
    c.to_device()
    at = [c.where(0, p) for p in range(ln)]
    for unit, off in ((2.0 ** 113, 0.0), (2.0 ** 113, 250.0), (2.0 ** 40, 0.0), (2.0 ** 30, 250.0), (2.0 ** 26, 0.0), (2.0 ** 22, 250.0)):
        k = torch.from_numpy(unit * (m - off)).to(P.TYPE[kv])
        assert np.array_equal(k.double().numpy(), unit * (m - off))
        c.d["K"][[a[0] for a in at], 0, [a[1] for a in at], 0] = k.to(DEV)
        got = c.attend().double().cpu().numpy()
        y = np.repeat(V[0, best][:, None], 3, axis=1)
        assert (np.abs(got - y) <= (0.0 if kv == "bf16" else 3.001 * 2.0 ** -24) * np.abs(y)).all(), (unit, off)


# ---- lengths -------------------------------------------------------------------------------------------
ONES, PAIR, TILE = [(1, 131072), (1, 0), (1, 1)], [(13, 131072), (2, 131001)], [(40, 131071)]


@pytest.mark.parametrize("seqs,kv,pages", [(ONES, "bf16", "e4m3"), (ONES, "f32", "f32"), (PAIR, "bf16", "i8"), (PAIR, "f32", "e4m3"),
                                           (TILE, "bf16", "bf16"), (TILE, "bf16", "e4m3")])
def test_128k(seqs, kv, pages):
    c = Case(seqs, 1, 4, 256, kv, pages, seed=68).to_device()
    out = c.attend().double()
    for b in range(c.B):
        lo, hi = int(c.start[b]), int(c.start[b + 1])
        if c.len[b] == 0:
            assert (out[lo:hi] == 0).all()
            continue
        y, mass, slack, Ln = exact_on_device(c, b)
        half = 2.0 ** -8 if kv == "bf16" else 2.0 ** -24
        tol = half * y.abs() + mass * (slack + 2 * Ln * 2.0 ** -24 + (2.0 ** -8 if kv == "bf16" else 0.0))
        assert float(((out[lo:hi] - y).abs() - tol).max()) <= 0, f"sequence {b}"

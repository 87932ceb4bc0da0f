"""GPU tests of pages of 4 bits (e2m1): rows written, read and attended.  Cases and bounds are those of
tests/test_gpu_pages.py: codes and scales bit for bit, rows read back exactly, an attention's output off by

  bf16:  2^-8 |y| (its own rounding) + 2^-8 sum_p w_p |V_p| (the weights' rounding)
  fp32:  2^-24 |y|
  both:  sum_p w_p |V_p| times (a weight's relative error in fp32 + 2 L 2^-24 for the two sums over L positions)."""
import numpy as np
import pytest
import torch

import paper_2510_23649_amd as L
import pages_plain as P
import test_gpu_pages as base
from test_gpu_pages import DEV, D, MARK, SETS, Case

pytestmark = pytest.mark.gpu
base.PAGE["e2m1"] = L.LRQK_PAGE_E2M1
KV = ["bf16", "f32"]
WAYS = {"one": (1, 40), "thin": (9, 75), "pair": (14, 75), "tile": (70, 150)}   # three heads a group


def make(seqs, Hkv=2, G=4, page=16, kv="bf16", **kw):
    return Case(seqs, Hkv, G, page, kv, "e2m1", **kw)


def set_code(c, name, pg, h, o, d, code):
    """Code of element d of a row, the other half of its byte as it was."""
    at = (pg, h, o, d // 2)
    c.pool[name][at] = (int(c.pool[name][at]) & (0xF0 if d % 2 == 0 else 0x0F)) | code << (4 * (d % 2))


# ---- codes -----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kv", KV)
def test_every_code_under_every_scale(kv):
    """16 codes times 256 scale bytes, read back; 255 is NaN, and what the type does not hold is an infinity."""
    c = make([(1, 64)], 4, 1, 64, kv, seed=1)
    code = np.arange(16, dtype=np.uint8)
    block = np.concatenate([code[0::2] | code[1::2] << 4, code[1::2] | code[0::2] << 4])   # 32 codes, all 16 twice
    for name in "KV":
        c.pool[name][:] = torch.from_numpy(np.tile(block, 4))
        c.sc[name][:] = torch.arange(c.sc[name].numel()).to(torch.uint8).view(c.sc[name].shape)
    assert c.sc["K"][c.table[0, 0]].unique().numel() == 256
    c.to_device()
    out = {n: torch.zeros((1, 4, 64, D), dtype=P.TYPE[kv], device=DEV) for n in "KV"}
    L.lrqk_pages_read(c.shape, c.pg, 0, out["K"], out["V"])
    for n in "KV":
        want = c.rows(n, 0)[0]
        big = float(torch.finfo(P.TYPE[kv]).max)
        want = np.where(np.abs(want) > big, np.copysign(np.inf, want), want)
        assert np.array_equal(out[n][0].double().cpu().numpy(), want, equal_nan=True), n


def blocks(kv, g):
    """Blocks of 32 elements at which a scale or a rounding can go wrong, as rows of 128 (four blocks a row)."""
    dt, big = P.TYPE[kv], float(torch.finfo(P.TYPE[kv]).max)
    up = lambda x, to: float(torch.nextafter(torch.tensor(x, dtype=dt), torch.tensor(to, dtype=dt)))  # noqa: E731
    one = lambda v, i=9: torch.randn(32, generator=g, dtype=torch.float64).index_fill_(0, torch.tensor(i), v)  # noqa: E731
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], dtype=torch.float64)
    near = torch.cat([ties, torch.tensor([up(float(t), 9.0) for t in ties]), torch.tensor([up(float(t), 0.0) for t in ties]), -ties,
                      torch.tensor([6.0, -6.0, -0.0, 5.5])])
    assert near.numel() == 32
    b = [torch.zeros(32), -torch.zeros(32), torch.full((32,), 3.0e38), torch.full((32,), 1.0e-30), torch.full((32,), 1.0e-40),
         torch.linspace(-6, 6, 32), near, near * 2.0 ** 60, near * 2.0 ** -100, -near * 2.0 ** -110, near * 2.0 ** -112, near * 2.0 ** 125,
         one(up(6.0, 9.0), 0), one(-up(6.0, 9.0)), one(up(6.0, 0.0)), one(3.0), one(up(3.0, 9.0), 31), one(6.0 * 2.0 ** -110),
         torch.full((32,), -6.0 * 2.0 ** -112), one(float("nan"), 3), one(float("inf")), one(-float("inf"), 31),
         torch.full((32,), big), -torch.full((32,), big), one(big), one(-big, 31), one(up(big, 0.0)),
         torch.linspace(-1, 1, 32, dtype=torch.float64) * big, torch.linspace(0.7, 1, 32, dtype=torch.float64) * big,
         one(1.5 * 2.0 ** 127), one(up(1.5 * 2.0 ** 127, big)), one(-1.75 * 2.0 ** 127), one(2.0 ** 127), one(1.25 * 2.0 ** 127)]
    b += [torch.randn(32, generator=g, dtype=torch.float64) for _ in range(-len(b) % 4)]
    return torch.stack([x.to(torch.float64) for x in b]).view(-1, D).to(dt)


def quantise(x):
    """P.quantise, but that no finite element becomes 4 * 2^126 = 2^128: the next lower code, 3 * 2^126."""
    code, byte = P.quantise(x, "e2m1")
    top = np.repeat(byte == 253, 16, axis=-1)
    lo, hi = code & 15, code >> 4
    lo, hi = (np.where(top & ((h & 7) == 6), h - 1, h) for h in (lo, hi))
    return (lo | hi << 4).astype(np.uint8), byte


@pytest.mark.parametrize("kv", KV)
@pytest.mark.parametrize("page,Hkv", [(16, 1), (4, 2), (64, 3)])
def test_special_blocks_are_written_and_read(page, Hkv, kv):
    x = blocks(kv, torch.Generator().manual_seed(7))
    n = -(-x.shape[0] // Hkv)
    c = make([(n, n + 5), (1, 3)], Hkv, 2, page, kv, seed=60, front=2, back=3)
    x = torch.cat([x, x[:n * Hkv - x.shape[0]]])
    c.k_new[2:2 + n] = x.view(n, Hkv, D)
    c.v_new[2:2 + n] = x.flip(0).view(n, Hkv, D)
    c.to_device()
    L.lrqk_pages_append(c.shape, c.pg, c.k_new.to(DEV), c.v_new.to(DEV))
    out = {a: torch.full((2, Hkv, n + 5, D), MARK, dtype=P.TYPE[kv], device=DEV) for a in "KV"}
    L.lrqk_pages_read(c.shape, c.pg, 0, out["K"], out["V"])
    for name, new in (("K", c.k_new), ("V", c.v_new)):
        code, byte = quantise(new[2:2 + n].double().numpy())
        at = [c.where(0, 5 + i) for i in range(n)]
        pg, off = [a[0] for a in at], [a[1] for a in at]
        assert np.array_equal(c.ds[name].cpu().numpy()[pg, :, off], byte), f"{name}: scales"
        assert np.array_equal(c.d[name].cpu().numpy()[pg, :, off], code), f"{name}: codes"
        got = out[name][0, :, 5:].transpose(0, 1).double().cpu().numpy()
        assert np.array_equal(got, P.values(code, byte, "e2m1"), equal_nan=True), f"{name}: values"
        fine = np.isfinite(new[2:2 + n].double().numpy().reshape(n, Hkv, 4, 32)).all(-1)
        assert np.isfinite(got.reshape(n, Hkv, 4, 32)).all(-1)[fine].all(), f"{name}: a finite element is read as an infinity"


@pytest.mark.parametrize("kv", KV)
@pytest.mark.parametrize("seqs", [[(1, 1)], [(1, 40), (1, 7), (1, 16)], [(70, 100), (0, 9), (33, 33), (5, 3)]], ids=["one", "step", "chunk"])
def test_append(seqs, kv):
    """What is written, and nothing beside it: rows of no token keep what they hold."""
    for page, Hkv in ((16, 2), (1, 3), (256, 1)):
        c = make(seqs, Hkv, 2, page, kv, seed=20, front=2, back=3, holes=0.1 if len(seqs) > 2 else 0.0).to_device()
        L.lrqk_pages_append(c.shape, c.pg, c.k_new.to(DEV), c.v_new.to(DEV))
        c.append_plain()
        for name in "KV":
            assert torch.equal(c.ds[name].cpu(), c.sc[name]) and torch.equal(c.d[name].cpu(), c.pool[name]), name


@pytest.mark.parametrize("kv", KV)
@pytest.mark.parametrize("first", [0, 50, 1000])
def test_read(first, kv):
    c = make([(1, 120), (0, 0), (1, 51), (2, 300)], 2, 2, 16, kv, seed=21, holes=0.15, l_max=290, l_cap=301).to_device()
    dev = lambda: torch.full((c.B, c.Hkv, 301, D), MARK, dtype=P.TYPE[kv], device=DEV)  # noqa: E731
    K, V, Kp = dev(), dev(), torch.full((c.B, c.Hkv, 301, D), MARK, dtype=P.TYPE[kv]).pin_memory()
    L.lrqk_pages_read(c.shape, c.pg, first, K, V)
    L.lrqk_pages_read(c.shape, c.pg, first, Kp, None)
    torch.cuda.synchronize()
    assert torch.equal(K.cpu(), Kp)
    for name, got in (("K", K.cpu()), ("V", V.cpu())):
        for b in range(c.B):
            ref, there = c.rows(name, b)
            want = np.full((c.Hkv, 301, D), MARK)
            for p in range(first, len(there)):
                if there[p]:
                    want[:, p] = ref[:, p]
            assert np.array_equal(got[b].double().numpy(), want), f"{name} of sequence {b}"


# ---- attention ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kv", KV)
@pytest.mark.parametrize("name", SETS)
def test_attend(name, kv):
    for j in range(3):                       # pages from one position to 1024, groups from one head to eight
        i = list(SETS).index(name) + 8 * KV.index(kv) + 5 * j
        Hkv, G = [(2, 4), (1, 1), (2, 3), (1, 5), (2, 7), (1, 8), (3, 2)][i % 7]
        c = make(SETS[name], Hkv, G, [16, 1, 64, 256, 32, 1024, 2][(i // 2) % 7], kv, seed=i, front=i % 3, back=i % 4).to_device()
        c.check_attend(c.attend())


@pytest.mark.parametrize("kv", KV)
@pytest.mark.parametrize("Hkv,G", [(1, 1), (1, 2), (2, 3), (1, 4), (3, 5), (1, 6), (4, 7), (8, 8)])
def test_groups(Hkv, G, kv):
    c = make([(1, 200), (2, 33), (9, 77), (70, 130)], Hkv, G, 16, kv, seed=G).to_device()
    c.check_attend(c.attend())
    c = make([(1, 200), (1, 1), (1, 77), (2, 130)], Hkv, G, 32, kv, seed=G + 10).to_device()
    c.check_attend(c.attend())


@pytest.mark.parametrize("kv", KV)
def test_split_over_the_context(kv):
    for seqs in ([(1, 9001), (1, 3), (2, 4096), (0, 7)], [(1, 2049)], [(1, 20001), (1, 70)]):
        c = make(seqs, 2, 4, 64, kv, seed=5).to_device()
        c.check_attend(c.attend())


@pytest.mark.parametrize("kv", KV)
@pytest.mark.parametrize("seqs", [[(1, 3000), (1, 500)], [(5, 3000), (1, 500)], [(12, 900), (1, 500)], [(90, 400), (4, 600)]],
                         ids=["one", "few", "pair", "chunk"])
def test_missing_pages(seqs, kv):
    """Positions on missing pages take no part; a token that sees none gets zeros."""
    c = make(seqs, 2, 4, 16, kv, seed=8, holes=0.5)
    c.table[1, :] = -1
    c.table[0, :3] = -1
    c.poison(np.ones((c.n_pages, c.page), bool) & ~np.isin(np.arange(c.n_pages), c.table)[:, None])
    c.to_device()
    c.check_attend(c.attend())


@pytest.mark.parametrize("kv", KV)
@pytest.mark.parametrize("way", WAYS)
def test_what_a_token_does_not_see_does_not_reach_it(way, kv):
    """Blocks that are NaN in K and V rows of later tokens, infinities in V rows of some, under scales from elsewhere."""
    n, ln = WAYS[way]
    c = make([(n, ln), (2, 40)], 2, 3, 16, kv, seed=n)
    pg, o = c.where(0, ln - 1)
    if n > 1:
        c.sc["K"][pg, 0, o, 1] = 255
        c.sc["V"][pg, 0, o, 2] = 255
    for p, h, d, code in ((ln - 1, 1, 5, 7), (ln - max(1, n // 2), 0, 41, 15), (ln - n, 0, 70, 6), (2, 1, 100, 14)):
        pg, o = c.where(0, p)                # +-4 or 6 times 2^127 among zeros
        c.pool["V"][pg, h, o, d // 32 * 16:d // 32 * 16 + 16] = 0
        set_code(c, "V", pg, h, o, d, code)
        c.sc["V"][pg, h, o, d // 32] = 254
    rows, big = c.rows, float(torch.finfo(torch.float32).max)

    def as_held(name, b):
        x, there = rows(name, b)
        return np.where(np.abs(x) > big, np.copysign(np.inf, x), x), there

    c.rows = as_held
    c.to_device()
    c.check_attend(c.attend())


@pytest.mark.parametrize("kv", KV)
@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0, 1e-4])
def test_scales(kv, scale):
    c = make([(1, 300), (3, 70), (40, 90)], 2, 4, 16, kv, seed=4, scale=scale).to_device()
    c.check_attend(c.attend())
    c = make([(1, 300), (1, 70), (2, 90)], 2, 4, 16, kv, seed=5, scale=scale).to_device()
    c.check_attend(c.attend())


@pytest.mark.parametrize("kv", KV)
@pytest.mark.parametrize("way", WAYS)
def test_weights_that_differ_widely(way, kv):
    """Scores that grow along the context by thousands, fall, or are huge: every block moves the maximum, or none."""
    n, ln = WAYS[way]
    for grows in (True, False):
        c = make([(n, ln), (1, 33)], 1, 3, 16, kv, seed=6)
        for b in range(2):
            for p in range(int(c.len[b])):   # 0.5 .. 6 times 2^e: grows with p
                pg, o = c.where(b, p)
                x = p if grows else int(c.len[b]) - 1 - p
                c.pool["K"][pg, :, o, :16] = 0
                set_code(c, "K", pg, 0, o, 0, 4 + x % 4)
                c.sc["K"][pg, :, o, 0] = 127 + x // 16
        c.q[..., 0] = 4.0
        c.to_device()
        c.check_attend(c.attend())


@pytest.mark.parametrize("kv", KV)
@pytest.mark.parametrize("way", WAYS)
def test_huge_scores_all_alike(way, kv):
    """Scores of 6 times a power of two, all alike: every weight is exactly 1 and the output the mean of what is seen, off by its own
    rounding, those of the two sums over L positions and two for the quotient."""
    n, ln = WAYS[way]
    c = make([(n, ln)], 1, 3, 16, kv, seed=65)
    c.q[..., 0], c.q[..., 1:] = 1.0, 0.0
    c.pool["K"][:] = 0
    V, _ = c.rows("V", 0)
    many = np.arange(ln - n, ln)[:, None] + 1.0
    y, mass = (np.cumsum(x, 0)[ln - n:, None] / many[:, None] for x in (V[0], np.abs(V[0])))
    tol = (2.0 ** -8 if kv == "bf16" else 2.0 ** -24) * np.abs(y) + mass * (2 * ln + 2) * 2.0 ** -24
    c.to_device()
    for code, byte in ((15, 252), (7, 252), (15, 220), (7, 160), (15, 145)):
        c.d["K"][..., 0] = code
        c.ds["K"][..., 0] = byte
        got = c.attend().double().cpu().numpy()
        assert (np.abs(got - y) <= tol).all(), (code, byte, np.abs(got - y).max())


@pytest.mark.parametrize("kv", KV)
@pytest.mark.parametrize("way", WAYS)
def test_queries_of_every_size(way, kv):
    """Blocks of q of very different size, those of K the other way round: every block counts for the score, in all its bits."""
    n, ln = WAYS[way]
    c = make([(n, ln), (1, 33)], 1, 3, 16, kv, seed=67, qs=1.0)
    for b, e in enumerate((-60, -20, 25, 70)):
        c.q[..., 32 * b:32 * b + 32] *= 2.0 ** e
        c.sc["K"][..., b] = (c.sc["K"][..., b].int() - e).to(torch.uint8)
    c.poison(np.ones((c.n_pages, c.page), bool) & ~np.isin(np.arange(c.n_pages), c.table)[:, None])
    c.to_device()
    c.check_attend(c.attend())


@pytest.mark.parametrize("kv", KV)
@pytest.mark.parametrize("way", WAYS)
def test_queries_that_are_no_numbers(way, kv):
    """NaN and infinities in q reach their own head and token alone; scores of -infinity alone give zeros."""
    n, ln = WAYS[way]
    c = make([(n, ln), (1, 33)], 1, 3, 16, kv, seed=68)
    low_nan = torch.tensor([0x7F800001], dtype=torch.int32).view(torch.float32)[0].to(P.TYPE[kv])   # (fp32: its upper half is an infinity)
    bad = [(0, 0, float("nan")), (n - 1, 1, low_nan if kv == "f32" else float("nan")), (n, 2, float("inf")), (n, 0, -float("inf")), (0, 2, 3.0e38)]
    clean = c.q.clone()
    for t, h, v in bad:
        c.q[t, h, 7] = v
    for p in range(int(c.len[1])):                           # sequence 1: -1 in K's element 7 under both infinities
        pg, o = c.where(1, p)
        set_code(c, "K", pg, 0, o, 7, 10)
        c.sc["K"][pg, 0, o, 0] = 127
    c.to_device()
    got = c.attend()
    assert torch.isnan(got[0, 0]).all() and torch.isnan(got[n - 1, 1]).all()
    assert (got[n, 2] == 0).all(), "infinity times -1: scores of -infinity alone"
    assert torch.isnan(got[n, 0]).all(), "scores of +infinity"
    # (3.0e38 times a K of 1.5 and more is beyond fp32: that token and head may be anything, the others not)
    c.q = clean
    want = c.attend()
    same = torch.ones_like(got, dtype=torch.bool)
    for t, h, _ in bad:
        same[t, h] = False
    # the others within the bound: rows that share a wavefront have their maxima raised together, so that their roundings may differ
    c.check_attend(want)
    c.check_attend(torch.where(same, got, want))


def test_n_max_only_chooses_the_kernel():
    for seqs in ([(1, 700), (1, 90)], [(4, 300), (1, 900)], [(30, 300), (64, 64)]):
        for n_max in (1, 2, 4, 8, 16, 40, 1000):
            c = make(seqs, 2, 4, 16, "bf16", seed=13, n_max=n_max).to_device()
            c.check_attend(c.attend())


def test_many_and_uneven_sequences():
    """More sequences than a wavefront has lanes; one long one among short ones, empty ones and ones without new tokens."""
    rng = np.random.default_rng(14)
    for kv in KV:
        for n in (1, 3, 12):
            seqs = [(int(rng.integers(0, n + 1)), int(rng.integers(0, 100))) for _ in range(149)] + [(n, 5000)]
            c = make([seqs[i] for i in rng.permutation(150)], 1, 4, 16, kv, seed=15, n_max=n).to_device()
            c.check_attend(c.attend())


@pytest.mark.parametrize("B,kv", [(2048, "f32"), (2049, "f32"), (2049, "bf16"), (4200, "bf16")])
def test_thousands_of_sequences(B, kv):
    rng = np.random.default_rng(B)
    seqs = [(int(rng.integers(0, 3)), int(rng.integers(2, 25))) for _ in range(B - 1)] + [(2, 700)]
    c = make([seqs[i] for i in rng.permutation(B)], 1, 2, 16, kv, seed=17).to_device()
    c.check_attend(c.attend())


def test_shared_pages():
    for kv in KV:
        c = make([(3, 100), (40, 90), (1, 60)], 2, 4, 16, kv, seed=12)
        c.table[1, :3] = c.table[0, :3]
        c.table[2, :2] = c.table[0, :2]
        c.to_device()
        c.check_attend(c.attend())


def test_offsets_beyond_32_bits():
    """A pool of more than 2^32 bytes (2^33 elements) of K, its last pages in use."""
    page, Hkv = 64, 8
    n_pages = (1 << 32) // (page * Hkv * D // 2) + 40
    small = make([(1, 500), (20, 130)], Hkv, 2, page, seed=15, spare=0)
    shift = n_pages - small.n_pages
    small.to_device()
    want = small.attend()
    small.check_attend(want)
    one = make([(1, 500), (1, 130)], Hkv, 2, page, seed=16, spare=0)
    assert one.n_pages == small.n_pages
    one.to_device()
    want1 = one.attend()
    one.check_attend(want1)
    big = {n: torch.zeros((n_pages, Hkv, page, D // 2), dtype=torch.uint8, device=DEV) for n in "KV"}
    bs = {n: torch.zeros((n_pages, Hkv, page, 4), dtype=torch.uint8, device=DEV) for n in "KV"}
    for c, w in ((one, want1), (small, want)):
        for n in "KV":
            big[n][shift:] = c.d[n]
            bs[n][shift:] = c.ds[n]
        table = torch.where(c.dtable >= 0, c.dtable + shift, c.dtable)
        c.shape.n_pages = n_pages
        c.pg = L.make_pages(K=big["K"], V=big["V"], K_scale=bs["K"], V_scale=bs["V"], table=table, start=c.dstart, kv_len=c.dlen)
        assert torch.equal(c.attend(), w)
    out = {n: torch.zeros((2, Hkv, small.l_max, D), dtype=torch.bfloat16, device=DEV) for n in "KV"}
    L.lrqk_pages_append(small.shape, small.pg, small.k_new.to(DEV), small.v_new.to(DEV))
    L.lrqk_pages_read(small.shape, small.pg, 0, out["K"], out["V"])
    small.append_plain()
    for b in range(2):
        for name in "KV":
            ref, _ = small.rows(name, b)
            assert np.array_equal(out[name][b, :, :small.len[b]].double().cpu().numpy(), ref)


def exact_on_device(c, b):
    """What check_attend compares with, for sequence b, in float64 on the GPU: for long contexts."""
    lo, hi = int(c.start[b]), int(c.start[b + 1])
    n, Ln = hi - lo, min(int(c.len[b]), c.l_max)
    p = torch.arange(Ln, device=DEV)
    pg = c.dtable[b, p // c.page].long()
    there = (pg >= 0) & (pg < c.n_pages)
    pg = pg.clamp(0, c.n_pages - 1)
    steps = torch.from_numpy(np.concatenate([P.STEPS, -P.STEPS])).to(DEV)

    def rows(name):
        x = c.d[name][pg, :, p % c.page]
        x = steps[torch.stack((x & 15, x >> 4), -1).flatten(-2).long()]
        x = x * torch.exp2(c.ds[name][pg, :, p % c.page].double() - 127).repeat_interleave(32, dim=-1)
        return torch.where(there[:, None, None], x, 0.0).transpose(0, 1)

    K, V, q = rows("K"), rows("V"), c.q[lo:hi].to(DEV).double()
    pos = int(c.len[b]) - n + torch.arange(n, device=DEV)
    hidden = (p[None, :] > pos[:, None]) | ~there[None, :]
    y, mass, slack = (torch.zeros(n, c.Hq, D, dtype=torch.float64, device=DEV) for _ in range(3))
    for h in range(c.Hq):
        k, v = K[h // c.G], V[h // c.G]
        s = (q[:, h] @ k.t()) * float(np.float32(c.scale))
        s[hidden] = -float("inf")
        w = torch.softmax(s, 1)
        y[:, h], mass[:, h] = w @ v, w @ v.abs()
        near = torch.where(s >= s.amax(1, keepdim=True) - 100, (q[:, h].abs() @ k.abs().t()) * abs(c.scale) * 130 + 3 * s.abs() + 4, 0.0)
        slack[:, h] = (2 * near.amax(1) * 2.0 ** -24)[:, None]
    return y, mass, slack, Ln


@pytest.mark.parametrize("kv", KV)
@pytest.mark.parametrize("seqs", [[(300, 20000)], [(1, 70001), (1, 300), (1, 33000)], [(1, 131072)], [(3, 40000), (1, 20000)],
                                  [(12, 30000), (3, 9000)], [(20, 40000)], [(700, 9000), (1, 40000), (2, 17000)]],
                         ids=["chunk", "ones", "one", "few", "pair", "tile", "mixed"])
def test_long_contexts(seqs, kv):
    """Many pieces for every shape of workgroup, some of the pages missing."""
    c = make(seqs, 2, 4, 64, kv, seed=50, holes=0.05).to_device()
    out = c.attend().double()
    for b in range(c.B):
        y, mass, slack, Ln = exact_on_device(c, b)
        half = 2.0 ** -8 if kv == "bf16" else 2.0 ** -24
        tol = half * y.abs() + mass * (slack + 2 * Ln * 2.0 ** -24 + (2.0 ** -8 if kv == "bf16" else 0.0))
        far = (out[int(c.start[b]):int(c.start[b + 1])] - y).abs() - tol
        assert float(far.max()) <= 0, f"sequence {b}: off by {float(far.max())} more than the bound"


def test_same_call_twice_is_the_same():
    for seqs in ([(1, 5000), (1, 300)], [(1, 5000)], [(200, 700), (3, 50)]):
        for kv in KV:
            c = make(seqs, 2, 4, 16, kv, seed=16).to_device()
            assert torch.equal(c.attend(), c.attend())


# ---- together ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kv", KV)
def test_prompt_in_chunks(kv):
    """A prompt runs through in chunks, each written and attended, and then a token at a time."""
    Hkv, G, l, page, dt = 2, 4, 203, 16, P.TYPE[kv]
    c = make([(0, l)], Hkv, G, page, kv, seed=30, spare=3)
    g = torch.Generator().manual_seed(31)
    k, v = (torch.randn(l, Hkv, D, generator=g).to(dt) for _ in range(2))
    q = (1.5 * torch.randn(l, Hkv * G, D, generator=g)).to(dt)
    c.poison(np.ones((c.n_pages, page), bool))
    c.to_device()
    at, outs = 0, []
    for n in (100, 1, 64, 12, 5, 20, 1):
        c.dstart.copy_(torch.tensor([0, n], dtype=torch.int32))
        c.dlen.copy_(torch.tensor([at + n], dtype=torch.int32))
        s = L.PagesShape.make(B=1, Hq=Hkv * G, Hkv=Hkv, T=n, n_max=n, l_max=l, page=page, n_pages=c.n_pages, max_pages=c.max_pages,
                              kv_dtype=base.KV[kv], page_dtype=L.LRQK_PAGE_E2M1)
        out = torch.empty((n, Hkv * G, D), dtype=dt, device=DEV)
        ws = torch.empty(L.lrqk_pages_workspace_bytes(s), dtype=torch.uint8, device=DEV)
        L.lrqk_pages_append(s, c.pg, k[at:at + n].to(DEV), v[at:at + n].to(DEV))
        L.lrqk_chunk_attend(s, c.pg, q[at:at + n].to(DEV), out, ws)
        outs.append(out)
        at += n
    assert at == l
    c.seqs, c.T, c.start, c.len = [(l, l)], l, np.array([0, l], np.int32), np.array([l], np.int32)
    c.k_new, c.v_new, c.q = k, v, q
    c.append_plain()
    c.check_attend(torch.cat(outs))


@pytest.mark.parametrize("kv", KV)
def test_captured_and_replayed(kv):
    """append, attend and read of a graph follow the lengths and tables that the memory holds at each replay; unreached rows
    hold NaN."""
    c = make([(1, 900), (1, 900), (1, 900)], 2, 4, 16, kv, seed=42).to_device()
    dt = P.TYPE[kv]
    bits = lambda x: x.view(torch.int16 if kv == "bf16" else torch.int32)  # noqa: E731
    q, k, v = c.q.to(DEV), c.k_new.to(DEV), c.v_new.to(DEV)
    out = torch.zeros((c.T, c.Hq, D), dtype=dt, device=DEV)
    K = torch.zeros((c.B, c.Hkv, c.l_max, D), dtype=dt, device=DEV)
    V = torch.zeros_like(K)

    def step(o, ws):
        L.lrqk_pages_append(c.shape, c.pg, k, v)
        L.lrqk_chunk_attend(c.shape, c.pg, q, o, ws)
        L.lrqk_pages_read(c.shape, c.pg, 0, K, V)

    step(out, c.ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(out, c.ws)
    other = torch.empty_like(c.ws)
    gen = torch.Generator().manual_seed(43)
    for lens in ([900, 1, 30], [2, 899, 450], [64, 65, 0], [1, 1, 1]):
        c.dlen.copy_(torch.tensor(lens, dtype=torch.int32))
        c.dtable[:, :57] = c.dtable[:, torch.randperm(57, generator=gen).to(DEV)]
        q.copy_((1.5 * torch.randn(q.shape, generator=gen)).to(dt))
        k.copy_(torch.randn(k.shape, generator=gen).to(dt))
        K.zero_()
        V.zero_()
        g.replay()
        torch.cuda.synchronize()
        got = out.clone(), K.clone(), V.clone()
        K.zero_()
        V.zero_()
        want = torch.zeros_like(out)
        step(want, other)
        torch.cuda.synchronize()
        assert all(torch.equal(bits(x), bits(y)) for x, y in zip(got, (want, K, V))), lens

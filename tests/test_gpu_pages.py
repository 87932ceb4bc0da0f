"""GPU tests of the paged cache: lrqk_pages_append, lrqk_pages_read, lrqk_chunk_attend against plain float64
(tests/pages_plain.py).  Rows and scales are compared bit for bit.  An attention's output may be off by

  bf16:  2^-8 |y| (its own rounding) + 2^-8 sum_p w_p |V_p| (the weights' rounding)
  fp32:  2^-24 |y|
  both:  sum_p w_p |V_p| times (a weight's relative error in fp32 + 2 L 2^-24 for the two sums over L positions)

(half a step of bf16 is 2^-8 relative, of fp32 2^-24; bounds of the worst case)."""
import numpy as np
import pytest
import torch

import paper_2510_23649_amd as L
import pages_plain as P

pytestmark = pytest.mark.gpu
DEV = "cuda"
D = 128
KINDS = [("bf16", "bf16"), ("f32", "f32"), ("bf16", "e4m3"), ("bf16", "i8"), ("f32", "e4m3"), ("f32", "i8")]
KV = {"bf16": L.LRQK_KV_BF16, "f32": L.LRQK_KV_F32}
PAGE = {"bf16": L.LRQK_PAGE_BF16, "f32": L.LRQK_PAGE_F32, "e4m3": L.LRQK_PAGE_E4M3, "i8": L.LRQK_PAGE_I8}
MARK = -77.0                                 # what output rows hold that nothing may touch


class Case:
    """Sequences [(new tokens, length), ...] on shuffled pages; unreached rows hold NaN."""

    def __init__(self, seqs, Hkv=2, G=4, page=16, kv="bf16", pages="bf16", seed=0, front=0, back=0, holes=0.0,
                 l_max=None, scale=None, qs=1.5, l_cap=0, n_max=None, spare=2):
        self.seqs, self.Hkv, self.G, self.page, self.kv, self.pages = seqs, Hkv, G, page, kv, pages
        self.rng = rng = np.random.default_rng(seed)
        self.g = torch.Generator().manual_seed(seed)
        self.l_max = l_max or max(1, max(x for _, x in seqs))
        self.B, self.Hq = len(seqs), Hkv * G
        self.T = max(1, front + sum(n for n, _ in seqs) + back)
        self.start = front + np.concatenate([[0], np.cumsum([n for n, _ in seqs])]).astype(np.int32)
        self.len = np.array([x for _, x in seqs], np.int32)
        self.max_pages = -(-self.l_max // page) + 1
        used = [min(-(-x // page), self.max_pages) for _, x in seqs]
        self.n_pages = sum(used) + spare
        ids = rng.permutation(self.n_pages)
        self.table = np.full((self.B, self.max_pages), -1, np.int32)
        at = 0
        for b, u in enumerate(used):
            self.table[b, :u] = ids[at:at + u]
            at += u
        if holes:
            miss = rng.random(self.table.shape) < holes
            self.table = np.where(miss, rng.choice([-1, self.n_pages, -2**31, 2**31 - 1], self.table.shape), self.table).astype(np.int32)
        self.scale = D ** -0.5 if scale is None else scale
        self.shape = L.PagesShape.make(B=self.B, Hq=self.Hq, Hkv=Hkv, T=self.T, n_max=n_max or max(1, max(n for n, _ in seqs)),
                                       l_max=self.l_max, l_cap=l_cap, page=page, n_pages=self.n_pages, max_pages=self.max_pages,
                                       kv_dtype=KV[kv], page_dtype=PAGE[pages], scale=self.scale)
        dt = P.TYPE[kv]
        self.q = (qs * torch.randn(self.T, self.Hq, D, generator=self.g)).to(dt)
        self.k_new = torch.randn(self.T, Hkv, D, generator=self.g).to(dt)
        self.v_new = torch.randn(self.T, Hkv, D, generator=self.g).to(dt)
        # the rows of the sequences before their new tokens, and NaN wherever no position reaches
        self.pool, self.sc = {}, {}
        for name in "KV":
            x = torch.randn(self.n_pages, Hkv, page, D, generator=self.g)
            if pages in P.TYPE:
                self.pool[name] = x.to(P.TYPE[pages])
                self.sc[name] = None
            else:
                code, byte = P.quantise(x.to(dt).double().numpy(), pages)
                self.pool[name], self.sc[name] = torch.from_numpy(code), torch.from_numpy(byte)
        reached = np.zeros((self.n_pages, page), bool)
        for b in range(self.B):
            for p in range(min(int(self.len[b]), self.l_max)):
                pg = self.table[b, p // page]
                if 0 <= pg < self.n_pages:
                    reached[pg, p % page] = True
        self.poison(~reached)

    def poison(self, rows):
        rows = torch.from_numpy(rows)[:, None, :].expand(-1, self.Hkv, -1)
        for name in "KV":
            if self.sc[name] is None:
                self.pool[name][rows] = float("nan")
            else:
                self.pool[name][rows] = 0x7F
                self.sc[name][rows] = 255

    def to_device(self):
        self.d = {n: self.pool[n].to(DEV) for n in "KV"}
        self.ds = {n: None if self.sc[n] is None else self.sc[n].to(DEV) for n in "KV"}
        self.dtable, self.dstart = torch.from_numpy(self.table).to(DEV), torch.from_numpy(self.start).to(DEV)
        self.dlen = torch.from_numpy(self.len).to(DEV)
        self.pg = L.make_pages(K=self.d["K"], V=self.d["V"], K_scale=self.ds["K"], V_scale=self.ds["V"], table=self.dtable,
                               start=self.dstart, kv_len=self.dlen)
        self.ws = torch.full((L.lrqk_pages_workspace_bytes(self.shape),), 0xFF, dtype=torch.uint8, device=DEV)
        return self

    def where(self, b, p):
        """Row (page, offset) of position p of sequence b, or None."""
        if not 0 <= p < self.l_max:
            return None
        pg = int(self.table[b, p // self.page])
        return (pg, p % self.page) if 0 <= pg < self.n_pages else None

    def rows(self, name, b):
        """float64 rows [Hkv, L, D] of sequence b and which of them are there."""
        Ln = max(0, min(int(self.len[b]), self.l_max))
        x, there = np.zeros((self.Hkv, Ln, D)), np.zeros(Ln, bool)
        pool = self.pool[name]
        whole = pool.double().numpy() if self.sc[name] is None else None
        for p in range(Ln):
            at = self.where(b, p)
            if at:
                there[p] = True
                if whole is not None:
                    x[:, p] = whole[at[0], :, at[1]]
                else:
                    x[:, p] = P.values(pool[at[0], :, at[1]].numpy(), self.sc[name][at[0], :, at[1]].numpy(), self.pages)
        return x, there

    def append_plain(self):
        """The pools after the new tokens were written."""
        for name, new in (("K", self.k_new), ("V", self.v_new)):
            for b in range(self.B):
                n = int(self.start[b + 1] - self.start[b])
                for i in range(n):
                    at = self.where(b, int(self.len[b]) - n + i)
                    if at is None:
                        continue
                    row = new[int(self.start[b]) + i]
                    if self.sc[name] is None:
                        self.pool[name][at[0], :, at[1]] = row
                    else:
                        code, byte = P.quantise(row.double().numpy(), self.pages)
                        self.pool[name][at[0], :, at[1]] = torch.from_numpy(code)
                        self.sc[name][at[0], :, at[1]] = torch.from_numpy(byte)

    def attend(self, stream=None):
        out = torch.full((self.T, self.Hq, D), MARK, dtype=P.TYPE[self.kv], device=DEV)
        L.lrqk_chunk_attend(self.shape, self.pg, self.q.to(DEV), out, self.ws, stream)
        return out

    def check_attend(self, out):
        got = out.double().cpu().numpy()
        untouched = np.ones(self.T, bool)
        for b in range(self.B):
            lo, hi = int(self.start[b]), int(self.start[b + 1])
            untouched[lo:hi] = False
            if lo == hi:
                continue
            K, there = self.rows("K", b)
            V, _ = self.rows("V", b)
            pos = int(self.len[b]) - (hi - lo) + np.arange(hi - lo)
            y, mass, slack = P.attend(self.q[lo:hi].double().numpy(), K, V, there, pos, float(np.float32(self.scale)))
            half = 2.0 ** -8 if self.kv == "bf16" else 2.0 ** -24
            tol = half * np.abs(y) + mass * (slack[..., None] + 2 * K.shape[1] * 2.0 ** -24 + (2.0 ** -8 if self.kv == "bf16" else 0.0)) + 1e-30
            g = got[lo:hi]
            assert np.array_equal(np.isnan(g), np.isnan(y)), f"sequence {b}: NaN where there is none, or none where there is"
            inf = np.isinf(y)
            assert np.array_equal(g[inf], y[inf]), f"sequence {b}: infinities"
            fine = np.isfinite(y)
            far = np.where(fine, np.abs(np.where(fine, g, 0) - np.where(fine, y, 0)), 0) - np.where(fine, tol, 0)
            assert far.max() <= 0, f"sequence {b}: off by {far.max()} more than the bound at {np.unravel_index(far.argmax(), far.shape)}"
        assert (got[untouched] == MARK).all(), "a row of no sequence was written"


SETS = {
    "single": [(1, 1)],
    "edges": [(1, 31), (1, 32), (1, 33), (1, 64), (1, 65), (1, 128), (1, 129)],
    "ragged_one": [(1, 700), (1, 2), (0, 50), (1, 1300), (1, 17)],
    "drafts": [(5, 300), (0, 40), (2, 2), (16, 257), (8, 8)],
    "chunks": [(100, 100), (33, 500), (1, 31), (129, 193), (0, 0), (64, 640)],
    "long_chunk": [(300, 900)],
    "before_the_context": [(10, 4), (3, 0), (40, 20), (1, 0)],
}


@pytest.mark.parametrize("kv,pages", KINDS)
@pytest.mark.parametrize("name", SETS)
def test_attend(name, kv, pages):
    i = list(SETS).index(name) + 7 * KINDS.index((kv, pages))
    Hkv, G = [(2, 4), (1, 1), (2, 3), (1, 5), (2, 7), (1, 8), (3, 2)][i % 7]
    c = Case(SETS[name], Hkv, G, [16, 1, 64, 256, 32, 1024, 2][(i // 2) % 7], kv, pages, seed=i, front=i % 3, back=i % 4).to_device()
    c.check_attend(c.attend())


@pytest.mark.parametrize("Hkv,G", [(1, 1), (1, 2), (2, 3), (1, 4), (3, 5), (1, 6), (4, 7), (8, 8)])
def test_attend_groups(Hkv, G):
    for kv, pages in (("bf16", "bf16"), ("f32", "f32")):
        c = Case([(1, 200), (9, 77), (70, 130)], Hkv, G, 16, kv, pages, seed=G).to_device()
        c.check_attend(c.attend())


@pytest.mark.parametrize("kv,pages", KINDS)
def test_attend_split_over_the_context(kv, pages):
    """Few rows and a long context: the work is split along it and joined; other sequences are short."""
    c = Case([(1, 9001), (1, 3), (2, 4096), (0, 7)], 2, 4, 64, kv, pages, seed=5).to_device()
    c.check_attend(c.attend())


@pytest.mark.parametrize("kv,pages", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "e4m3"), ("f32", "i8")])
@pytest.mark.parametrize("seqs", [[(1, 3000), (1, 500)], [(90, 400), (4, 600)]], ids=["one", "chunk"])
def test_attend_missing_pages(seqs, kv, pages):
    """Positions on missing pages take no part; a token that sees none gets zeros."""
    c = Case(seqs, 2, 4, 16, kv, pages, seed=8, holes=0.5)
    c.table[1, :] = -1
    c.table[0, :3] = -1
    c.poison(np.ones((c.n_pages, c.page), bool) & ~np.isin(np.arange(c.n_pages), c.table)[:, None])
    c.to_device()
    c.check_attend(c.attend())


@pytest.mark.parametrize("kv,pages", [("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("n,ln", [(1, 200), (6, 70), (150, 150), (200, 900)])
def test_what_a_token_does_not_see_does_not_reach_it(n, ln, kv, pages):
    """Infinities and NaN in K and V rows of later tokens, and in V rows of earlier ones."""
    c = Case([(n, ln), (2, 40)], 2, 3, 16, kv, pages, seed=n)
    some = np.random.default_rng(n).integers(ln - n, ln, 3) if n > 1 else []
    for j, p in enumerate(some):
        pg, o = c.where(0, int(p))
        c.pool["V"][pg, 0, o, 5 + j] = [float("inf"), float("-inf"), float("nan")][j % 3]
        if j == 2 and p > ln - n:
            c.pool["K"][pg, 1, o, 3] = float("nan")
    pg, o = c.where(0, max(0, ln - n - 1))
    c.pool["V"][pg, 1, o, 100] = float("inf")
    c.to_device()
    c.check_attend(c.attend())


@pytest.mark.parametrize("kv", ["bf16", "f32"])
def test_positions_beyond_l_max_do_not_exist(kv):
    c = Case([(20, 150), (3, 90), (1, 400)], 2, 4, 16, kv, kv, seed=3, l_max=100).to_device()
    c.check_attend(c.attend())


@pytest.mark.parametrize("kv", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0, 1e-4])
def test_scales(kv, scale):
    c = Case([(1, 300), (40, 90)], 2, 4, 16, kv, kv, seed=4, scale=scale).to_device()
    c.check_attend(c.attend())


@pytest.mark.parametrize("kv", ["bf16", "f32"])
@pytest.mark.parametrize("grows", [True, False])
def test_weights_that_differ_widely(kv, grows):
    """Scores that grow (or fall) along the context by thousands: every tile moves the maximum, or none."""
    c = Case([(1, 500), (40, 300)], 1, 4, 16, kv, kv, seed=6)
    for b in range(2):
        for p in range(int(c.len[b])):
            pg, o = c.where(b, p)
            c.pool["K"][pg, :, o, 0] = (p if grows else -p) * 8.0
    c.q[..., 0] = 4.0
    c.to_device()
    c.check_attend(c.attend())


def test_scores_of_the_lowest_value():
    """Scores down to the largest negative number, and of -infinity, beside ordinary ones."""
    c = Case([(1, 100), (30, 90)], 1, 2, 16, "f32", "f32", seed=9)
    c.q[..., 0] = 1.0
    for b, p, v in ((0, 7, -3.0e38), (0, 60, -float("inf")), (1, 3, -3.0e38), (1, 80, -float("inf"))):
        pg, o = c.where(b, p)
        c.pool["K"][pg, :, o, 1:] = 0.0
        c.pool["K"][pg, :, o, 0] = v
    c.to_device()
    c.check_attend(c.attend())


def test_a_token_with_scores_of_minus_infinity_alone_gets_zeros():
    for seqs in ([(1, 40)], [(70, 90)]):
        c = Case(seqs, 1, 4, 16, "f32", "f32", seed=10)
        c.q[..., 0], c.q[..., 1:] = 1.0, 0.0
        c.pool["K"][..., 0] = -float("inf")
        c.to_device()
        assert (c.attend() == 0).all()


@pytest.mark.parametrize("kv,pages", KINDS)
def test_shared_pages(kv, pages):
    """Two sequences with a common prefix on the same pages."""
    c = Case([(3, 100), (40, 90)], 2, 4, 16, kv, pages, seed=12)
    c.table[1, :3] = c.table[0, :3]
    c.to_device()
    c.check_attend(c.attend())


def test_n_max_only_chooses_the_kernel():
    for seqs in ([(1, 700), (1, 90)], [(4, 300), (1, 900)], [(30, 300), (64, 64)]):
        for n_max in (1, 8, 16, 40, 1000):
            c = Case(seqs, 2, 4, 16, "bf16", "bf16", seed=13, n_max=n_max).to_device()
            c.check_attend(c.attend())


@pytest.mark.parametrize("seqs", [[(1, 700), (1, 90)], [(12, 1300), (2, 40)], [(60, 700), (1, 300)]], ids=["ones", "pair", "tile"])
def test_l_max_far_above_the_lengths(seqs):
    """A call may be made for contexts much longer than those that there are."""
    for l_max in (2000, 131072, 3000001):
        c = Case(seqs, 2, 4, 64, "bf16", "bf16", seed=17, l_max=l_max).to_device()
        c.check_attend(c.attend())


def test_many_sequences():
    """More sequences than a wavefront has lanes."""
    rng = np.random.default_rng(14)
    c = Case([(int(rng.integers(0, 4)), int(rng.integers(4, 60))) for _ in range(150)], 1, 2, 16, "bf16", "bf16", seed=14).to_device()
    c.check_attend(c.attend())


@pytest.mark.parametrize("B", [2, 64, 65, 150])
@pytest.mark.parametrize("n,kv", [(12, "bf16"), (25, "bf16"), (3, "f32"), (20, "f32")], ids=["pair", "tile", "thin_f32", "tile_f32"])
def test_uneven_batches(n, kv, B):
    """One long sequence among short ones, empty ones and ones without new tokens: their pieces, up to 64 sequences and beyond."""
    rng = np.random.default_rng(B)
    seqs = [(int(rng.integers(0, n + 1)), int(rng.integers(0, 200))) for _ in range(B - 1)] + [(n, 9000)]
    c = Case([seqs[i] for i in rng.permutation(B)], 1, 4, 16, kv, kv, seed=15, n_max=n).to_device()
    c.check_attend(c.attend())


@pytest.mark.parametrize("pages", ["e4m3", "bf16"])
def test_offsets_beyond_32_bits(pages):
    """A pool of more than 2^32 elements, its last pages in use."""
    page, Hkv = 64, 8
    n_pages = (1 << 32) // (page * Hkv * D) + 40
    small = Case([(1, 500), (20, 130)], Hkv, 2, page, "bf16", pages, seed=15, spare=0)
    shift = n_pages - small.n_pages
    small.to_device()
    want = small.attend()
    small.check_attend(want)
    big = {n: torch.zeros((n_pages, Hkv, page, D), dtype=small.d[n].dtype, device=DEV) for n in "KV"}
    bs = {n: None if small.ds[n] is None else torch.zeros((n_pages, Hkv, page, 4), dtype=torch.uint8, device=DEV) for n in "KV"}
    for n in "KV":
        big[n][shift:] = small.d[n]
        if bs[n] is not None:
            bs[n][shift:] = small.ds[n]
    table = torch.where(small.dtable >= 0, small.dtable + shift, small.dtable)
    small.shape.n_pages = n_pages
    small.pg = L.make_pages(K=big["K"], V=big["V"], K_scale=bs["K"], V_scale=bs["V"], table=table, start=small.dstart, kv_len=small.dlen)
    assert torch.equal(small.attend(), want)
    k_out, v_out = (torch.zeros((2, Hkv, small.l_max, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    L.lrqk_pages_append(small.shape, small.pg, small.k_new.to(DEV), small.v_new.to(DEV))
    L.lrqk_pages_read(small.shape, small.pg, 0, k_out, v_out)
    small.append_plain()
    for b in range(2):
        for name, got in (("K", k_out), ("V", v_out)):
            ref, _ = small.rows(name, b)
            assert np.array_equal(got[b, :, :small.len[b]].double().cpu().numpy(), ref)


def test_same_call_twice_is_the_same():
    for seqs in ([(1, 5000), (1, 300)], [(200, 700), (3, 50)]):
        for kv, pages in KINDS[:3]:
            c = Case(seqs, 2, 4, 16, kv, pages, seed=16).to_device()
            assert torch.equal(c.attend(), c.attend())


def exact_on_device(c, b):
    """What check_attend compares with, for sequence b, in float64 on the GPU: for long contexts."""
    lo, hi = int(c.start[b]), int(c.start[b + 1])
    n, Ln = hi - lo, min(int(c.len[b]), c.l_max)
    p = torch.arange(Ln, device=DEV)
    pg = c.dtable[b, p // c.page].long()
    there = (pg >= 0) & (pg < c.n_pages)
    pg = pg.clamp(0, c.n_pages - 1)

    def rows(name):
        x = c.d[name][pg, :, p % c.page]
        if c.sc[name] is None:
            x = x.double()
        else:
            x = x.view(torch.float8_e4m3fn).double() if c.pages == "e4m3" else x.view(torch.int8).double()
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


@pytest.mark.parametrize("kv,pages", KINDS)
@pytest.mark.parametrize("seqs", [[(300, 20000)], [(1, 70001), (1, 300), (1, 33000)], [(12, 30000), (3, 9000)], [(20, 40000)],
                                  [(700, 9000), (1, 40000), (2, 17000)]], ids=["chunk", "ones", "pair", "tile", "mixed"])
def test_long_contexts(seqs, kv, pages):
    """Many pieces for every shape of workgroup, some of the pages missing."""
    c = Case(seqs, 2, 4, 64, kv, pages, seed=50, holes=0.05).to_device()
    out = c.attend().double()
    for b in range(c.B):
        y, mass, slack, Ln = exact_on_device(c, b)
        half = 2.0 ** -8 if kv == "bf16" else 2.0 ** -24
        tol = half * y.abs() + mass * (slack + 2 * Ln * 2.0 ** -24 + (2.0 ** -8 if kv == "bf16" else 0.0))
        far = (out[int(c.start[b]):int(c.start[b + 1])] - y).abs() - tol
        assert float(far.max()) <= 0, f"sequence {b}: off by {float(far.max())} more than the bound"


@pytest.mark.parametrize("n,ln", [(1, 3000), (12, 3000), (100, 3000)])
def test_codes_that_are_no_numbers(n, ln):
    """A pool from elsewhere may hold the code that e4m3 has for NaN, under an ordinary scale."""
    c = Case([(n, ln), (1, 70)], 1, 4, 16, "bf16", "e4m3", seed=51)
    for p, d in ((ln - 1, 7), (ln - max(1, n // 2), 40), (10, 100)):
        pg, o = c.where(0, p)
        c.pool["V"][pg, 0, o, d] = 0x7F if p % 2 else 0xFF
    c.to_device()
    c.check_attend(c.attend())


def test_captured_before_any_call():
    """A call that is recorded before its kernel has ever run."""
    c = Case([(1, 333), (2, 40)], 1, 2, 8, "f32", "i8", seed=52).to_device()
    q, out = c.q.to(DEV), torch.zeros((c.T, c.Hq, D), device=DEV)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        L.lrqk_chunk_attend(c.shape, c.pg, q, out, c.ws)
    for _ in range(3):
        out.fill_(MARK)
        g.replay()
        torch.cuda.synchronize()
        c.check_attend(out)


# ---- rows written and read ---------------------------------------------------------------------------
def odd_rows(x, pages):
    """Blocks at which a scale or a rounding can go wrong."""
    top = P.TOP[pages]
    flat = x.view(-1, 32)
    m = flat.shape[0]
    flat[0 % m] = 0.0
    flat[1 % m] = 3.0e38
    flat[2 % m, :] = 1.0e-30
    flat[3 % m] = torch.linspace(-top, top, 32, dtype=torch.float64).to(x.dtype)
    flat[4 % m, 0] = float(torch.nextafter(torch.tensor(top, dtype=torch.float32), torch.tensor(1e9)))
    flat[5 % m] = (torch.arange(32, dtype=torch.float64) * 0.5 + 0.25).to(x.dtype)
    flat[5 % m, 31] = top
    flat[6 % m, 3] = float("nan")
    flat[7 % m, 9] = float("inf")
    flat[8 % m, 9] = -float("inf")
    flat[9 % m] = -0.0
    flat[10 % m] = 1.0e-40                   # a subnormal number
    flat[11 % m] = -top * 2.0 ** -112
    return x


@pytest.mark.parametrize("kv,pages", KINDS)
@pytest.mark.parametrize("seqs", [[(1, 1)], [(1, 40), (1, 7), (1, 16)], [(70, 100), (0, 9), (33, 33), (5, 3)]], ids=["one", "step", "chunk"])
def test_append(seqs, kv, pages):
    for page, Hkv in ((16, 2), (1, 3), (256, 1)):
        c = Case(seqs, Hkv, 2, page, kv, pages, seed=20, front=2, back=3, holes=0.1 if len(seqs) > 2 else 0.0)
        if pages in P.TOP:
            odd_rows(c.k_new, pages)
        c.to_device()
        L.lrqk_pages_append(c.shape, c.pg, c.k_new.to(DEV), c.v_new.to(DEV))
        c.append_plain()
        for name in "KV":
            a, b = c.d[name].cpu(), c.pool[name]
            if pages in P.TYPE:
                a, b = a.view(torch.int16 if pages == "bf16" else torch.int32), b.view(torch.int16 if pages == "bf16" else torch.int32)
            else:
                assert torch.equal(c.ds[name].cpu(), c.sc[name]), f"{name}: scales"
            assert torch.equal(a, b), f"{name}: rows"


@pytest.mark.parametrize("kv,pages", KINDS)
@pytest.mark.parametrize("first", [0, 1, 50, 1000])
def test_read(first, kv, pages):
    c = Case([(1, 120), (0, 0), (1, 51), (2, 300)], 2, 2, 16, kv, pages, seed=21, holes=0.15, l_max=290, l_cap=301).to_device()
    outs = []
    for make in (lambda: torch.full((c.B, c.Hkv, 301, D), MARK, dtype=P.TYPE[kv], device=DEV),
                 lambda: torch.full((c.B, c.Hkv, 301, D), MARK, dtype=P.TYPE[kv]).pin_memory()):
        K, V = make(), make()
        L.lrqk_pages_read(c.shape, c.pg, first, K, V)
        torch.cuda.synchronize()
        outs.append((K.cpu(), V.cpu()))
        K1 = make()
        L.lrqk_pages_read(c.shape, c.pg, first, K1, None)
        V1 = make()
        L.lrqk_pages_read(c.shape, c.pg, first, None, V1)
        torch.cuda.synchronize()
        assert torch.equal(K1, K) and torch.equal(V1, V)
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    for name, got in zip("KV", outs[0]):
        for b in range(c.B):
            ref, there = c.rows(name, b)
            want = np.full((c.Hkv, 301, D), MARK)
            for p in range(first, len(there)):
                if there[p]:
                    want[:, p] = ref[:, p]
            assert np.array_equal(got[b].double().numpy(), want), f"{name} of sequence {b}"


def test_all_codes_read_back_exactly():
    """Every code with scales over the written range and the marked one, in bf16 and fp32."""
    for pages in ("e4m3", "i8"):
        for kv in ("bf16", "f32"):
            c = Case([(1, 64)], 2, 1, 64, kv, pages, seed=22)
            for name in "KV":
                c.pool[name][:] = torch.arange(c.pool[name].numel(), dtype=torch.int64).to(torch.uint8).view(c.pool[name].shape)
                n = c.sc[name].numel()
                c.sc[name][:] = torch.from_numpy(np.random.default_rng(1).choice([17, 60, 126, 127, 128, 200, 240, 255], n).astype(np.uint8)).view(c.sc[name].shape)
            c.to_device()
            out = torch.zeros((1, 2, 64, D), dtype=P.TYPE[kv], device=DEV)
            L.lrqk_pages_read(c.shape, c.pg, 0, out, None)
            assert np.array_equal(out[0].double().cpu().numpy(), c.rows("K", 0)[0], equal_nan=True)


# ---- together ------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kv,pages", [("bf16", "bf16"), ("bf16", "e4m3"), ("f32", "f32")])
def test_prompt_in_chunks_then_factors_and_a_decode_step(kv, pages):
    """A prompt runs through in chunks, each written and attended; its rows are read back into the host store,
    factorised, and the next token decodes with every position selected: the same as one token's attention
    over the pages."""
    Hkv, G, l, page, dt = 2, 4, 333, 16, P.TYPE[kv]
    Hq = Hkv * G
    c = Case([(0, l)], Hkv, G, page, kv, pages, seed=30, spare=3)
    g = torch.Generator().manual_seed(31)
    k, v = (torch.randn(l, Hkv, D, generator=g).to(dt) for _ in range(2))
    q = (1.5 * torch.randn(l, Hq, D, generator=g)).to(dt)
    c.poison(np.ones((c.n_pages, page), bool))
    c.to_device()
    Kp, Vp = (torch.zeros((1, Hkv, l, D), dtype=dt).pin_memory() for _ in range(2))
    at, outs = 0, []
    for n in (100, 1, 64, 168):
        c.dstart.copy_(torch.tensor([0, n], dtype=torch.int32))
        c.dlen.copy_(torch.tensor([at + n], dtype=torch.int32))
        s = L.PagesShape.make(B=1, Hq=Hq, Hkv=Hkv, T=n, n_max=n, l_max=l, page=page, n_pages=c.n_pages, max_pages=c.max_pages,
                              kv_dtype=KV[kv], page_dtype=PAGE[pages])
        out = torch.empty((n, Hq, D), dtype=dt, device=DEV)
        ws = torch.empty(L.lrqk_pages_workspace_bytes(s), dtype=torch.uint8, device=DEV)
        L.lrqk_pages_append(s, c.pg, k[at:at + n].to(DEV), v[at:at + n].to(DEV))
        L.lrqk_chunk_attend(s, c.pg, q[at:at + n].to(DEV), out, ws)
        L.lrqk_pages_read(s, c.pg, at, Kp, Vp)
        outs.append(out)
        at += n
    torch.cuda.synchronize()
    # all rows as the pages hold them
    c.seqs, c.T, c.start, c.len = [(l, l)], l, np.array([0, l], np.int32), np.array([l], np.int32)
    c.k_new, c.v_new, c.q = k, v, q
    c.append_plain()
    c.check_attend(torch.cat(outs))
    for name, got in (("K", Kp), ("V", Vp)):
        assert np.array_equal(got[0].double().numpy(), c.rows(name, 0)[0])
    # factors of the prompt, then a step that selects everything
    r, w, ksel = 32, 16, l - 16
    shp = L.Shape.make(B=1, Hq=Hq, Hkv=Hkv, l=l, r=r, k=ksel, w=w, C_slots=ksel, kv_dtype=KV[kv])
    A_Q, A_K = torch.randn(1, Hq, l, r, generator=g).to(DEV), torch.randn(1, Hkv, l, r, generator=g).to(DEV)
    B_Q, B_K = torch.zeros(1, Hq, r, D, device=DEV), torch.zeros(1, Hkv, r, D, device=DEV)
    ws = torch.empty(L.lrqk_workspace_bytes(shp, L.LRQK_WS_PREFILL), dtype=torch.uint8, device=DEV)
    Qd = q.permute(1, 0, 2)[None].contiguous().to(DEV)
    L.lrqk_prefill_factorize(shp, Qd, Kp.to(DEV), A_Q, A_K, B_Q, B_K, 1.0, 1.0, 2, ws)
    assert torch.isfinite(A_K).all()
    buf = L.LayerBuffers(shp, A_K, Kp, Vp)
    plan = L.Plan(shp)
    q1 = torch.randn(1, Hq, D, generator=g).to(dt)
    out1 = torch.zeros(1, Hq, D, device=DEV)
    L.lrqk_decode_step(plan, shp, 0, buf.struct, A_Q[:, :, -1].contiguous(), q1.float().to(DEV), out1, L.LRQK_FETCH_DIRECT | L.LRQK_SELECT_FRESH)
    s = L.PagesShape.make(B=1, Hq=Hq, Hkv=Hkv, T=1, n_max=1, l_max=l, page=page, n_pages=c.n_pages, max_pages=c.max_pages,
                          kv_dtype=KV[kv], page_dtype=PAGE[pages])
    c.dstart.copy_(torch.tensor([0, 1], dtype=torch.int32))
    out2 = torch.empty(1, Hq, D, dtype=dt, device=DEV)
    L.lrqk_chunk_attend(s, c.pg, q1.to(DEV), out2, torch.empty(L.lrqk_pages_workspace_bytes(s), dtype=torch.uint8, device=DEV))
    torch.cuda.synchronize()
    c.T, c.start, c.q = 1, np.array([0, 1], np.int32), q1
    c.check_attend(out1.to(dt))
    c.check_attend(out2)
    plan.close()


def test_streams_and_overlap():
    """Calls on two streams, each with its workspace, give what they give alone."""
    a = Case([(1, 6000), (1, 500)], 2, 4, 16, "bf16", "bf16", seed=40).to_device()
    b = Case([(80, 700)], 2, 4, 16, "bf16", "e4m3", seed=41).to_device()
    want = a.attend(), b.attend()
    qa, qb = a.q.to(DEV), b.q.to(DEV)
    oa, ob = (torch.full_like(w, MARK) for w in want)
    torch.cuda.synchronize()
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        L.lrqk_chunk_attend(a.shape, a.pg, qa, oa, a.ws, sa)
        L.lrqk_chunk_attend(b.shape, b.pg, qb, ob, b.ws, sb)
    torch.cuda.synchronize()
    assert torch.equal(oa, want[0]) and torch.equal(ob, want[1])


@pytest.mark.parametrize("kv,pages", [("bf16", "bf16"), ("bf16", "i8"), ("f32", "f32")])
@pytest.mark.parametrize("clean", [False, True], ids=["nan_rows", "clean"])
def test_captured_and_replayed(kv, pages, clean):
    """append, attend and read of a graph follow the lengths and tables that the memory holds at each replay.
    The tables are shuffled, so that rows that nothing had reached come into reach: with NaN, or not."""
    c = Case([(1, 900), (1, 900), (1, 900)], 2, 4, 16, kv, pages, seed=42)
    if clean:
        for name in "KV":
            x = torch.randn(c.pool[name].shape, generator=c.g).to(P.TYPE[kv])
            if pages in P.TYPE:
                c.pool[name] = x
            else:
                c.pool[name], c.sc[name] = (torch.from_numpy(y) for y in P.quantise(x.double().numpy(), pages))
    c.to_device()
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
        assert not clean or torch.isfinite(want).all()
        assert all(torch.equal(bits(x), bits(y)) for x, y in zip(got, (want, K, V))), lens

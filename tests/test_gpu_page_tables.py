"""GPU tests of the tables made on the device: lrqk_pages_advance against the same in plain Python (tests/tables_plain.py),
every number equal, and a serving run of all calls together."""
import numpy as np
import pytest
import torch

import paper_2510_23649_amd as L
import pages_plain as P
import tables_plain as X

pytestmark = pytest.mark.gpu
DEV, D = "cuda", 128
MARK = 1234567
NAMES = ("refs", "table", "kv_len", "start", "status", "seq", "pos", "slot")


class Tables:
    """State on the host and on the device; step() advances both and compares."""

    def __init__(self, B, page, n_pages, T, n_max, l_max, max_pages=None, maps=("seq", "pos", "slot"), Hkv=1, Hq=1, **kw):
        self.page, self.T, self.n_max, self.l_max = page, T, n_max, l_max
        self.max_pages = max_pages or -(-l_max // page)
        self.shape = L.PagesShape.make(B=B, Hq=Hq, Hkv=Hkv, T=T, n_max=n_max, l_max=l_max, page=page, n_pages=n_pages,
                                       max_pages=self.max_pages, **kw)
        self.refs, self.table = np.zeros(n_pages, np.int32), np.full((B, self.max_pages), -1, np.int32)
        self.kv_len = np.zeros(B, np.int32)
        i32 = lambda *s: torch.full(s, MARK, dtype=torch.int32, device=DEV)  # noqa: E731
        self.d = dict(refs=i32(n_pages), table=i32(B, self.max_pages), kv_len=i32(B), start=i32(B + 1), status=i32(B))
        self.d.update({m: i32(T) for m in maps})
        self.tables = L.make_pages_tables(**self.d)
        self.ws = torch.full((L.lrqk_pages_advance_workspace_bytes(self.shape),), 0xA5, dtype=torch.uint8, device=DEV)
        L.lrqk_pages_tables_init(self.shape, self.tables)
        self.same(("refs", "table", "kv_len"), dict(refs=self.refs, table=self.table, kv_len=self.kv_len), "init")

    def put(self):
        for n in ("refs", "table", "kv_len"):
            self.d[n].copy_(torch.from_numpy(getattr(self, n)))

    def same(self, names, want, what):
        for n in names:
            if n in self.d:
                got = self.d[n].cpu().numpy()
                assert np.array_equal(got, want[n]), f"{what}: {n} differs at {np.argwhere(got != want[n])[:4].tolist()}"

    def step(self, keep, n_new, what="", twice=False):
        keep = None if keep is None else np.asarray(keep, np.int32)
        n_new = np.asarray(n_new, np.int32)
        want = X.advance(self.refs, self.table, self.kv_len, keep, n_new, page=self.page, n_max=self.n_max, l_max=self.l_max, T=self.T)
        dk = None if keep is None else torch.from_numpy(keep).to(DEV)
        dn = torch.from_numpy(n_new).to(DEV)
        for _ in range(2 if twice else 1):
            L.lrqk_pages_advance(self.shape, self.tables, dk, dn, self.ws)
            self.same(NAMES, want, what)
        self.refs, self.table, self.kv_len = want["refs"], want["table"], want["kv_len"]
        return want


def consistent(t):
    """Every page counted as often as a table names it, and enough of them for the lengths."""
    count = np.zeros(len(t.refs), np.int64)
    for b, n in enumerate(t.kv_len):
        held = -(-int(n) // t.page)
        assert (t.table[b, :held] >= 0).all() and (t.table[b, held:] == -1).all()
        np.add.at(count, t.table[b, :held], 1)
    assert np.array_equal(count, t.refs)


@pytest.mark.parametrize("page", [1, 2, 16, 64, 1024])
@pytest.mark.parametrize("B", [1, 3, 64, 65, 300])
def test_a_run_of_steps(B, page):
    """Prompts, single tokens, drafts of which some are rejected, requests that end and new ones in their place."""
    rng = np.random.default_rng(B * 1000 + page)
    l_max = 60 * page if page < 64 else 3000
    t = Tables(B, page, max(8, B * 20), B * 40 + 7, 40 if B > 1 else 200, l_max)
    for i in range(25):
        old = t.kv_len.copy()
        keep = old - rng.integers(0, 6, B)
        ends = rng.random(B) < 0.1
        keep[ends] = rng.choice([0, -3], ends.sum())
        n = rng.integers(0, 6, B)
        new = (old == 0) & (rng.random(B) < 0.6)
        n[new] = rng.integers(1, t.n_max + 1, new.sum())
        t.step(None if i % 7 == 3 else keep, n, f"step {i}", twice=i % 3 == 0 and i % 7 != 3)
        consistent(t)


def test_refused_for_what():
    t = Tables(6, 16, 20, 50, 30, 100)
    w = t.step(None, [30, 31, 100, -5, 1 << 30, 2])
    assert w["status"].tolist() == [0, X.LONG, X.LONG, 0, X.LONG, 0] and w["start"].tolist() == [0, 30, 30, 30, 30, 30, 32]
    w = t.step(None, [0, 20, 0, 0, 10, 20])
    assert w["status"].tolist() == [0, 0, 0, 0, 0, 0]
    w = t.step(None, [18, 0, 30, 3, 0, 0])                   # 18 + 30 + 3 rows of 50
    assert w["status"].tolist() == [0, 0, 0, X.ROWS, 0, 0] and w["start"].tolist() == [0, 18, 18, 48, 48, 48, 48]
    w = t.step(None, [30, 2, 0, 0, 0, 0])                    # l_max: 78 + 30 > ...
    assert w["status"].tolist() == [0, 0, 0, 0, 0, 0]
    w = t.step(None, [30, 1, 0, 0, 0, 0])
    assert w["status"].tolist() == [X.LONG, 0, 0, 0, 0, 0]
    consistent(t)
    free = int((t.refs <= 0).sum())
    w = t.step([78, 23, 30, 0, 10, 22], [0, 0, 0, 30, 30, 1])
    assert free >= 0
    t.step([0] * 6, [0] * 6)
    assert (t.refs == 0).all() and (t.table == -1).all()
    # two of three get pages; who needs none is not refused
    t.step(None, [30, 30, 30, 30, 30, 30])
    assert t.kv_len.tolist() == [30, 0, 0, 0, 0, 0]          # 50 rows
    for _ in range(2):
        t.step(None, [0, 30, 0, 0, 0, 0])
        t.step(None, [0, 0, 30, 0, 0, 0])
        t.step(None, [0, 0, 0, 30, 0, 0])
    t.step(None, [0, 0, 0, 0, 30, 0])
    left = int((t.refs <= 0).sum())
    w = t.step(None, [2, 0, 0, 0, 0, 30])
    assert left < 2 or w["status"][5] == 0
    w = t.step(None, [30, 30, 1, 0, 1, 0])
    assert X.PAGES in w["status"].tolist()
    consistent(t)


def test_pages_that_others_count():
    """Pages kept by the caller are not handed out; a shared page is given back by both, and not written to by one."""
    t = Tables(3, 16, 40, 64, 64, 640)
    t.refs[[0, 2, 3, 39]] = 1
    t.put()
    w = t.step(None, [40, 0, 0])
    assert w["table"][0, :3].tolist() == [1, 4, 5]
    # sequence 1 shares two whole pages and a part of the third
    t.table[1, :3], t.kv_len[1] = t.table[0, :3], 36
    t.refs[[1, 4, 5]] += 1
    t.put()
    assert t.step(None, [1, 1, 0])["status"].tolist() == [X.SHARED, X.SHARED, 0]
    w = t.step([40, 32, 0], [1, 5, 3])                       # sequence 1 gives its share of the third page back
    assert w["status"].tolist() == [0, 0, 0] and w["refs"][[1, 4, 5]].tolist() == [2, 2, 1]
    assert t.step([41, 20, 0], [0, 1, 0])["status"].tolist() == [0, X.SHARED, 0]
    assert t.step([41, 16, 0], [0, 1, 0])["status"].tolist() == [0, 0, 0]
    t.step([0, 17, 0], [0, 0, 0])
    assert t.refs[1] == 1 and t.refs[4] == 0
    t.step([0, 0, 0], [0, 0, 0])
    assert t.refs.sum() == 4


def test_tables_that_hold_nonsense():
    """Entries that are no pages, counts below 0, lengths out of range: no address comes of them."""
    t = Tables(4, 16, 30, 40, 30, 300)
    t.table[0, :4] = [-1, 30, (1 << 31) - 1, -(1 << 31)]
    t.table[1, :3] = [0x10000000, 5, 5]
    t.kv_len[:] = [60, 40, (1 << 31) - 1, -7]
    t.refs[[7, 8]] = [-3, -(1 << 31) + 1]
    t.refs[5] = 2
    t.put()
    t.step([33, 20, 5, 9], [10, 20, 30, 2], twice=True)
    t.step([33, 1 << 30, -(1 << 31), (1 << 31) - 1], [1, 1, -(1 << 31), (1 << 31) - 1])


@pytest.mark.parametrize("B", [1024, 1025, 2048, 2049, 5000])
def test_many_sequences(B):
    rng = np.random.default_rng(B)
    t = Tables(B, 16, 3 * B, 4 * B, 60, 900)
    t.step(None, rng.integers(0, 8, B))
    consistent(t)
    for i in range(3):
        keep = np.maximum(t.kv_len - rng.integers(0, 3, B), 0)
        keep[rng.random(B) < 0.1] = 0
        n = rng.integers(0, 5, B)
        n[rng.integers(0, B, 20)] = 60
        t.step(keep, n, f"step {i}", twice=True)
        consistent(t)
    w = t.step(None, np.full(B, 40))                          # neither pages nor rows for all
    assert len(set(w["status"].tolist())) > 1
    consistent(t)


@pytest.mark.parametrize("n_pages", [1, 3, 1023, 4097, 16384, 16385, 50001, 81920, 81921, 140001, 147456, 147457, 200003])
def test_pools(n_pages):
    """Pools up to many times of what is looked at together: free pages only at their end, all over, or none."""
    rng = np.random.default_rng(n_pages)
    for used in (0.0, 0.97, 1.0, "front"):
        t = Tables(5, 4, n_pages, 3000, 700, 4000, maps=("slot",))
        t.refs[:] = (np.arange(n_pages) < n_pages - 7) if used == "front" else rng.random(n_pages) < used
        t.put()
        t.step(None, [1, 600, 17, 0, 300])
        t.step(np.minimum([1, 300, 9, 5, 299], t.kv_len), [0, 2, 3, 25, 8], twice=True)
        t.step([0, 0, 0, 0, 0], [700, 4, 700, 4, 4])


@pytest.mark.parametrize("B", [1500, 2500])
def test_many_sequences_and_a_large_pool(B):
    rng = np.random.default_rng(B)
    t = Tables(B, 2, 170000, 6 * B, 300, 900)
    t.refs[:] = rng.random(170000) < 0.9
    t.refs[:120000] = 1
    t.put()
    n = rng.integers(0, 6, B)
    n[::200] = 300
    t.step(None, n)
    for i in range(3):
        keep = np.maximum(t.kv_len - rng.integers(0, 5, B), 0)
        keep[rng.random(B) < 0.05] = 0
        t.step(keep, rng.integers(0, 7, B), f"step {i}", twice=True)


@pytest.mark.parametrize("T", [1, 6144, 6145, 8191, 8192, 8193, 40000])
def test_rows(T):
    """Maps of few rows and of many, rows of no sequence behind them, one map alone or none."""
    for maps in (("seq", "pos", "slot"), ("pos",), ("slot",), ("seq",), ()):
        for B in (4, 2500):
            if B > T:
                continue
            t = Tables(B, 64, 4000, T, 30000, 30000, max_pages=500, maps=maps)
            n = np.zeros(B, np.int64)
            n[[0, B // 2, B - 1]] = [T // 3, T // 4, max(1, T // 5)]
            if B > 4:
                n[1:B // 2:3] = 1 if T > 8192 else 0
            t.step(None, n)
            t.step(np.maximum(t.kv_len - 2, 0), n, twice=True)


def test_rows_that_pass_32_bits():
    """1023 sequences ask for 1023 * 4198405 = 2^32 + 1019 rows: the last one's row is not the 1020th."""
    B, page, n = 1024, 1024, 4198405
    t = Tables(B, page, 2 * B, 10000, n, n + 1)
    t.refs[:B], t.table[:, 0], t.kv_len[:] = 1, np.arange(B), 1
    t.put()
    w = t.step(None, [n] * (B - 1) + [1])
    assert (w["status"][:-1] == X.PAGES).all() and w["status"][-1] == X.ROWS and w["start"][-1] == 0


def test_captured_and_replayed():
    """A graph follows keep, n_new and the tables; eager steps between its replays."""
    rng = np.random.default_rng(3)
    B = 40
    t = Tables(B, 16, 700, 400, 90, 900)
    keep, n = (torch.zeros(B, dtype=torch.int32, device=DEV) for _ in range(2))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        L.lrqk_pages_advance(t.shape, t.tables, keep, n, t.ws)
    for i in range(6):
        k = np.maximum(t.kv_len - rng.integers(0, 4, B), 0).astype(np.int32)
        m = rng.integers(0, 12, B).astype(np.int32)
        want = X.advance(t.refs, t.table, t.kv_len, k, m, page=16, n_max=90, l_max=900, T=400)
        keep.copy_(torch.from_numpy(k))
        n.copy_(torch.from_numpy(m))
        g.replay()
        torch.cuda.synchronize()
        t.same(NAMES, want, f"replay {i}")
        t.refs, t.table, t.kv_len = want["refs"], want["table"], want["kv_len"]
        t.step(np.maximum(t.kv_len - 1, 0), rng.integers(0, 3, B), f"eager {i}")


def test_streams():
    """Two caches advanced on two streams at once, each with its workspace."""
    rng = np.random.default_rng(4)
    ts = [Tables(3000, 16, 9000, 9000, 20, 300) for _ in range(2)]
    ns = [rng.integers(0, 3, 3000).astype(np.int32) for _ in range(2)]
    want = [X.advance(t.refs, t.table, t.kv_len, None, n, page=16, n_max=20, l_max=300, T=9000) for t, n in zip(ts, ns)]
    dn = [torch.from_numpy(n).to(DEV) for n in ns]
    streams = [torch.cuda.Stream() for _ in ts]
    torch.cuda.synchronize()
    for t, n, s in zip(ts, dn, streams):
        L.lrqk_pages_advance(t.shape, t.tables, None, n, t.ws, s)
    torch.cuda.synchronize()
    for t, w in zip(ts, want):
        t.same(NAMES, w, "stream")


# ---- together ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kv,pages", [("bf16", "e2m1"), ("bf16", "bf16"), ("f32", "e2m1"), ("bf16", "e4m3")])
def test_a_serving_run(kv, pages):
    """Requests come, get drafts of which some are rejected, and end: a captured step of lengths, tables, turned and appended rows and
    attention, replayed, against the attention of each request's tokens from the start, turned in float64, in float64.  The keys
    that the reference attends to are those that the pages hold: what a page holds is compared on its own."""
    Hkv, G, page, B, T, l_max = 2, 4, 16, 4, 72, 160
    Hq, dt = Hkv * G, P.TYPE[kv]
    rng = np.random.default_rng(6)
    types = dict(kv_dtype={"bf16": L.LRQK_KV_BF16, "f32": L.LRQK_KV_F32}[kv],
                 page_dtype={"bf16": L.LRQK_PAGE_BF16, "e2m1": L.LRQK_PAGE_E2M1, "e4m3": L.LRQK_PAGE_E4M3}[pages])
    t = Tables(B, page, 31, T, 64, l_max, Hkv=Hkv, Hq=Hq, **types)
    row = {"bf16": (D, torch.bfloat16), "e2m1": (D // 2, torch.uint8), "e4m3": (D, torch.uint8)}[pages]
    pool = {n: torch.zeros(31, Hkv, page, row[0], dtype=row[1], device=DEV) for n in "KV"}
    if pages == "bf16":
        for n in "KV":
            pool[n].fill_(float("nan"))
    sc = {n: None if pages == "bf16" else torch.full((31, Hkv, page, 4), 255, dtype=torch.uint8, device=DEV) for n in "KV"}
    pg = L.make_pages(K=pool["K"], V=pool["V"], K_scale=sc["K"], V_scale=sc["V"], table=t.d["table"], start=t.d["start"], kv_len=t.d["kv_len"])
    turns, _ = L.lrqk_rope_turns(64, L.LRQK_ROPE_BANDS, base=10000.0, factor=4.0, l_orig=32)
    f, _ = X.frequencies(64, X.BANDS, 10000.0, 4.0, l_orig=32)
    rope = L.make_rope(turns=turns.to(DEV), rot=64)
    qkv = torch.zeros(T, Hq + 2 * Hkv, D, dtype=dt, device=DEV)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    keep, n_new = (torch.zeros(B, dtype=torch.int32, device=DEV) for _ in range(2))
    q_out, out = (torch.full((T, Hq, D), -77.0, dtype=dt, device=DEV) for _ in range(2))
    ws = torch.empty(L.lrqk_pages_workspace_bytes(t.shape), dtype=torch.uint8, device=DEV)

    def step():
        L.lrqk_pages_advance(t.shape, t.tables, keep, n_new, t.ws)
        L.lrqk_pages_rotate_append(t.shape, pg, rope, q, k, v, q_out, pos=t.d["pos"], slot=t.d["slot"])
        L.lrqk_chunk_attend(t.shape, pg, q_out, out, ws)

    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    kept_k = [np.zeros((0, Hkv, D)) for _ in range(B)]        # turned in float64
    kept_v = [np.zeros((0, Hkv, D)) for _ in range(B)]
    plans = [([0, 0, 0, 0], [50, 1, 0, 20]), ([50, 1, 0, 20], [5, 64, 0, 1]), ([53, 65, 0, 20], [1, 1, 3, 2]), ([54, 0, 2, 22], [4, 17, 1, 1]),
             ([58, 17, 3, 0], [1, 2, 60, 1]), ([57, 18, 63, 1], [2, 1, 1, 1])]
    for i, (ks, ns) in enumerate(plans):
        x = torch.from_numpy(rng.standard_normal(tuple(qkv.shape))).to(dt)
        qkv.copy_(x)
        out.fill_(-77.0)
        ka, na = np.array(ks, np.int32), np.array(ns, np.int32)
        keep.copy_(torch.from_numpy(ka))
        n_new.copy_(torch.from_numpy(na))
        want = X.advance(t.refs, t.table, t.kv_len, ka, na, page=page, n_max=64, l_max=l_max, T=T)
        assert not want["status"].any(), "the plan fits"
        g.replay()
        torch.cuda.synchronize()
        t.same(NAMES, want, f"step {i}")
        t.refs, t.table, t.kv_len = want["refs"], want["table"], want["kv_len"]
        xd = x.double().numpy()
        st = want["start"]
        qt, q_mass = X.turned(xd[:, :Hq], want["pos"], f, 1.0, False, False)
        kt, k_mass = X.turned(xd[:, Hq:Hq + Hkv], want["pos"], f, 1.0, False, False)
        half = 2.0 ** -8 if kv == "bf16" else 2.0 ** -24
        rows = slice(0, int(st[-1]))
        got_q = q_out.double().cpu().numpy()
        assert (np.abs(got_q - qt)[rows] <= (8 * 2.0 ** -24 * q_mass + half * 1.001 * np.abs(qt))[rows] + 1e-37).all()
        got = out.double().cpu().numpy()
        assert (got[st[-1]:] == -77.0).all()
        dense = {n: torch.zeros(B, Hkv, l_max, D, dtype=dt, device=DEV) for n in "KV"}
        L.lrqk_pages_read(t.shape, pg, 0, dense["K"], dense["V"])
        for b in range(B):
            lo, hi = int(st[b]), int(st[b + 1])
            kept_k[b] = np.concatenate([kept_k[b][:ks[b]], kt[lo:hi]])
            kept_v[b] = np.concatenate([kept_v[b][:ks[b]], xd[lo:hi, Hq + Hkv:]])
            ln = int(want["kv_len"][b])
            assert len(kept_k[b]) == ln
            K, V = (dense[n][b, :, :ln].double().cpu().numpy() for n in "KV")
            # what the pages hold: values exactly, keys up to the turn and the steps of their codes
            hv = kept_v[b].transpose(1, 0, 2)
            assert np.array_equal(V, hv if pages == "bf16" else P.values(*P.quantise(hv, pages), pages))
            hk = kept_k[b].transpose(1, 0, 2)
            step_of = {"bf16": 2.0 ** -8, "e4m3": 2.0 ** -4, "e2m1": 2.0 ** -2}[pages]
            top = np.repeat(np.abs(hk).reshape(Hkv, ln, 4, 32).max(-1), 32, axis=-1)
            # e2m1: half of the widest step, 2 of 6, under a scale of at most a third of the largest element (6 2^e < 2 max);
            # e4m3: half a step is 2^-4 of a number, or of the smallest normal one, 2^-6 2^e < 2^-6 max / 224
            tol = {"bf16": 0.0 * top, "e4m3": step_of * np.abs(hk) + 2.0 ** -9 * top / 200, "e2m1": top / 3}[pages] * 1.02 + half * 2 * np.abs(hk) + 1e-5
            assert (np.abs(K - hk) <= tol).all()
            if lo == hi:
                continue
            posn = np.arange(ln - (hi - lo), ln)
            y, mass, slack = P.attend(got_q[lo:hi], K, V, np.ones(ln, bool), posn, float(np.float32(D ** -0.5)))
            tol = half * np.abs(y) + mass * (slack[..., None] + 2 * ln * 2.0 ** -24 + (2.0 ** -8 if kv == "bf16" else 0.0)) + 1e-30
            assert (np.abs(got[lo:hi] - y) <= tol).all(), f"step {i}, sequence {b}"

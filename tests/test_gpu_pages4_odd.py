"""GPU tests of pages of 4 bits with V elements that are no numbers anywhere in a context: behind the first blocks of a wavefront, in
a later piece of a split context, in some of the units that a workgroup takes one after the other.  Bounds are those of
tests/test_gpu_pages4.py."""
import numpy as np
import pytest
import torch

import paper_2510_23649_amd as L
import pages_plain as P
import test_gpu_pages as base
from test_gpu_pages import DEV, D, Case

pytestmark = pytest.mark.gpu
base.PAGE["e2m1"] = L.LRQK_PAGE_E2M1
KV = ["bf16", "f32"]
NAN, PLUS, MINUS = "nan", 7, 15              # a whole block; 6 or -6 times 2^127 among zeros


def make(seqs, Hkv=2, G=4, page=16, kv="bf16", **kw):
    c = Case(seqs, Hkv, G, page, kv, "e2m1", **kw)
    rows, big = c.rows, float(torch.finfo(torch.float32).max)

    def as_held(name, b):
        x, there = rows(name, b)
        return np.where(np.abs(x) > big, np.copysign(np.inf, x), x), there

    c.rows = as_held
    return c


def put(c, b, p, h, d, what):
    """Element d of V's row at position p (or its block) becomes `what`."""
    pg, o = c.where(b, p)
    if what == NAN:
        c.sc["V"][pg, h, o, d // 32] = 255
        return
    if c.sc["V"][pg, h, o, d // 32] != 254:
        c.pool["V"][pg, h, o, d // 32 * 16:d // 32 * 16 + 16] = 0
        c.sc["V"][pg, h, o, d // 32] = 254
    c.pool["V"][pg, h, o, d // 2] = int(c.pool["V"][pg, h, o, d // 2]) & (0xF0 if d % 2 == 0 else 0x0F) | what << (4 * (d % 2))


@pytest.mark.parametrize("kv", KV)
@pytest.mark.parametrize("G", [1, 3, 8])
def test_in_later_blocks(kv, G):
    """One piece and several; each kind of element in an early block, in late ones and in the last; two that cancel, the second of
    them seen by later tokens alone."""
    for seqs in ([(1, 1500), (1, 40)], [(5, 3000), (2, 700)], [(40, 1100), (3, 65)]):
        c = make(seqs, 2, G, 16, kv, seed=G + len(seqs[0]))
        for b, (n, ln) in enumerate(seqs):
            put(c, b, 7 if b else 70, 0, 3, PLUS)
            put(c, b, ln // 2, 0, 40, MINUS)
            put(c, b, ln // 2 + 1, 0, 41, PLUS)
            put(c, b, ln // 2 + 1, 1, 64, NAN)
            put(c, b, ln - n, 1, 5, MINUS)
            put(c, b, 3, 0, 100, PLUS)       # until the last token this is an infinity, then a NaN
            put(c, b, ln - 1, 0, 100, MINUS)
            put(c, b, ln - 1, 1, 33, NAN)
        c.to_device()
        c.check_attend(c.attend())


@pytest.mark.parametrize("kv", KV)
@pytest.mark.parametrize("seqs", [[(1, 20001), (1, 3000)], [(6, 9000), (1, 16)], [(300, 5000)]], ids=["one", "few", "chunk"])
def test_in_every_piece(seqs, kv):
    """Infinities far apart in a split context: elements of their own, in the first rows of wavefronts' blocks and the last ones."""
    c = make(seqs, 1, 4, 64, kv, seed=3, holes=0.05)
    n, ln = seqs[0]
    at = [p for p in (64, 511, 1024, 2047, 2300, ln // 2, ln - n - 70, ln - n - 1, ln - n) if c.where(0, p)]
    for i, p in enumerate(at):
        put(c, 0, p, 0, 9 + 12 * i, (PLUS, MINUS)[i % 2])
    c.to_device()
    out = c.attend()
    got = out[:int(c.start[1])].double().cpu().numpy()
    for i, p in enumerate(at):
        assert (got[..., 9 + 12 * i] == (np.inf, -np.inf)[i % 2]).all(), (p, got[0, 0, 9 + 12 * i])
    fine = [d for d in range(D) if d not in [9 + 12 * i for i in range(len(at))]]
    assert np.isfinite(got[..., fine]).all()


@pytest.mark.parametrize("kv", KV)
@pytest.mark.parametrize("n", [1, 3])
def test_in_some_units_of_a_workgroup(n, kv):
    """More units than workgroups: what a unit left out belongs to its own rows.  Sequences without such elements have the bits that
    they have in a call without any."""
    rng = np.random.default_rng(n)
    B = 700
    seqs = [(n, int(rng.integers(n, 400))) for _ in range(B)]  # 512 workgroups
    c = make(seqs, 1, 4, 16, kv, seed=40)
    c.to_device()
    clean = c.attend()
    odd = rng.random(B) < 0.3
    for b in np.flatnonzero(odd):
        for _ in range(2):
            put(c, b, int(rng.integers(0, seqs[b][1])), 0, int(rng.integers(0, D)), (NAN, PLUS, MINUS)[rng.integers(0, 3)])
    c.to_device()
    got = c.attend()
    same = torch.from_numpy(np.repeat(~odd, n)).to(DEV)
    assert torch.equal(got[same], clean[same])
    c.check_attend(got)
    assert torch.equal(c.attend().view(torch.uint8), got.view(torch.uint8))


@pytest.mark.parametrize("kv", KV)
def test_rows_without_a_weight_stay_zero(kv):
    """Scores of -infinity alone: zeros, whatever V holds."""
    c = make([(3, 1200), (2, 90)], 1, 2, 16, kv, seed=5)
    c.q[..., 7] = float("inf")
    for b in range(2):
        for p in range(int(c.len[b])):       # -1 in K's element 7: a score of -infinity
            pg, o = c.where(b, p)
            at = int(c.pool["K"][pg, 0, o, 3])
            c.pool["K"][pg, 0, o, 3] = at & 0x0F | 10 << 4
            c.sc["K"][pg, 0, o, 0] = 127
        put(c, b, 70, 0, 9, PLUS)
        put(c, b, 2, 0, 40, NAN)
    c.to_device()
    assert (c.attend() == 0).all()


def milliseconds(c, q, out):
    best = 1e9
    for _ in range(4):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        L.lrqk_chunk_attend(c.shape, c.pg, q, out, c.ws)
        b.record()
        torch.cuda.synchronize()
        best = min(best, a.elapsed_time(b))
    return best


@pytest.mark.parametrize("kv", KV)
def test_one_element_does_not_slow_the_call_down(kv):
    """A NaN block early in a prompt of 8K: every unit meets it, none may look through the context for more."""
    c = make([(256, 8192)], 1, 4, 16, kv, seed=6).to_device()
    q, out = c.q.to(DEV), torch.empty((c.T, c.Hq, D), dtype=P.TYPE[kv], device=DEV)
    clean = milliseconds(c, q, out)
    pg, o = c.where(0, 70)
    c.ds["V"][pg, 0, o, 1] = 255
    odd = milliseconds(c, q, out)
    assert torch.isnan(out[..., 32:64]).all() and torch.isfinite(out[..., :32]).all() and torch.isfinite(out[..., 64:]).all()
    assert odd <= 3 * clean, f"{odd:.3f} ms, {clean:.3f} without"

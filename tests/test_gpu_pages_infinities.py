"""GPU tests of elements of V that are infinite because their code under its scale exceeds the type: two of opposite signs are a
NaN, not the first of them, for tokens that see both, in blocks that some rows of a workgroup see and others do not (where they are left out
and added at the end) and in blocks that all of them see."""
import numpy as np
import pytest
import torch

import paper_2510_23649_amd as L
import test_gpu_pages as base
from test_gpu_pages import D, Case

pytestmark = pytest.mark.gpu
base.PAGE["e2m1"] = L.LRQK_PAGE_E2M1
CODE = {"e2m1": (7, 15), "e4m3": (0x7E, 0xFE), "i8": (127, 129)}     # the largest and its negative
SEQS = {"one": [(1, 40), (1, 300)], "thin": [(6, 75), (2, 900)], "pair": [(14, 75)], "tile": [(70, 150)]}


def put(c, p, d, negative):
    """Element d of head 0 at position p of sequence 0: +-infinity, the others of its block 0."""
    pg, o = c.where(0, p)
    code = CODE[c.pages][negative]
    if c.pages == "e2m1":
        c.pool["V"][pg, 0, o, d // 32 * 16:d // 32 * 16 + 16] = 0
        c.pool["V"][pg, 0, o, d // 2] = code << (4 * (d % 2))
    else:
        c.pool["V"][pg, 0, o, d // 32 * 32:d // 32 * 32 + 32] = 0
        c.pool["V"][pg, 0, o, d] = code
    c.sc["V"][pg, 0, o, d // 32] = 254


@pytest.mark.parametrize("kv", ["bf16", "f32"])
@pytest.mark.parametrize("pages", CODE)
@pytest.mark.parametrize("page", [16, 4])
@pytest.mark.parametrize("way", SEQS)
def test_of_both_signs(way, page, pages, kv):
    seqs = SEQS[way]
    n, ln = seqs[0]
    c = Case(seqs, 2, 3, page, kv, pages, seed=n)
    pairs = ((4, 3, ln - 1), (37, 3, ln - 1), (70, 0, ln // 2), (77, ln - n, ln - 1))   # element, position of either: no block twice
    for d, p, r in pairs:
        if p == r:
            continue
        put(c, p, d, False)
        put(c, r, d, True)
    put(c, 7, 110, True)                                     # one alone stays what it is
    c.to_device()
    got = c.attend()[:n].double().cpu().numpy()
    for d, p, r in pairs:
        if p == r:
            continue
        for i in range(n):                                   # token i sees the positions up to ln - n + i
            sees = [x <= ln - n + i for x in (p, r)]
            y = got[i, :c.G, d]
            if all(sees):
                assert np.isnan(y).all(), (d, i, y)
            elif any(sees):
                assert (y == (np.inf if sees[0] else -np.inf)).all(), (d, i, y)
            else:
                assert np.isfinite(y).all(), (d, i, y)
    if ln - n >= 7:
        assert (got[:, :c.G, 110] == -np.inf).all()
    assert np.isfinite(got[:, c.G:]).all()

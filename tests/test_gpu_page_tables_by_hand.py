"""GPU tests of lrqk_pages_advance whose statuses and pages are worked out by hand, and of what a caller does with a shared page."""
import numpy as np
import pytest
import torch

import paper_2510_23649_amd as L
import tables_plain as X
from test_gpu_page_tables import DEV, Tables, consistent

pytestmark = pytest.mark.gpu


def test_each_refusal():
    """Six pages of 16 positions, four sequences, 40 rows a step, 30 of one sequence."""
    t = Tables(4, 16, 6, 40, 30, 64)
    w = t.step(None, [20, 16, 0, 0])                         # 2 + 1 pages, 36 rows
    assert w["status"].tolist() == [X.OK] * 4 and w["start"].tolist() == [0, 20, 36, 36, 36]
    assert w["table"][:, :2].tolist() == [[0, 1], [2, -1], [-1, -1], [-1, -1]]
    w = t.step(None, [12, 0, 30, 17])                        # 0, 0, 2, 4 pages asked for, 3 are free; 12, 12, 42, 59 rows of 40
    assert w["status"].tolist() == [X.OK, X.OK, X.ROWS, X.PAGES] and w["kv_len"].tolist() == [32, 16, 0, 0]
    assert w["start"].tolist() == [0, 12, 12, 12, 12] and (w["seq"][:12] == 0).all() and (w["seq"][12:] == -1).all()
    w = t.step(None, [8, 31, 65, -1])                        # more than n_max asks for nothing; no new tokens is no refusal
    assert w["status"].tolist() == [X.OK, X.LONG, X.LONG, X.OK] and w["table"][0, :3].tolist() == [0, 1, 3]
    w = t.step(None, [25, 16, 16, 1])                        # 40 + 25 > 64; 1, 2, 3 pages of 2
    assert w["status"].tolist() == [X.LONG, X.OK, X.OK, X.PAGES] and w["kv_len"].tolist() == [40, 32, 16, 0]
    assert w["table"][1, :2].tolist() == [2, 4] and w["table"][2, 0] == 5
    w = t.step(None, [8, 1, 1, 1])                           # no page is free: who needs none gets its rows
    assert w["status"].tolist() == [X.OK, X.PAGES, X.PAGES, X.PAGES] and w["kv_len"].tolist() == [48, 32, 16, 0]
    w = t.step([48, 20, 16, 0], [0, 12, 0, 16])              # a page comes back only if none of its positions is kept
    assert w["status"].tolist() == [X.OK, X.OK, X.OK, X.PAGES] and w["kv_len"].tolist() == [48, 32, 16, 0]
    w = t.step([48, 16, 16, 0], [0, 0, 0, 16])               # and is handed out in the same call
    assert w["status"].tolist() == [X.OK] * 4 and w["table"][3, 0] == 4 and w["table"][1, :2].tolist() == [2, -1]
    consistent(t)


def test_a_shared_page_is_copied_by_the_caller():
    """A prefix of 40 positions is shared: the sequence that goes on from it is refused while its next row lies on the shared third page, and
    goes on once the caller has copied that page and counted the copy."""
    t = Tables(2, 16, 12, 64, 64, 160)
    t.step(None, [40, 0])
    t.table[1, :3], t.kv_len[1] = t.table[0, :3], 40
    t.refs[:3] += 1
    t.put()
    w = t.step(None, [0, 5])
    assert w["status"].tolist() == [X.OK, X.SHARED] and w["kv_len"].tolist() == [40, 40]
    pool = torch.arange(12 * 16, device=DEV).view(12, 16).clone()      # (a layer's pool: each of K, V and their scales)
    old, new = int(t.table[1, 2]), int(np.flatnonzero(t.refs <= 0)[-1])
    pool[new] = pool[old]
    t.refs[old] -= 1
    t.refs[new] = 1
    t.table[1, 2] = new
    t.put()
    w = t.step(None, [3, 5])
    assert w["status"].tolist() == [X.OK, X.OK] and w["kv_len"].tolist() == [43, 45]
    slot = w["slot"].tolist()
    assert slot[:8] == [16 * old + 8, 16 * old + 9, 16 * old + 10] + [16 * new + 8 + i for i in range(5)]
    assert w["refs"][[old, new]].tolist() == [1, 1]
    consistent(t)

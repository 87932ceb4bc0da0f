"""The package is imported with a torch that has no type of its own for 4 bits; rows of 4 bits are uint8 there."""
import os
import subprocess
import sys

PROGRAM = """
import torch
if hasattr(torch, "float4_e2m1fn_x2"):
    del torch.float4_e2m1fn_x2
import paper_2510_23649_amd as L
from paper_2510_23649_amd import binding
binding._dev = lambda x, dtype=None: None if x is None else 0x10000
binding._raw_stream = lambda *a: 0
i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
u8 = lambda d: torch.zeros(20, 2, 16, d, dtype=torch.uint8)
s = L.PagesShape.make(B=1, Hq=4, Hkv=2, T=3, n_max=3, l_max=100, page=16, n_pages=20, max_pages=7, page_dtype=L.LRQK_PAGE_E2M1)
pages = lambda d: L.make_pages(K=u8(d), V=u8(d), K_scale=u8(4), V_scale=u8(4), table=i32(1, 7), start=i32(2), kv_len=i32(1))
binding._hold(pages(64), s)
try:
    binding._hold(pages(63), s)
except ValueError:
    print("as it should be")
"""


def test_without_the_type():
    root = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..")
    r = subprocess.run([sys.executable, "-c", PROGRAM], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "as it should be", r.stderr

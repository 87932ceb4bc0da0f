"""The paged cache and its attention in plain float64 on the host: what the GPU tests compare with.
Written from the definitions; neither the HIP library nor its plain torch forms are called."""
from __future__ import annotations

import numpy as np
import torch

D, BLOCK, E_MIN = 128, 32, -110
TOP = {"e4m3": 448.0, "i8": 127.0}
TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


def quantise(x: np.ndarray, pages: str):
    """Rows x [..., 128] (float64 values of the inputs) -> codes uint8 [..., 128], scale bytes [..., 4]."""
    shape = x.shape
    x = x.reshape(-1, BLOCK).astype(np.float64)
    bad = ~np.isfinite(x).all(1)
    x = np.where(bad[:, None], 0.0, x)
    top = np.abs(x).max(1)
    m, e = np.frexp(top / TOP[pages])        # exact: a quotient of float64 by 448 or 127 is compared below
    e = e.astype(np.int64) - 2
    for _ in range(4):
        e = np.where(top > np.ldexp(TOP[pages], e), e + 1, e)
    e = np.maximum(np.where(top == 0, E_MIN, e), E_MIN)
    y = np.ldexp(x, -e[:, None])             # exact: a power of two
    if pages == "e4m3":                      # float64 -> float32 is exact here or far below half a step
        code = torch.from_numpy(y).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    else:
        code = np.rint(y).astype(np.int8).view(np.uint8)
    code = np.where(bad[:, None], 0, code).astype(np.uint8)
    byte = np.where(bad, 255, e + 127).astype(np.uint8)
    return code.reshape(shape), byte.reshape(*shape[:-1], D // BLOCK)


def values(code: np.ndarray, byte: np.ndarray, pages: str) -> np.ndarray:
    """float64 values of codes [..., 128] with scale bytes [..., 4]."""
    if pages == "e4m3":
        v = torch.from_numpy(np.ascontiguousarray(code)).view(torch.float8_e4m3fn).double().numpy()
    else:
        v = code.view(np.int8).astype(np.float64)
    s = np.where(byte == 255, np.nan, np.ldexp(1.0, byte.astype(np.int64) - 127))
    return v * np.repeat(s, BLOCK, axis=-1)


def attend(q, K, V, there, pos, scale):
    """One sequence.  q [n,Hq,D], K, V [Hkv,L,D] float64, there [L] bool, pos [n] -> out [n,Hq,D] float64,
    mass [n,Hq,D] = sum_p w_p |V_p|, slack [n,Hq]: relative error of a weight in fp32 (worst case)."""
    n, Hq, _ = q.shape
    G = Hq // K.shape[0]
    out, mass, slack = np.zeros((n, Hq, D)), np.zeros((n, Hq, D)), np.zeros((n, Hq))
    for i in range(n):
        see = np.flatnonzero(there[:max(0, min(int(pos[i]) + 1, len(there)))])
        if len(see) == 0:
            continue
        for h in range(Hq):
            k, v = K[h // G, see], V[h // G, see]
            with np.errstate(invalid="ignore", over="ignore"):
                s = scale * (k @ q[i, h])
                w = np.exp(s - s.max())
                w = w / w.sum()
                out[i, h] = (w[:, None] * v).sum(0)
                mass[i, h] = (w[:, None] * np.abs(v)).sum(0)
                # a dot product of 128 terms in fp32, the scaling, the subtraction and the exponential; what lies 100
                # below the largest score has a weight under 2^-144 however it is rounded
                near = s >= s.max() - 100
                if near.any():
                    slack[i, h] = 2 * (abs(scale) * (np.abs(k[near]) @ np.abs(q[i, h])).max() * 130 + 3 * np.abs(s[near]).max() + 4) * 2.0 ** -24
    return out, mass, slack

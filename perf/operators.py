"""The paged K/V cache and the attention of new tokens over it, measured as a serving program calls them.

Three operators that share one cache of pages:

  attend   lrqk_chunk_attend: exact causal attention of each sequence's new tokens (one, a drafted
           handful, a chunk, a whole prompt) over its paged rows
  append   lrqk_pages_append: the new tokens' K and V rows go into their pages; where pages hold
           8-bit rows the case also reads the rows back, since values are what a program gets
  read     lrqk_pages_read: rows of the pages as dense per-head arrays, the layout that the prompt's
           factorisation and the host store take

`listed()` names the cases, `draw()` gives more of the same ranges, `prepare()` makes what a program
holds before the call (inputs, pages, table, workspace), `run()` makes one pass.  With `own` false the
pass is the plain form in elementary torch operations.

8-bit rows: every 32 elements share a scale 2^e, the smallest (e >= -110) for which none of them
exceeds the largest code (448 for e4m3, 127 for i8); codes are rounded to nearest, ties to even.  The
scale is kept as the byte e + 127.
"""
import math
import random

import torch

own = False

DEV = "cuda"
D = 128
BLOCK = 32                                   # elements that share a scale
TOP = {"e4m3": 448.0, "i8": 127.0}
TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
E_MIN = -110
ROWS_AT_ONCE = 1 << 28                       # scores held at a time


def _case(kind, name, B, Hq, Hkv, n, l, page, kv="bf16", pages="bf16", ragged=0):
    """n new tokens at most and l positions at most a sequence; ragged: seed of their spread, or 0."""
    c = dict(kind=kind, B=B, Hq=Hq, Hkv=Hkv, n=n, l=l, page=page, kv=kv, pages=pages, ragged=ragged)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of one sequence over a short context: launches and latency
        _case("attend", "attend_one_4k", 1, 32, 8, 1, 4096, 16),
        # a decode step of sixteen sequences of very different lengths, 8-bit rows: the stream of rows
        _case("attend", "attend_decode_128k_b16_e4m3", 16, 32, 8, 1, 131072, 64, pages="e4m3", ragged=11),
        # five drafted tokens of eight sequences to be verified, heads in groups of seven
        _case("attend", "attend_draft_64k_b8_i8", 8, 28, 4, 5, 65536, 32, pages="i8", ragged=12),
        # a chunk in the middle of a prompt of 32K
        _case("attend", "attend_chunk_32k", 1, 32, 8, 2048, 32768, 64),
        # whole prompts of several lengths in one call
        _case("attend", "attend_prompts_b6", 6, 32, 8, 8192, 8192, 128, ragged=13),
        # fp32 rows, odd sizes
        _case("attend", "attend_chunk_f32_odd", 2, 28, 4, 1001, 5003, 16, "f32", "f32", ragged=14),
        # the last chunk of a prompt of 128K, 8-bit rows
        _case("attend", "attend_chunk_128k_e4m3", 1, 32, 8, 1024, 131072, 256, pages="e4m3"),
        # the rows of one decode step of sixteen sequences
        _case("append", "append_one_b16", 16, 32, 8, 1, 1000, 16, ragged=15),
        # prompts of several lengths, quantised as they are written, read back
        _case("append", "append_prompts_e4m3", 4, 32, 8, 8192, 8192, 64, pages="e4m3", ragged=16),
        # fp32 rows into 8-bit integers, odd sizes
        _case("append", "append_f32_i8_odd", 3, 28, 4, 777, 777, 32, "f32", "i8", ragged=17),
        # a prompt of 32K for the factorisation
        _case("read", "read_32k_e4m3", 1, 32, 8, 1, 32768, 64, pages="e4m3"),
        # short contexts of several lengths
        _case("read", "read_b8_i8_odd", 8, 28, 4, 1, 1003, 16, pages="i8", ragged=18),
    ]


def draw(rng):
    spread = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    Hkv, G = rng.choice([(8, 4), (4, 7), (8, 1), (2, 8), (5, 3), (1, 5), (8, 2)])
    kv, pages = rng.choice([("bf16", "bf16"), ("bf16", "e4m3"), ("bf16", "i8"), ("f32", "f32"),
                            ("f32", "e4m3"), ("f32", "i8")])
    page = 1 << rng.randint(4, 8)
    ragged = rng.randint(1, 1 << 20)
    kind = rng.choice(["one", "draft", "chunk", "prompt", "append", "read"])
    if kind in ("one", "draft"):
        n = 1 if kind == "one" else rng.randint(2, 16)
        B = spread(1, 32)
        return _case("attend", None, B, Hkv * G, Hkv, n, n + spread(16, min(131072, 1000000 // B)), page, kv, pages, ragged)
    if kind in ("chunk", "prompt"):
        most = 12000 if kv == "f32" else 40000
        B, n = spread(1, 8), spread(17, 2048)
        c = spread(16, max(32, min(most, 60000000 // (B * n)))) if kind == "chunk" else 0
        return _case("attend", None, B, Hkv * G, Hkv, n, n + c, page, kv, pages, ragged)
    B, n = spread(1, 16), spread(1, 2048)
    c = spread(1, 4096) if kind == "read" else 0
    return _case(kind, None, B, Hkv * G, Hkv, n, n + c, page, kv, pages, ragged)


def lengths(c):
    """New tokens and positions (the new ones among them) of each sequence."""
    if not c["ragged"]:
        return [c["n"]] * c["B"], [c["l"]] * c["B"]
    r = random.Random(c["ragged"])
    some = lambda top, by: int(round(top * by ** -r.random())) if top else 0  # noqa: E731
    n = [c["n"]] + [max(1, some(c["n"], 16.0)) for _ in range(c["B"] - 1)]
    old = [c["l"] - c["n"]] + [some(c["l"] - c["n"], 16.0) for _ in range(c["B"] - 1)]
    return n, [a + b for a, b in zip(n, old)]


# ---- 8-bit rows in elementary operations ---------------------------------------------------------
def quantise(x, pages):
    """Codes and scale bytes of rows x [..., D]."""
    x = x.float().unflatten(-1, (D // BLOCK, BLOCK))
    top = x.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(top / TOP[pages])     # top = TOP m 2^e up to rounding: settled by comparing
    e = torch.where(top <= torch.ldexp(torch.full_like(top, TOP[pages]), e - 1), e - 1, e)
    e = torch.where(top > torch.ldexp(torch.full_like(top, TOP[pages]), e), e + 1, e)
    e = torch.where(top > 0, e, torch.full_like(e, E_MIN)).clamp_min(E_MIN)
    x = torch.ldexp(x, -e)
    codes = x.to(torch.float8_e4m3fn).view(torch.uint8) if pages == "e4m3" else torch.round(x).to(torch.int8).view(torch.uint8)
    return codes.flatten(-2), (e.squeeze(-1) + 127).to(torch.uint8)


def values(codes, scales, pages):
    """Rows in 32 bits from codes [..., D] and scale bytes [..., D / BLOCK]."""
    x = codes.view(torch.float8_e4m3fn if pages == "e4m3" else torch.int8).float()
    return torch.ldexp(x.unflatten(-1, (D // BLOCK, BLOCK)), scales.int()[..., None] - 127).flatten(-2)


# ---- inputs --------------------------------------------------------------------------------------
def prepare(c, seed):
    g = torch.Generator(device=DEV).manual_seed(seed * 7919 + 13)
    rn = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    B, Hq, Hkv, page, kvt = c["B"], c["Hq"], c["Hkv"], c["page"], TYPE[c["kv"]]
    G = Hq // Hkv
    n, ln = lengths(c)
    T = sum(n)
    max_pages = -(-c["l"] // page)
    used = [-(-x // page) for x in ln]
    n_pages = sum(used) + 3
    # pages lie in the pool as they were handed out and given back: in no order
    ids = torch.randperm(n_pages, generator=g, device=DEV)[:sum(used)].to(torch.int32)
    table = torch.full((B, max_pages), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b in range(B):
        table[b, :used[b]] = ids[at:at + used[b]]
        at += used[b]
    s = dict(c=c, n=n, ln=ln, table=table,
             start=torch.tensor([0] + [sum(n[:b + 1]) for b in range(B)], dtype=torch.int32, device=DEV),
             kv_len=torch.tensor(ln, dtype=torch.int32, device=DEV))
    # K: channels of different size and a direction that some rows share and queries look for, so that a
    # head's weights are neither flat nor one row's; V about a mean of its own
    size = torch.exp(0.5 * rn(Hkv, 1, D))
    look = rn(Hkv, 1, D)
    look = look / look.norm(dim=-1, keepdim=True)
    mean = 0.5 * rn(Hkv, 1, D)

    def fill(make):
        if c["pages"] in TYPE:
            pool = torch.empty((n_pages, Hkv, page, D), dtype=TYPE[c["pages"]], device=DEV)
            scale = None
        else:
            pool = torch.empty((n_pages, Hkv, page, D), dtype=torch.uint8, device=DEV)
            scale = torch.empty((n_pages, Hkv, page, D // BLOCK), dtype=torch.uint8, device=DEV)
        step = max(1, (1 << 26) // (Hkv * page * D))
        for i in range(0, n_pages, step):
            x = make(min(step, n_pages - i))
            if scale is None:
                pool[i:i + step] = x
            else:
                pool[i:i + step], scale[i:i + step] = quantise(x, c["pages"])
        return pool, scale

    heavy = lambda *s: (torch.rand(*s, 1, generator=g, device=DEV) < 0.01) * 12.0  # noqa: E731
    s["K"], s["K_scale"] = fill(lambda p: rn(p, Hkv, page, D) * size + heavy(p, Hkv, page) * look)
    s["V"], s["V_scale"] = fill(lambda p: rn(p, Hkv, page, D) + mean)
    if c["kind"] == "attend":
        q = rn(T, Hkv, G, D) + 4.0 * look[None]
        s["q"] = q.reshape(T, Hq, D).to(kvt)
        s["out"] = torch.zeros((T, Hq, D), dtype=kvt, device=DEV)
    else:
        if c["kind"] == "append":
            s["k_new"] = (rn(T, Hkv, D) * size[:, 0]).to(kvt)
            s["v_new"] = (rn(T, Hkv, D) + mean[:, 0]).to(kvt)
        s["K_out"] = torch.zeros((B, Hkv, c["l"], D), dtype=kvt, device=DEV)
        s["V_out"] = torch.zeros((B, Hkv, c["l"], D), dtype=kvt, device=DEV)
    if own:
        import paper_2510_23649_amd as L
        s["shape"] = L.PagesShape.make(
            B=B, Hq=Hq, Hkv=Hkv, T=T, n_max=c["n"], l_max=c["l"], page=page, n_pages=n_pages, max_pages=max_pages,
            kv_dtype={"bf16": L.LRQK_KV_BF16, "f32": L.LRQK_KV_F32}[c["kv"]],
            page_dtype={"bf16": L.LRQK_PAGE_BF16, "f32": L.LRQK_PAGE_F32, "e4m3": L.LRQK_PAGE_E4M3, "i8": L.LRQK_PAGE_I8}[c["pages"]])
        s["pages"] = L.make_pages(K=s["K"], V=s["V"], K_scale=s["K_scale"], V_scale=s["V_scale"], table=table,
                                  start=s["start"], kv_len=s["kv_len"])
        s["ws"] = torch.empty(max(256, L.lrqk_pages_workspace_bytes(s["shape"])), dtype=torch.uint8, device=DEV)
    return s


# ---- one pass ------------------------------------------------------------------------------------
def run(s):
    kind, pages = s["c"]["kind"], s["c"]["pages"]
    if own:
        import paper_2510_23649_amd as L
        if kind == "attend":
            L.lrqk_chunk_attend(s["shape"], s["pages"], s["q"], s["out"], s["ws"])
            return s["out"]
        if kind == "append":
            L.lrqk_pages_append(s["shape"], s["pages"], s["k_new"], s["v_new"])
            if pages in TYPE:
                return s["K"], s["V"]
        L.lrqk_pages_read(s["shape"], s["pages"], 0, s["K_out"], s["V_out"])
        return s["K_out"], s["V_out"]
    if kind == "attend":
        return _attend(s)
    if kind == "append":
        _append(s)
        if pages in TYPE:
            return s["K"], s["V"]
    for b in range(s["c"]["B"]):
        s["K_out"][b, :, :s["ln"][b]] = _rows(s, b, "K")
        s["V_out"][b, :, :s["ln"][b]] = _rows(s, b, "V")
    return s["K_out"], s["V_out"]


def _rows(s, b, name):
    """Sequence b's rows in 32 bits, [Hkv, length, D]."""
    p = torch.arange(s["ln"][b], device=DEV)
    page = s["table"][b, p // s["c"]["page"]].long()
    x = s[name][page, :, p % s["c"]["page"]]
    if s["c"]["pages"] in TYPE:
        x = x.float()
    else:
        x = values(x, s[name + "_scale"][page, :, p % s["c"]["page"]], s["c"]["pages"])
    return x.transpose(0, 1)


def _append(s):
    page, at = s["c"]["page"], 0
    for b, (n, ln) in enumerate(zip(s["n"], s["ln"])):
        p = torch.arange(ln - n, ln, device=DEV)
        to = s["table"][b, p // page].long()
        for name in ("K", "V"):
            x = s[name.lower() + "_new"][at:at + n]
            if s["c"]["pages"] in TYPE:
                s[name][to, :, p % page] = x.to(s[name].dtype)
            else:
                s[name][to, :, p % page], s[name + "_scale"][to, :, p % page] = quantise(x, s["c"]["pages"])
        at += n


def _attend(s):
    c = s["c"]
    Hkv, G = c["Hkv"], c["Hq"] // c["Hkv"]
    out, at = torch.empty_like(s["out"]), 0
    for b, (n, ln) in enumerate(zip(s["n"], s["ln"])):
        K, V = _rows(s, b, "K").transpose(1, 2).contiguous(), _rows(s, b, "V").contiguous()
        p = torch.arange(ln, device=DEV)
        step = max(1, ROWS_AT_ONCE // (ln * c["Hq"]))
        for i in range(0, n, step):
            m = min(step, n - i)
            q = s["q"][at + i:at + i + m].float().reshape(m, Hkv, G, D).permute(1, 0, 2, 3).reshape(Hkv, m * G, D)
            x = torch.matmul(q, K).mul_(D ** -0.5).reshape(Hkv, m, G, ln)
            own_p = torch.arange(ln - n + i, ln - n + i + m, device=DEV)
            x.masked_fill_((p[None, :] > own_p[:, None])[None, :, None, :], -math.inf)
            x = torch.exp_(x.sub_(x.amax(-1, keepdim=True)))
            w = x.sum(-1, keepdim=True)
            y = torch.matmul(x.reshape(Hkv, m * G, ln), V).reshape(Hkv, m, G, D) / w
            out[at + i:at + i + m] = y.permute(1, 0, 2, 3).reshape(m, c["Hq"], D)
        at += n
    return out


# ---- the same from the definitions, in 64 bits -----------------------------------------------------
def _grid64(x, pages):
    """What rows x (float64) stand for once they are held in 8 bits."""
    shape = x.shape
    x = x.reshape(-1, BLOCK)
    top = x.abs().max(dim=1, keepdim=True).values
    unit = torch.exp2(torch.ceil(torch.log2(top.clamp_min(1e-300))) - (9 if pages == "e4m3" else 7) - 1)
    for _ in range(3):                       # up to the smallest power of two that holds the block
        unit = torch.where(top > TOP[pages] * unit, 2 * unit, unit)
    unit = unit.clamp_min(2.0 ** E_MIN)
    y = x / unit
    if pages == "i8":
        return (torch.round(y) * unit).reshape(shape)
    # e4m3: three bits behind the leading one, down to steps of 2^-9
    ulp = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3)
    return (torch.round(y / ulp) * ulp * unit).reshape(shape)


def exact(c, seed):
    s = prepare(c, seed)
    page = c["page"]
    where = lambda b, lo, hi: (s["table"][b].long().repeat_interleave(page)[lo:hi],  # noqa: E731
                               torch.arange(hi, device=DEV)[lo:] % page)

    def dense(b, name):
        pg, off = where(b, 0, s["ln"][b])
        x = s[name].permute(1, 0, 2, 3)[:, pg, off]
        if c["pages"] in TYPE:
            return x.double()
        x = x.view(torch.int8).double() if c["pages"] == "i8" else x.view(torch.float8_e4m3fn).double()
        sc = torch.exp2(s[name + "_scale"].permute(1, 0, 2, 3)[:, pg, off].double() - 127)
        return x * sc.repeat_interleave(BLOCK, dim=-1)

    if c["kind"] == "read":
        got = []
        for name in ("K", "V"):
            o = torch.zeros(c["B"], c["Hkv"], c["l"], D, dtype=torch.float64, device=DEV)
            for b in range(c["B"]):
                o[b, :, :s["ln"][b]] = dense(b, name)
            got.append(o)
        return tuple(got)
    if c["kind"] == "append":
        got = []
        for name in ("K", "V"):
            x = s[name.lower() + "_new"].double()
            o = s[name].double() if c["pages"] in TYPE else torch.zeros(c["B"], c["Hkv"], c["l"], D, dtype=torch.float64, device=DEV)
            at = 0
            for b in range(c["B"]):
                n, ln = s["n"][b], s["ln"][b]
                if c["pages"] in TYPE:
                    o[where(b, ln - n, ln)[0], :, where(b, ln - n, ln)[1]] = x[at:at + n]
                else:
                    o[b, :, :ln] = dense(b, name)
                    o[b, :, ln - n:ln] = _grid64(x[at:at + n], c["pages"]).permute(1, 0, 2)
                at += n
            got.append(o)
        return tuple(got)
    G, at = c["Hq"] // c["Hkv"], 0
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    for b in range(c["B"]):
        n, ln = s["n"][b], s["ln"][b]
        K, V = dense(b, "K"), dense(b, "V")
        for h in range(c["Hq"]):
            step = max(1, (1 << 27) // ln)
            for i in range(0, n, step):
                j = min(n, i + step)
                x = (s["q"][at + i:at + j, h].double() @ K[h // G].t()) / math.sqrt(D)
                hidden = torch.ones(j - i, ln, dtype=torch.bool, device=DEV).triu(ln - n + i + 1)
                x[hidden] = -math.inf
                out[at + i:at + j, h] = torch.softmax(x, dim=1) @ V[h // G]
        at += n
    return out


def work(c):
    """Each input read once and each output written once; a page's unwritten rows are no work."""
    n, ln = lengths(c)
    e = {"bf16": 2.0, "f32": 4.0}
    row = D * e[c["kv"]]
    held = D * e[c["pages"]] if c["pages"] in e else D + D / BLOCK
    index = 4.0 * (2 * c["B"] + 1) + 4.0 * sum(-(-x // c["page"]) for x in ln)
    if c["kind"] == "attend":
        seen = sum(a * (b - a) + a * (a + 1) / 2 for a, b in zip(n, ln))
        return {"bytes": 2 * sum(n) * c["Hq"] * row + 2 * sum(ln) * c["Hkv"] * held + index, "flops": 4.0 * D * c["Hq"] * seen}
    back = 2 * sum(ln) * c["Hkv"] * (held + row)
    if c["kind"] == "read":
        return {"bytes": back + index, "flops": 0.0}
    wrote = 2 * sum(n) * c["Hkv"] * (row + held)
    return {"bytes": wrote + index if c["pages"] in e else wrote + back + index, "flops": 0.0}

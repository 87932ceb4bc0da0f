"""A serving step around the paged K/V cache, measured as a serving program calls it.

Four operators that a step runs one after the other:

  advance  lrqk_pages_advance: from what each request keeps and gets, the lengths, the packed starts, the block table
           (pages given back and taken) and each packed row's sequence, position and slot
  rotate   lrqk_rotate: rotary positions of queries and keys at positions of their own
  write    lrqk_pages_rotate_append: queries and keys out of a projection turned, keys and values into their
           pages; where pages hold 4 or 8 bits the case also reads the rows back, since values are what a program gets
  attend   lrqk_chunk_attend over pages of 4 bits: exact causal attention of each sequence's new tokens

`listed()` names the cases, `draw()` gives more of the same ranges, `prepare()` makes what a program holds before the
call, `run()` makes one pass.  With `own` false the pass is the plain form in elementary torch operations.

Rows of 4 bits: every 32 elements share a scale 2^e, the smallest (e >= -110) for which none of them exceeds 6, kept as
the byte e + 127; a code is a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6, the nearest, ties to the even code; element 2 i
is the low half of byte i.  Rows of 8 bits likewise, with the codes of e4m3.
"""
import math
import random

import torch

own = False

DEV = "cuda"
D = 128
BLOCK = 32                                   # elements that share a scale
TOP = {"e2m1": 6.0, "e4m3": 448.0}
TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
E_MIN = -110
STEPS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
ROWS_AT_ONCE = 1 << 28                       # scores held at a time


def _attend(name, B, Hq, Hkv, n, l, page, kv="bf16", ragged=0):
    """n new tokens at most and l positions at most a sequence; ragged: seed of their spread, or 0."""
    return _named(name, dict(kind="attend", B=B, Hq=Hq, Hkv=Hkv, n=n, l=l, page=page, kv=kv, pages="e2m1", ragged=ragged))


def _write(name, B, Hq, Hkv, n, l, page, kv="bf16", pages="bf16", layout="halves", rot=128, scaling="none", maps=True, ragged=0):
    """maps: positions and slots of the packed rows are at hand (lrqk_pages_advance made them)."""
    return _named(name, dict(kind="write", B=B, Hq=Hq, Hkv=Hkv, n=n, l=l, page=page, kv=kv, pages=pages, layout=layout, rot=rot,
                             scaling=scaling, maps=maps, ragged=ragged))


def _rotate(name, T, Hq, Hkv, far, q="bf16", q_out="bf16", k="bf16", layout="halves", rot=128, scaling="none", back=False, packed=True):
    """T tokens at positions below `far`; packed: q and k are parts of one projection's rows."""
    return _named(name, dict(kind="rotate", T=T, Hq=Hq, Hkv=Hkv, far=far, q=q, q_out=q_out, k=k, layout=layout, rot=rot,
                             scaling=scaling, back=back, packed=packed))


def _advance(name, B, n, l, page, fresh, used, seed):
    """n new tokens at most of a running sequence, prompts of up to l in `fresh` of the B, `used` of the pool taken."""
    return _named(name, dict(kind="advance", B=B, n=n, l=l, page=page, fresh=fresh, used=used, spread=seed))


def _named(name, c):
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of one sequence over a short context: launches and latency
        _attend("attend_one_4k", 1, 32, 8, 1, 4096, 16),
        # a decode step of sixteen sequences of very different lengths: the stream of rows
        _attend("attend_decode_128k_b16", 16, 32, 8, 1, 131072, 64, ragged=11),
        # five drafted tokens of eight sequences to be verified, heads in groups of seven
        _attend("attend_draft_64k_b8", 8, 28, 4, 5, 65536, 32, ragged=12),
        # a chunk in the middle of a prompt of 32K
        _attend("attend_chunk_32k", 1, 32, 8, 2048, 32768, 64),
        # fp32 queries, odd sizes
        _attend("attend_chunk_f32_odd", 2, 28, 4, 1001, 5003, 16, "f32", ragged=14),
        # a layer's part of a decode step of sixteen sequences: latency
        _write("write_one_b16", 16, 32, 8, 1, 1000, 16, ragged=15),
        # prompts of several lengths into pages of 4 bits, scaled for long contexts
        _write("write_prompts_e2m1", 4, 32, 8, 8192, 8192, 64, pages="e2m1", scaling="bands", ragged=16),
        # fp32 rows, part of the head in pairs, odd sizes, positions from the tables
        _write("write_f32_pairs_odd", 3, 28, 4, 777, 2777, 32, "f32", "f32", "pairs", 68, "linear", maps=False, ragged=17),
        # the queries (wanted in fp32) and keys of a decode step of 64 sequences, far positions
        _rotate("rotate_decode_b64", 64, 32, 8, 1 << 20, q_out="f32", scaling="ramp"),
        # gradients of a long sequence's queries and keys turned back, half of the head in pairs
        _rotate("rotate_back_32k", 32768, 32, 8, 32768, layout="pairs", rot=64, back=True, packed=False),
        # a decode step of 256 sequences with drafts, some of them rejected, some requests at their end, some new
        _advance("advance_decode_b256", 256, 5, 4000, 16, 0.02, 0.8, 18),
        # prompts of several lengths into a pool that is nearly full
        _advance("advance_prompts_b24", 24, 2, 30000, 64, 0.5, 0.9, 19),
    ]


def draw(rng):
    spread = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    Hkv, G = rng.choice([(8, 4), (4, 7), (8, 1), (2, 8), (5, 3), (1, 5), (8, 2)])
    page, ragged = 1 << rng.randint(4, 8), rng.randint(1, 1 << 20)
    layout, scaling = rng.choice(["halves", "pairs"]), rng.choice(["none", "linear", "base", "bands", "ramp"])
    rot = rng.choice([128, 128, 64, 32, 96, 2 * rng.randint(2, 64)])
    kind = rng.choice(["one", "draft", "chunk", "write", "rotate", "advance"])
    if kind in ("one", "draft"):
        n = 1 if kind == "one" else rng.randint(2, 16)
        B = spread(1, 32)
        return _attend(None, B, Hkv * G, Hkv, n, n + spread(16, min(131072, 1000000 // B)), page, rng.choice(["bf16", "bf16", "f32"]), ragged)
    if kind == "chunk":
        kv = rng.choice(["bf16", "bf16", "f32"])
        B, n = spread(1, 8), spread(17, 2048)
        return _attend(None, B, Hkv * G, Hkv, n, n + spread(16, max(32, min(12000 if kv == "f32" else 40000, 60000000 // (B * n)))), page, kv, ragged)
    if kind == "write":
        kv, pages = rng.choice([("bf16", "bf16"), ("bf16", "e2m1"), ("bf16", "e4m3"), ("f32", "f32")])
        B, n = spread(1, 16), spread(1, 2048)
        return _write(None, B, Hkv * G, Hkv, n, n + spread(1, 4096), page, kv, pages, layout, rot, scaling, rng.random() < 0.5, ragged)
    if kind == "rotate":
        q, q_out = rng.choice([("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
        return _rotate(None, spread(1, 16384), Hkv * G, Hkv, spread(16, 1 << 22), q, q_out, q, layout, rot, scaling, rng.random() < 0.3, rng.random() < 0.5)
    return _advance(None, spread(1, 512), rng.randint(1, 8), spread(64, 20000), page, rng.choice([0.02, 0.3]), rng.uniform(0.3, 0.95), ragged)


def lengths(c):
    """New tokens and positions (the new ones among them) of each sequence."""
    if not c["ragged"]:
        return [c["n"]] * c["B"], [c["l"]] * c["B"]
    r = random.Random(c["ragged"])
    some = lambda top, by: int(round(top * by ** -r.random())) if top else 0  # noqa: E731
    n = [c["n"]] + [max(1, some(c["n"], 16.0)) for _ in range(c["B"] - 1)]
    old = [c["l"] - c["n"]] + [some(c["l"] - c["n"], 16.0) for _ in range(c["B"] - 1)]
    return n, [a + b for a, b in zip(n, old)]


def requests(c):
    """What an advance finds: each sequence's length, what it keeps of it, its new tokens; pages taken by others."""
    r = random.Random(c["spread"])
    ln, keep, new = [], [], []
    for b in range(c["B"]):
        if r.random() < c["fresh"] or b == c["B"] - 1:   # a prompt
            ln.append(0)
            keep.append(0)
            new.append(max(1, int(c["l"] * 16.0 ** -r.random())))
            continue
        x = max(1, int((c["l"] - c["n"]) * 16.0 ** -r.random()))
        end = r.random() < 0.05
        ln.append(x)
        keep.append(0 if end else max(0, x - r.randint(0, c["n"] - 1)))
        new.append(0 if end else r.randint(1, c["n"]))
    page = c["page"]
    held = sum(-(-x // page) for x in ln)
    wanted = sum(-(-(k + n) // page) + -(-x // page) for k, n, x in zip(keep, new, ln))
    n_pages = max(2 * wanted + 64, int(held / c["used"]))
    others = max(0, min(n_pages - wanted - 8, int(c["used"] * n_pages) - held))
    return ln, keep, new, n_pages, others


# ---- rotary positions: frequencies ---------------------------------------------------------------------------
BASE, FACTOR, LOW, HIGH, L_ORIG = 500000.0, 8.0, 1.0, 4.0, 8192


def frequencies(rot, scaling):
    """Radians a position of each of the rot / 2 pairs, and what the turned elements are multiplied by."""
    j = torch.arange(rot // 2, dtype=torch.float64)
    if scaling == "base":
        base = BASE * FACTOR ** (rot / (rot - 2)) if rot > 2 else BASE
        return base ** (-2 * j / rot), 1.0
    f = BASE ** (-2 * j / rot)
    if scaling == "linear":
        return f / FACTOR, 1.0
    if scaling == "bands":
        s = ((L_ORIG * f / (2 * math.pi) - LOW) / (HIGH - LOW)).clamp(0.0, 1.0)
        return f * (s + (1 - s) / FACTOR), 1.0
    if scaling == "ramp":
        at = lambda turns: rot * math.log(L_ORIG / (turns * 2 * math.pi)) / (2 * math.log(BASE))  # noqa: E731
        lo, hi = max(0, math.floor(at(HIGH))), min(rot // 2 - 1, math.ceil(at(LOW)))
        s = 1 - ((j - lo) / max(hi - lo, 0.001)).clamp(0.0, 1.0)
        return f * (s + (1 - s) / FACTOR), 0.1 * math.log(FACTOR) + 1.0
    return f, 1.0


def turn(x, pos, c, f, amplitude, back=False):
    """Rows x [T, H, D] in 32 bits, turned to positions pos [T]; the angles in 64 bits."""
    rot = c["rot"]
    a = pos.double()[:, None] * f[None, :]
    cos, sin = (amplitude * torch.cos(a)).float()[:, None, :], (amplitude * torch.sin(a)).float()[:, None, :]
    if back:
        sin = -sin
    y = x.float().clone()
    if c["layout"] == "halves":
        p, q = slice(0, rot // 2), slice(rot // 2, rot)
    else:
        p, q = slice(0, rot, 2), slice(1, rot, 2)
    u, v = y[..., p].clone(), y[..., q].clone()
    y[..., p] = u * cos - v * sin
    y[..., q] = v * cos + u * sin
    return y


# ---- rows of 4 and 8 bits in elementary operations -------------------------------------------------------------
def quantise(x, pages):
    """Codes (e2m1: two a byte) and scale bytes of rows x [..., D]."""
    x = x.float().unflatten(-1, (D // BLOCK, BLOCK))
    top = x.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(top / TOP[pages])     # top = TOP m 2^e up to rounding: settled by comparing
    e = torch.where(top <= torch.ldexp(torch.full_like(top, TOP[pages]), e - 1), e - 1, e)
    e = torch.where(top > torch.ldexp(torch.full_like(top, TOP[pages]), e), e + 1, e)
    e = torch.where(top > 0, e, torch.full_like(e, E_MIN)).clamp_min(E_MIN)
    x = torch.ldexp(x, -e)
    if pages == "e4m3":
        codes = x.to(torch.float8_e4m3fn).view(torch.uint8).flatten(-2)
    else:
        a, codes = x.abs(), torch.signbit(x).to(torch.uint8) * 8
        for i in range(1, 8):                # a tie goes to the even one of i - 1 and i
            mid = (STEPS[i - 1] + STEPS[i]) / 2
            codes += (a >= mid) if i % 2 == 0 else (a > mid)
        codes = codes.flatten(-2)
        codes = codes[..., 0::2] | codes[..., 1::2] << 4
    return codes, (e.squeeze(-1) + 127).to(torch.uint8)


def values(codes, scales, pages):
    """Rows in 32 bits from codes and scale bytes [..., D / BLOCK]."""
    if pages == "e4m3":
        x = codes.view(torch.float8_e4m3fn).float()
    else:
        table = torch.tensor(STEPS + tuple(-v for v in STEPS), device=codes.device)
        x = table[torch.stack((codes & 15, codes >> 4), dim=-1).flatten(-2).long()]
    return torch.ldexp(x.unflatten(-1, (D // BLOCK, BLOCK)), scales.int()[..., None] - 127).flatten(-2)


# ---- inputs --------------------------------------------------------------------------------------------------
def prepare(c, seed):
    g = torch.Generator(device=DEV).manual_seed(seed * 7919 + 29)
    return {"attend": _prepare_pages, "write": _prepare_pages, "rotate": _prepare_rotate, "advance": _prepare_advance}[c["kind"]](c, g)


def _rope(s, c, back=False):
    """The frequencies, and what a program keeps of them on the GPU."""
    f, s["amplitude"] = frequencies(c["rot"], c["scaling"])
    s["f"] = f.to(DEV)
    if own:
        import paper_2510_23649_amd as L
        kind = {"none": L.LRQK_ROPE_PLAIN, "linear": L.LRQK_ROPE_LINEAR, "base": L.LRQK_ROPE_BASE, "bands": L.LRQK_ROPE_BANDS,
                "ramp": L.LRQK_ROPE_RAMP}[c["scaling"]]
        turns, amplitude = L.lrqk_rope_turns(c["rot"], kind, base=BASE, factor=FACTOR, low=LOW, high=HIGH, l_orig=L_ORIG)
        s["rope"] = L.make_rope(turns=turns.to(DEV), rot=c["rot"], amplitude=amplitude, back=back,
                                layout=L.LRQK_ROPE_HALVES if c["layout"] == "halves" else L.LRQK_ROPE_PAIRS)


def _prepare_pages(c, g):
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
            pool, scale = torch.empty((n_pages, Hkv, page, D), dtype=TYPE[c["pages"]], device=DEV), None
        else:
            pool = torch.empty((n_pages, Hkv, page, D // 2 if c["pages"] == "e2m1" else D), dtype=torch.uint8, device=DEV)
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
        # rows of one projection: queries, keys, values
        qkv = torch.cat((rn(T, Hq, D), rn(T, Hkv, D) * size[:, 0], rn(T, Hkv, D) + mean[:, 0]), dim=1).to(kvt)
        s["q"], s["k_new"], s["v_new"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        s["q_out"] = torch.zeros((T, Hq, D), dtype=kvt, device=DEV)
        where = [torch.arange(b - a, b, device=DEV) for a, b in zip(n, ln)]
        s["pos"] = torch.cat(where).to(torch.int32)
        s["slot"] = torch.cat([table[b, p // page] * page + p % page for b, p in enumerate(where)]).to(torch.int32)
        if c["pages"] not in TYPE:
            s["K_out"] = torch.zeros((B, Hkv, c["l"], D), dtype=kvt, device=DEV)
            s["V_out"] = torch.zeros((B, Hkv, c["l"], D), dtype=kvt, device=DEV)
        _rope(s, c)
    if own:
        import paper_2510_23649_amd as L
        s["shape"] = L.PagesShape.make(
            B=B, Hq=Hq, Hkv=Hkv, T=T, n_max=c["n"], l_max=c["l"], page=page, n_pages=n_pages, max_pages=max_pages,
            kv_dtype={"bf16": L.LRQK_KV_BF16, "f32": L.LRQK_KV_F32}[c["kv"]],
            page_dtype={"bf16": L.LRQK_PAGE_BF16, "f32": L.LRQK_PAGE_F32, "e4m3": L.LRQK_PAGE_E4M3, "e2m1": L.LRQK_PAGE_E2M1}[c["pages"]])
        s["pages"] = L.make_pages(K=s["K"], V=s["V"], K_scale=s["K_scale"], V_scale=s["V_scale"], table=table,
                                  start=s["start"], kv_len=s["kv_len"])
        if c["kind"] == "attend":
            s["ws"] = torch.empty(max(256, L.lrqk_pages_workspace_bytes(s["shape"])), dtype=torch.uint8, device=DEV)
    return s


def _prepare_rotate(c, g):
    T, Hq, Hkv = c["T"], c["Hq"], c["Hkv"]
    s = dict(c=c, pos=torch.randint(0, c["far"], (T,), generator=g, device=DEV, dtype=torch.int32))
    if c["back"]:                            # a sequence's gradients: one token after the other
        s["pos"] = (torch.arange(T, device=DEV) % c["far"]).to(torch.int32)
    x = torch.randn((T, Hq + 2 * Hkv, D), generator=g, device=DEV)
    if c["packed"] and c["q"] == c["k"]:
        x = x.to(TYPE[c["q"]])
        s["q"], s["k"] = x[:, :Hq], x[:, Hq:Hq + Hkv]
    else:
        s["q"], s["k"] = x[:, :Hq].to(TYPE[c["q"]]).contiguous(), x[:, Hq:Hq + Hkv].to(TYPE[c["k"]]).contiguous()
    s["q_out"] = torch.zeros((T, Hq, D), dtype=TYPE[c["q_out"]], device=DEV)
    s["k_out"] = torch.zeros((T, Hkv, D), dtype=TYPE[c["k"]], device=DEV)
    _rope(s, c, c["back"])
    return s


def _prepare_advance(c, g):
    ln, keep, new, n_pages, others = requests(c)
    page, B = c["page"], c["B"]
    most = max(max(k + n for k, n in zip(keep, new)), max(ln))
    max_pages = -(-most // page) + 1
    used = [-(-x // page) for x in ln]
    ids = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    table, at = torch.full((B, max_pages), -1, dtype=torch.int32), 0
    own_ids = ids[:sum(used)].cpu()
    for b in range(B):
        table[b, :used[b]] = own_ids[at:at + used[b]]
        at += used[b]
    refs = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    refs[ids[:sum(used) + others].long()] = 1
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    T = sum(new) + 5                         # a captured step has room for more rows than it meets
    s = dict(c=c, refs=refs, table=table.to(DEV), kv_len=i32(ln), keep=i32(keep), n_new=i32(new), T=T, l_max=most, n_max=max(new),
             **{k: torch.zeros(m, dtype=torch.int32, device=DEV) for k, m in
                (("start", B + 1), ("status", B), ("seq", T), ("pos", T), ("slot", T))})
    if own:
        import paper_2510_23649_amd as L
        s["shape"] = L.PagesShape.make(B=B, Hq=8, Hkv=8, T=T, n_max=s["n_max"], l_max=most, page=page, n_pages=n_pages, max_pages=max_pages)
        s["tables"] = L.make_pages_tables(**{k: s[k] for k in ("refs", "table", "kv_len", "start", "status", "seq", "pos", "slot")})
        s["ws"] = torch.empty(L.lrqk_pages_advance_workspace_bytes(s["shape"]), dtype=torch.uint8, device=DEV)
    return s


# ---- one pass --------------------------------------------------------------------------------------------------
TABLES = ("refs", "table", "kv_len", "start", "status", "seq", "pos", "slot")


def run(s):
    c = s["c"]
    kind = c["kind"]
    if own:
        import paper_2510_23649_amd as L
        if kind == "attend":
            L.lrqk_chunk_attend(s["shape"], s["pages"], s["q"], s["out"], s["ws"])
            return s["out"]
        if kind == "rotate":
            L.lrqk_rotate(s["rope"], s["pos"], s["q"], s["q_out"], s["k"], s["k_out"])
            return s["q_out"], s["k_out"]
        if kind == "advance":
            L.lrqk_pages_advance(s["shape"], s["tables"], s["keep"], s["n_new"], s["ws"])
            return tuple(s[k] for k in TABLES)
        maps = dict(pos=s["pos"], slot=s["slot"]) if c["maps"] else {}
        L.lrqk_pages_rotate_append(s["shape"], s["pages"], s["rope"], s["q"], s["k_new"], s["v_new"], s["q_out"], **maps)
        if c["pages"] in TYPE:
            return s["q_out"], s["K"], s["V"]
        L.lrqk_pages_read(s["shape"], s["pages"], 0, s["K_out"], s["V_out"])
        return s["q_out"], s["K_out"], s["V_out"]
    if kind == "attend":
        return _plain_attend(s)
    if kind == "rotate":
        s["q_out"].copy_(turn(s["q"], s["pos"], c, s["f"], s["amplitude"], c["back"]))
        s["k_out"].copy_(turn(s["k"], s["pos"], c, s["f"], s["amplitude"], c["back"]))
        return s["q_out"], s["k_out"]
    if kind == "advance":
        return _plain_advance(s)
    return _plain_write(s)


def _rows(s, b, name):
    """Sequence b's rows in 32 bits, [Hkv, length, D]."""
    p = torch.arange(s["ln"][b], device=DEV)
    page = s["table"][b, p // s["c"]["page"]].long()
    x = s[name][page, :, p % s["c"]["page"]]
    return values(x, s[name + "_scale"][page, :, p % s["c"]["page"]], s["c"]["pages"]).transpose(0, 1)


def _plain_write(s):
    c = s["c"]
    s["q_out"].copy_(turn(s["q"], s["pos"], c, s["f"], s["amplitude"]))
    k = turn(s["k_new"], s["pos"], c, s["f"], s["amplitude"]).to(TYPE[c["kv"]])
    to, off = (s["slot"] // c["page"]).long(), (s["slot"] % c["page"]).long()
    for name, x in (("K", k), ("V", s["v_new"])):
        if c["pages"] in TYPE:
            s[name][to, :, off] = x.to(s[name].dtype)
        else:
            s[name][to, :, off], s[name + "_scale"][to, :, off] = quantise(x, c["pages"])
    if c["pages"] in TYPE:
        return s["q_out"], s["K"], s["V"]
    for b in range(c["B"]):
        s["K_out"][b, :, :s["ln"][b]] = _rows(s, b, "K")
        s["V_out"][b, :, :s["ln"][b]] = _rows(s, b, "V")
    return s["q_out"], s["K_out"], s["V_out"]


def _plain_advance(s):
    c, T = s["c"], s["T"]
    B, page, l_max = c["B"], c["page"], s["l_max"]
    pages = lambda x: (x + page - 1) // page  # noqa: E731
    i = torch.arange(s["table"].shape[1], device=DEV)[None, :]
    old, new = s["kv_len"].long().clamp(0, l_max), s["n_new"].long().clamp_min(0)
    keep = torch.minimum(s["keep"].long().clamp_min(0), old)
    gone = (i >= pages(keep)[:, None]) & (i < pages(old)[:, None])
    s["refs"].index_add_(0, torch.where(gone, s["table"], 0).flatten(), -gone.flatten().to(torch.int32))
    s["table"].masked_fill_(gone, -1)
    free = s["refs"] <= 0
    over = (new > s["n_max"]) | (keep + new > l_max)
    last = s["table"].gather(1, (pages(keep) - 1).clamp_min(0)[:, None])[:, 0].long().clamp_min(0)
    shared = (new > 0) & (keep % page != 0) & (s["refs"][last] > 1)
    fits = ~over & ~shared
    need = torch.where(fits, pages(keep + new) - pages(keep), 0)
    rows = torch.where(fits, new, 0)
    no_page = (need > 0) & (need.cumsum(0) > free.sum())
    no_row = (rows > 0) & (rows.cumsum(0) > T)
    status = torch.where(over, 1, torch.where(shared, 2, torch.where(no_page, 3, torch.where(no_row, 4, 0))))
    n = torch.where(status == 0, new, 0)
    s["status"].copy_(status)
    s["start"][1:] = n.cumsum(0)
    s["kv_len"].copy_(keep + n)
    need = torch.where(status == 0, need, 0)
    # the j-th page that is asked for is the j-th free one
    order = torch.argsort((~free).to(torch.uint8), stable=True).to(torch.int32)
    first = need.cumsum(0) - need
    j = i - pages(keep)[:, None]
    taken = (j >= 0) & (j < need[:, None])
    s["table"].copy_(torch.where(taken, order[(first[:, None] + j).clamp(0, order.numel() - 1)], s["table"]))
    s["refs"].copy_(torch.where(free & (free.cumsum(0) <= need.sum()), 1, s["refs"]))
    t = torch.arange(T, device=DEV)
    b = torch.searchsorted(s["start"][1:].long(), t, right=True)
    there, b = b < B, b.clamp_max(B - 1)
    pos = keep[b] + t - s["start"][b]
    s["seq"].copy_(torch.where(there, b, -1))
    s["pos"].copy_(torch.where(there, pos, -1))
    at = s["table"][b, torch.where(there, pos // page, 0)].long() * page + pos % page
    s["slot"].copy_(torch.where(there, at, -1))
    return tuple(s[k] for k in TABLES)


def _plain_attend(s):
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


# ---- the same from the definitions, in 64 bits -------------------------------------------------------------------
def _grid64(x, pages):
    """What rows x (float64) stand for once they are held in 4 or 8 bits."""
    shape = x.shape
    x = x.reshape(-1, BLOCK)
    top = x.abs().max(dim=1, keepdim=True).values
    unit = torch.exp2(torch.ceil(torch.log2(top.clamp_min(1e-300))) - (9 if pages == "e4m3" else 3) - 1)
    for _ in range(3):                       # up to the smallest power of two that holds the block
        unit = torch.where(top > TOP[pages] * unit, 2 * unit, unit)
    unit = unit.clamp_min(2.0 ** E_MIN)
    y = x / unit
    # bits behind the leading one: three, down to steps of 2^-9; one, down to steps of 1 / 2
    least, bits = (2.0 ** -6, 3) if pages == "e4m3" else (1.0, 1)
    ulp = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(least))) - bits)
    return (torch.round(y / ulp) * ulp * unit).reshape(shape)


def _turned64(x, pos, c, back=False):
    """Rows x [T, H, D] times the complex numbers of their positions."""
    f, amplitude = frequencies(c["rot"], c["scaling"])
    z = torch.polar(torch.full((1,), amplitude, dtype=torch.float64, device=DEV),
                    pos.double()[:, None] * f.to(DEV)[None, :] * (-1 if back else 1))[:, None, :]
    x, rot = x.double(), c["rot"]
    head, tail = x[..., :rot], x[..., rot:]
    pair = head.unflatten(-1, (2, rot // 2)).transpose(-1, -2) if c["layout"] == "halves" else head.unflatten(-1, (rot // 2, 2))
    y = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * z)
    y = y.transpose(-1, -2).flatten(-2) if c["layout"] == "halves" else y.flatten(-2)
    return torch.cat((y, tail), dim=-1)


def exact(c, seed):
    if c["kind"] == "advance":               # whole numbers
        return None
    s = prepare(c, seed)
    if c["kind"] == "rotate":
        return tuple(_turned64(s[k], s["pos"], c, c["back"]) for k in "qk")
    page = c["page"]
    where = lambda b, lo, hi: (s["table"][b].long().repeat_interleave(page)[lo:hi],  # noqa: E731
                               torch.arange(hi, device=DEV)[lo:] % page)

    def dense(b, name):
        pg, off = where(b, 0, s["ln"][b])
        x = s[name].permute(1, 0, 2, 3)[:, pg, off]
        if c["pages"] == "e4m3":
            x = x.view(torch.float8_e4m3fn).double()
        else:                                # a sign, two bits of exponent, one behind the leading one
            x = torch.stack((x % 16, x // 16), dim=-1).flatten(-2).long()
            e, m = x // 2 % 4, (x % 2).double()
            x = torch.where(e == 0, m / 2, torch.exp2(e.double() - 1) * (1 + m / 2)) * (1 - 2 * (x // 8)).double()
        sc = torch.exp2(s[name + "_scale"].permute(1, 0, 2, 3)[:, pg, off].double() - 127)
        return x * sc.repeat_interleave(BLOCK, dim=-1)

    if c["kind"] == "write":
        got = [_turned64(s["q"], s["pos"], c)]
        k = _turned64(s["k_new"], s["pos"], c)
        if c["pages"] not in TYPE:           # a key is one of the rows' own type before it is held in fewer bits
            k = k.to(TYPE[c["kv"]]).double()
        for name, x in (("K", k), ("V", s["v_new"].double())):
            at = 0
            o = s[name].double() if c["pages"] in TYPE else torch.zeros(c["B"], c["Hkv"], c["l"], D, dtype=torch.float64, device=DEV)
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
    e = {"bf16": 2.0, "f32": 4.0}
    if c["kind"] == "rotate":
        rows = c["T"] * D
        return {"bytes": rows * (c["Hq"] * (e[c["q"]] + e[c["q_out"]]) + 2 * c["Hkv"] * e[c["k"]]) + 4.0 * c["T"],
                "flops": 3.0 * c["T"] * (c["Hq"] + c["Hkv"]) * c["rot"]}
    if c["kind"] == "advance":
        ln, keep, new, _, _ = requests(c)
        taken = sum(-(-(k + n) // c["page"]) - -(-k // c["page"]) for k, n in zip(keep, new))
        return {"bytes": 4.0 * (6 * c["B"] + 3 * sum(new) + 4 * taken), "flops": 0.0}
    n, ln = lengths(c)
    row = D * e[c["kv"]]
    held = D * e[c["pages"]] if c["pages"] in e else D * (0.5 if c["pages"] == "e2m1" else 1.0) + D / BLOCK
    index = 4.0 * (2 * c["B"] + 1) + 4.0 * sum(-(-x // c["page"]) for x in ln)
    if c["kind"] == "attend":
        seen = sum(a * (b - a) + a * (a + 1) / 2 for a, b in zip(n, ln))
        return {"bytes": 2 * sum(n) * c["Hq"] * row + 2 * sum(ln) * c["Hkv"] * held + index, "flops": 4.0 * D * c["Hq"] * seen}
    wrote = sum(n) * (2 * c["Hq"] * row + 2 * c["Hkv"] * (row + held))
    back = 0.0 if c["pages"] in e else 2 * sum(ln) * c["Hkv"] * (held + row)
    return {"bytes": wrote + back + index, "flops": 3.0 * sum(n) * (c["Hq"] + c["Hkv"]) * c["rot"]}

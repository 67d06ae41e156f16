"""Cases and plain forms of the operators around a paged nugget cache and rotary positions:

  rope           rotary positions of a packed batch's queries and keys
  rope_backward  its gradient: what arrives at the rotated queries and keys, turned back
  append         selected K/V rows (or all of them) appended to a paged cache, K rotated at its position on the way
  attend         attention of new tokens (a chunk or single ones) over a paged cache and uncompressed local tokens; query heads
                 may share KV heads

A case is one batch of one layer: per-sequence lengths as text ("205x8" is eight sequences of 205, "3,0,17" three sequences).
``run`` is one pass through one operator, as a program that serves or trains one layer calls it.

Row r of sequence b lies in row r % page of page ``table[first_entry_of_b + r // page]``.  Feature pair i of a head is turned by
position x freq[i]; pairs are (i, i + rot / 2) ("half") or (2 i, 2 i + 1) ("interleaved") of the head's first ``rot`` features.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_context = []


# ---- cases ------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # one decode step of 8 sequences at 7B heads: the smallest call there is, all latency
        dict(name="rope_token", op="rope", dtype="bf16", H=32, Hkv=32, dh=128, rot=128, layout="half", scaling="plain", factor=1.0, n="1x8", pos=2112),
        # a prompt of 16,384 tokens at 13B heads
        dict(name="rope_prompt", op="rope", dtype="bf16", H=40, Hkv=40, dh=128, rot=128, layout="half", scaling="linear", factor=4.0, n="16384", pos=0),
        # ragged fp32 batch, neighbouring pairs, part of the head, far positions
        dict(name="rope_ragged_f32", op="rope", dtype="f32", H=12, Hkv=4, dh=64, rot=24, layout="interleaved", scaling="base", factor=8.0,
             n="1639,70,0,33,1,407", pos=1000000),
        # training: gradients of blocks of 256 queries and the 1280 tokens before and in them
        dict(name="rope_backward_block", op="rope_backward", dtype="bf16", H=32, Hkv=32, dh=128, rot=128, layout="interleaved", scaling="parts",
             factor=8.0, n="1280x4", pos=7168),
        # one decode step of 8 sequences: one row each, all latency
        dict(name="append_token", op="append", dtype="bf16", H=32, dh=128, rot=128, layout="half", scaling="plain", factor=1.0, n="1x8", nug="1x8",
             used="205x8", page=16, all=True, pos=2112),
        # a compressed context of 8 sequences (ratio 10, 7B heads) appended to an empty cache
        dict(name="append_nuggets", op="append", dtype="bf16", H=32, dh=128, rot=128, layout="half", scaling="plain", factor=1.0, n="2048x8", nug="205x8",
             used="0x8", page=16, all=False, pos=0),
        # the smallest layer of the configurations: 16 fp32 queries over 52 nuggets and, causally, themselves
        dict(name="attend_tiny_f32", op="attend", dtype="f32", H=4, Hkv=4, dh=64, tq="16", nug="52", loc="16", page=16, inside=False),
        # single-token decode, ratio 10, 64-token window (7B heads)
        dict(name="attend_token", op="attend", dtype="bf16", H=32, Hkv=32, dh=128, tq="1x8", nug="205x8", loc="64x8", page=16, inside=False),
        # decode over a long uncompressed-length cache (13B heads, ratio 1)
        dict(name="attend_token_long", op="attend", dtype="bf16", H=40, Hkv=40, dh=128, tq="1", nug="16384", loc="64", page=64, inside=False),
        # ragged serving batch, contexts of 512 to 32768 tokens at ratio 1 to 10, four query heads a KV head
        dict(name="attend_token_shared", op="attend", dtype="bf16", H=32, Hkv=8, dh=128, tq="1x16",
             nug="520,32770,970,12110,6400,710,2330,18900,4100,580,1330,8120,26500,3050,1800,770", loc="64,1,127,30,90,64,0,12,100,64,3,77,128,64,5,41",
             page=32, inside=False),
        # a chunk of 256 queries over a compressed past and 1024 + 256 uncompressed tokens
        dict(name="attend_chunk", op="attend", dtype="bf16", H=32, Hkv=8, dh=128, tq="256x4", nug="717x4", loc="1280x4", page=16, inside=False),
        # a prompt's next 512 tokens, already appended to a cache that nothing was dropped from (13B heads)
        dict(name="attend_chunk_long", op="attend", dtype="bf16", H=40, Hkv=40, dh=128, tq="512", nug="16896", loc="0", page=64, inside=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _text(v):
    return ",".join(str(int(x)) for x in v)


def draw(rng):
    op = rng.choice(["rope", "rope_backward", "append", "attend", "attend", "attend"])
    dtype, B = rng.choice(["bf16", "bf16", "bf16", "f32"]), rng.randint(1, 8)
    Hkv = rng.randint(1, 40)
    group = rng.choice([1, 1, 2, 3, 4, 7, 8])
    while Hkv * group > 64:
        Hkv = (Hkv + 1) // 2
    case = dict(op=op, dtype=dtype, H=Hkv * group, page=rng.choice([1, 8, 16, 16, 24, 32, 64, 128, 256]))
    if op in ("rope", "rope_backward", "append"):
        dh = rng.choice([64, 80, 96, 128, 128, 256])
        rot = rng.choice([dh, dh, dh // 2, 2 * rng.randint(1, dh // 2)])
        scaling = rng.choice(["plain", "linear", "base", "parts"])
        case.update(dh=dh, rot=rot, layout=rng.choice(["half", "interleaved"]), scaling=scaling,
                    factor=1.0 if scaling == "plain" else rng.choice([2.0, 4.0, 8.0, 32.0]), pos=rng.choice([0, _log(rng, 1, 1 << 20)]))
        hi = rng.choice([1, 64, 16384 // B])
        n = [_log(rng, 1, hi) if rng.random() > 0.1 else 0 for _ in range(B)]
        if sum(n) == 0:
            n[0] = 1
        while sum(n) * case["H"] * dh > 16384 * 40 * 64:
            n = [(k + 1) // 2 for k in n]
        if op == "append":
            case["H"] = Hkv
            every = rng.random() < 0.4
            nug = n if every else [(k + 3) // rng.randint(4, 20) if k > 3 else min(k, 1) for k in n]
            if sum(nug) == 0:
                n[0] = nug[0] = 1
            case.update(nug=_text(nug), used=_text(rng.choice([0, 0, 1, 33, 256]) for _ in n), all=every)
        else:
            case["Hkv"] = Hkv
        case["n"] = _text(n)
        return case
    dh = rng.choice([128, 128, 64])
    tq = rng.choice([1, 1, 1, 2, 5, 16, _log(rng, 17, 512)])
    tqs = [max(1, tq - rng.randint(0, tq // 3)) if tq > 1 else 1 for _ in range(B)]
    nug = [_log(rng, 1, 32768 // B) if rng.random() > 0.1 else 0 for _ in range(B)]
    loc = [t + _log(rng, 1, 1024) if rng.random() > 0.2 else t for t in tqs]
    cached = rng.random() < 0.3                            # the chunk's own rows lie in the cache, no local tokens
    pairs = 512 * 16896 * 40 * 128 // (32 if dtype == "f32" else 8 if dh == 64 else 2)
    while sum(t * (k + n) for t, k, n in zip(tqs, nug, loc)) * case["H"] * dh > pairs or sum(nug) * Hkv * dh > 16384 * 40 * 128:
        tqs, nug = [max(1, t * 3 // 4) for t in tqs], [k // 2 for k in nug]
        loc = [max(t, n * 3 // 4) for t, n in zip(tqs, loc)]
    if cached:
        nug, loc = [k + t for k, t in zip(nug, tqs)], [0] * B
    case.update(Hkv=Hkv, dh=dh, tq=_text(tqs), nug=_text(nug), loc=_text(loc), inside=not cached and rng.random() < 0.25)
    return case


def _ints(text):
    out = []
    for part in text.split(","):
        value, _, times = part.partition("x")
        out += [int(value)] * (int(times) if times else 1)
    return out


def _offsets(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


# ---- inputs -----------------------------------------------------------------------------------------------------------
BASE, TRAINED, LOW, HIGH = 10000.0, 4096, 1.0, 32.0


def _frequencies(case):
    """Radians per position of each feature pair, in 64 bits."""
    rot, factor, scaling = case["rot"], case["factor"], case["scaling"]
    base = BASE * factor ** (rot / (rot - 2)) if scaling == "base" and rot > 2 else BASE
    f = base ** (-2.0 * np.arange(rot // 2) / rot)
    if scaling == "linear":
        f = f / factor
    if scaling == "parts":            # pairs that turn often over the trained length keep their speed, slow ones are slowed down
        keep = np.clip((TRAINED * f / (2.0 * math.pi) - LOW) / (HIGH - LOW), 0.0, 1.0)
        f = f * (keep + (1.0 - keep) / factor)
    return f


def _amplitude(case):
    return 0.1 * math.log(case["factor"]) + 1.0 if case["scaling"] == "parts" else 1.0


def _rope(case):
    """The rotation as the framework's calls take it."""
    from paper_2310_02409_b200 import api
    kind = {"plain": api.ROPE_PLAIN, "linear": api.ROPE_LINEAR, "base": api.ROPE_BASE, "parts": api.ROPE_PARTS}[case["scaling"]]
    freq = api.rope_frequencies(case["rot"], BASE, kind, case["factor"], TRAINED, LOW, HIGH)
    return api.Rope(freq, api.ROPE_HALF if case["layout"] == "half" else api.ROPE_INTERLEAVED, _amplitude(case))


def _cache(s):
    """The cache's arrays and page table as a program that serves from it keeps them."""
    from paper_2310_02409_b200 import api
    return api.PagedCache(s["cacheK"], s["cacheV"], s["cache_pos"], s["page_table"])


def _randn(g, shape, dtype):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(dtype)


def _positions(g, k, span):
    """k ascending distinct positions out of [0, span)."""
    return torch.sort(torch.randperm(span, generator=g, device=DEV)[:k]).values


def _pages(s, g, rows, page):
    """A page table for sequences of so many rows, in a pool with pages to spare, and the pool's row of each of them."""
    need = [-(-r // page) for r in rows]
    pool = sum(need) + 3
    s["page"], s["pool"] = page, pool
    s["page_off"] = _offsets(need)
    s["page_table"] = torch.randperm(pool, generator=g, device=DEV)[:sum(need)].to(torch.int32)
    at = [torch.arange(r, device=DEV) for r in rows]
    s["row"] = torch.cat([s["page_table"][int(o) + a // page].long() * page + a % page for o, a in zip(s["page_off"], at)])


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1_000_003 + 29)
    dtype, dh = TYPES[case["dtype"]], case["dh"]
    s = dict(op=case["op"], dtype=dtype, H=case["H"], Hkv=case.get("Hkv", case["H"]), dh=dh)
    if s["op"] != "attend":
        n = _ints(case["n"])
        s.update(rot=case["rot"], layout=case["layout"], freq=_frequencies(case), amplitude=_amplitude(case), off=_offsets(n),
                 pos0=np.asarray([case["pos"] + 7 * b for b in range(len(n))], np.int32))
        if own:
            s["rope"] = _rope(case)
        if s["op"] != "append":
            s["Q"], s["K"] = _randn(g, (sum(n), s["H"], dh), dtype), _randn(g, (sum(n), s["Hkv"], dh), dtype)
            s["pos"] = torch.cat([torch.arange(k, device=DEV) + int(p) for k, p in zip(n, s["pos0"])])
            return s
        nug, used = _ints(case["nug"]), _ints(case["used"])
        s["K"], s["V"] = _randn(g, (sum(n), s["H"], dh), dtype), _randn(g, (sum(n), s["H"], dh), dtype)
        s["used"], s["nug_off"] = np.asarray(used, np.int32), _offsets(nug)
        idx = [torch.arange(k, device=DEV) if case["all"] else _positions(g, k, m) for k, m in zip(nug, n)]
        s["idx"] = None if case["all"] else torch.cat(idx).to(torch.int32)
        _pages(s, g, [k + u for k, u in zip(nug, used)], case["page"])
        s["src"] = torch.cat([i + int(o) for i, o in zip(idx, s["off"])])
        first = _offsets([k + u for k, u in zip(nug, used)])
        s["dst"] = s["row"][torch.cat([torch.arange(k, device=DEV) + int(o) + u for k, o, u in zip(nug, first, used)])]
        s["pos"] = torch.cat([i + int(p) for i, p in zip(idx, s["pos0"])])
        shape = (s["pool"], case["page"], s["H"], dh)
        s["cacheK"], s["cacheV"] = _randn(g, shape, dtype), _randn(g, shape, dtype)
        s["cache_pos"] = torch.full(shape[:2], -1, dtype=torch.int32, device=DEV)
        if own:
            s["cache"] = _cache(s)
        return s
    tq, nug, loc = _ints(case["tq"]), _ints(case["nug"]), _ints(case["loc"])
    B = len(tq)
    _pages(s, g, nug, case["page"])
    cached = sum(loc) == 0                             # the new tokens' own rows lie in the cache, nothing was dropped
    span = nug if cached else [10 * k for k in nug]    # otherwise nuggets are chosen out of ten times as many tokens
    pos = torch.cat([_positions(g, k, m) for k, m in zip(nug, span)]).to(torch.int32)
    if case["inside"]:                                 # queries inside the context: some nuggets, or all, lie ahead of them
        q_pos0 = [m * (2 * b + 1) // (2 * B + 2) for b, m in enumerate(span)]
    else:                                              # queries are the last tokens
        q_pos0 = [m + n - t for m, n, t in zip(span, loc, tq)]
    shape = (s["pool"], case["page"], s["Hkv"], dh)
    s["cacheK"], s["cacheV"] = _randn(g, shape, dtype), _randn(g, shape, dtype)
    s["cache_pos"] = torch.full((shape[0] * shape[1],), 2 ** 31 - 1, dtype=torch.int32, device=DEV)
    s["cache_pos"][s["row"]] = pos
    s["cache_pos"] = s["cache_pos"].view(shape[:2])
    if own:
        s["cache"] = _cache(s)
    s.update(scale=dh ** -0.5, q_off=_offsets(tq), q_pos0=np.asarray(q_pos0, np.int32), cache_len=np.asarray(nug, np.int32), loc_off=_offsets(loc),
             loc_len=np.asarray(loc, np.int32), loc_pos0=np.asarray(span, np.int32))
    s["Q"] = _randn(g, (sum(tq), s["H"], dh), dtype)
    s["locK"], s["locV"] = _randn(g, (sum(loc), s["Hkv"], dh), dtype), _randn(g, (sum(loc), s["Hkv"], dh), dtype)
    # index tables of the padded form
    first, T, L = _offsets(nug), max(tq), max(k + n for k, n in zip(nug, loc))
    q_row, q_pos = np.zeros((B, T), np.int64), np.full((B, T), -1, np.int64)
    k_row, k_pos = np.zeros((B, L), np.int64), np.full((B, L), 2 ** 31 - 1, np.int64)
    at_q, host, total = np.zeros(sum(tq), np.int64), pos.cpu().numpy(), sum(nug)
    for b in range(B):
        q_row[b, :tq[b]] = s["q_off"][b] + np.arange(tq[b])
        q_pos[b, :tq[b]] = q_pos0[b] + np.arange(tq[b])
        at_q[s["q_off"][b]:s["q_off"][b + 1]] = b * T + np.arange(tq[b])
        k_row[b, :nug[b]] = first[b] + np.arange(nug[b])
        k_pos[b, :nug[b]] = host[first[b]:first[b + 1]]
        k_row[b, nug[b]:nug[b] + loc[b]] = total + s["loc_off"][b] + np.arange(loc[b])
        k_pos[b, nug[b]:nug[b] + loc[b]] = span[b] + np.arange(loc[b])
    for name, v in (("q_row", q_row), ("q_pos", q_pos), ("k_row", k_row), ("k_pos", k_pos), ("at_q", at_q)):
        s[name] = torch.from_numpy(v).to(DEV)
    return s


# ---- plain forms ------------------------------------------------------------------------------------------------------
def _turn(s, x, pos, back=False):
    """x [rows, heads, dh] with its first features turned by pos x freq (angles in 64 bits), as x's type."""
    f = torch.from_numpy(s["freq"]).to(DEV)
    angle = torch.remainder(pos.double()[:, None] * f, 2.0 * math.pi)
    c, n = torch.cos(angle).float()[:, None] * s["amplitude"], torch.sin(angle).float()[:, None] * s["amplitude"]
    if back:
        n = -n
    y, half, rot = x.float(), s["rot"] // 2, s["rot"]
    a, b = (y[..., :half], y[..., half:rot]) if s["layout"] == "half" else (y[..., 0:rot:2], y[..., 1:rot:2])
    p, q = a * c - b * n, a * n + b * c
    turned = torch.cat([p, q], -1) if s["layout"] == "half" else torch.stack([p, q], -1).flatten(-2)
    return torch.cat([turned, y[..., rot:]], -1).to(x.dtype)


def _plain(s):
    if s["op"] in ("rope", "rope_backward"):
        back = s["op"] == "rope_backward"
        return {"Q": _turn(s, s["Q"], s["pos"], back), "K": _turn(s, s["K"], s["pos"], back)}
    if s["op"] == "append":
        K, V, pos = s["cacheK"].clone(), s["cacheV"].clone(), s["cache_pos"].clone()
        K.flatten(0, 1)[s["dst"]] = _turn(s, s["K"][s["src"]], s["pos"])
        V.flatten(0, 1)[s["dst"]] = s["V"][s["src"]]
        pos.view(-1)[s["dst"]] = s["pos"].to(torch.int32)
        return {"K": K, "V": V, "cache_pos": pos}
    rows = lambda cache, loc: torch.cat([cache.flatten(0, 1)[s["row"]], loc])[s["k_row"]].float()  # noqa: E731
    q, k, v = s["Q"][s["q_row"]].float().unflatten(2, (s["Hkv"], -1)), rows(s["cacheK"], s["locK"]), rows(s["cacheV"], s["locV"])
    see = (s["k_pos"][:, None, :] <= s["q_pos"][:, :, None])[:, None, None]
    x = torch.einsum("bqhgd,bkhd->bhgqk", q, k) * s["scale"]
    x = torch.where(see, x, torch.full_like(x, -math.inf))
    top = x.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    lse = (torch.log(total) + top)[..., 0].permute(0, 3, 1, 2).flatten(2)
    o = torch.einsum("bhgqk,bkhd->bqhgd", p / torch.where(total > 0, total, torch.ones_like(total)), v).flatten(2, 3)
    return {"O": o.flatten(0, 1)[s["at_q"]].to(s["dtype"]), "lse": lse.flatten(0, 1)[s["at_q"]]}


# ---- the framework's calls --------------------------------------------------------------------------------------------
def _new(s, name, shape, dtype):
    """A buffer that the program keeps from call to call."""
    if name not in s:
        s[name] = torch.empty(shape, dtype=dtype, device=DEV)
    return s[name]


def _called(s):
    if not _context:
        from paper_2310_02409_b200 import api
        _context.append(api.Dodo(0))
    dodo = _context[0]
    if s["op"] in ("rope", "rope_backward"):
        outQ, outK = _new(s, "outQ", s["Q"].shape, s["dtype"]), _new(s, "outK", s["K"].shape, s["dtype"])
        call = dodo.rope if s["op"] == "rope" else dodo.rope_backward
        call(s["rope"], s["off"], s["pos0"], s["Q"], s["K"], outQ, outK)
        return {"Q": outQ, "K": outK}
    if s["op"] == "append":
        used = s["used"].copy()
        dodo.gather_kv_paged(s["K"], s["V"], s["off"], s["idx"], s["nug_off"], s["pos0"], s["rope"], s["cache"], s["page_off"], used)
        return {"K": s["cacheK"], "V": s["cacheV"], "cache_pos": s["cache_pos"]}
    if "workspace" not in s:
        s["workspace"] = torch.empty(dodo.attend_paged_workspace_bytes(s["dh"]), dtype=torch.uint8, device=DEV)
    O, lse = _new(s, "O", s["Q"].shape, s["dtype"]), _new(s, "lse", s["Q"].shape[:2], torch.float32)
    dodo.attend_paged(s["Q"], s["q_off"], s["q_pos0"], s["scale"], s["cache"], s["page_off"], s["cache_len"], s["locK"], s["locV"],
                      s["loc_off"][:-1], s["loc_len"], s["loc_pos0"], O, lse, s["workspace"])
    return {"O": O, "lse": lse}


def run(state):
    return _called(state) if own else _plain(state)


# ---- what a pass cannot do without ------------------------------------------------------------------------------------
def work(case):
    dh, e, H = case["dh"], 2 if case["dtype"] == "bf16" else 4, case["H"]
    Hkv = case.get("Hkv", H)
    if case["op"] in ("rope", "rope_backward"):        # rows read and written
        n = sum(_ints(case["n"]))
        return {"bytes": 2 * n * (H + Hkv) * dh * e, "flops": 3 * n * (H + Hkv) * case["rot"]}
    nug = _ints(case["nug"])
    if case["op"] == "append":                         # K and V rows read and written, the index read, the position written
        k = sum(nug)
        pages = sum(-(-(u + n) // case["page"]) - u // case["page"] for u, n in zip(_ints(case["used"]), nug) if n)
        return {"bytes": k * (4 * H * dh * e + (4 if case["all"] else 8)) + 4 * pages, "flops": 3 * k * H * case["rot"]}
    tq, loc = _ints(case["tq"]), _ints(case["loc"])
    pairs = 0
    for t, k, n in zip(tq, nug, loc):                  # visible (query, key) pairs; inside the context about half of the nuggets
        own_rows = t * (t + 1) // 2 if n or sum(loc) == 0 else 0
        pairs += t * k // 2 if case["inside"] else t * (k + n - (t if own_rows else 0)) + own_rows
    rows = sum(nug) + sum(loc)
    return {"bytes": rows * 2 * Hkv * dh * e + sum(nug) * 4 + sum(-(-k // case["page"]) for k in nug) * 4 + sum(tq) * (2 * H * dh * e + 4 * H),
            "flops": 4 * pairs * H * dh}


# ---- the same in 64 bits, row by row or head by head ------------------------------------------------------------------
def _turned64(s, x, pos, sign):
    """The rotation as a product with the complex numbers amplitude * exp(i sign angle)."""
    z = x.double()
    turn = torch.polar(torch.full((pos.shape[0], s["rot"] // 2), s["amplitude"], dtype=torch.float64, device=DEV),
                       sign * pos.double()[:, None] * torch.from_numpy(s["freq"]).to(DEV))[:, None]
    y, rot = z.clone(), s["rot"]
    at = (slice(0, rot // 2), slice(rot // 2, rot)) if s["layout"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    pair = torch.complex(z[..., at[0]], z[..., at[1]]) * turn
    y[..., at[0]], y[..., at[1]] = pair.real, pair.imag
    return y


def exact(case, seed):
    s = prepare(case, seed)
    if s["op"] in ("rope", "rope_backward"):
        sign = 1.0 if s["op"] == "rope" else -1.0
        return {"Q": _turned64(s, s["Q"], s["pos"], sign), "K": _turned64(s, s["K"], s["pos"], sign)}
    if s["op"] == "append":
        K, V = s["cacheK"].double(), s["cacheV"].double()
        K.flatten(0, 1)[s["dst"]], V.flatten(0, 1)[s["dst"]] = _turned64(s, s["K"][s["src"]], s["pos"], 1.0), s["V"][s["src"]].double()
        return {"K": K, "V": V, "cache_pos": None}
    O = torch.zeros(s["Q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(s["Q"].shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    first, cacheK, cacheV, cpos = _offsets(s["cache_len"]), s["cacheK"].flatten(0, 1), s["cacheV"].flatten(0, 1), s["cache_pos"].view(-1)
    for b in range(len(s["q_off"]) - 1):
        rows, q = s["row"][int(first[b]):int(first[b + 1])], slice(int(s["q_off"][b]), int(s["q_off"][b + 1]))
        l0, n = int(s["loc_off"][b]), int(s["loc_len"][b])
        pos = torch.cat([cpos[rows].long(), int(s["loc_pos0"][b]) + torch.arange(n, device=DEV)])
        hidden = pos[None, :] > int(s["q_pos0"][b]) + torch.arange(q.stop - q.start, device=DEV)[:, None]
        if pos.numel() == 0:
            continue
        for h in range(s["H"]):
            kv = h * s["Hkv"] // s["H"]
            K = torch.cat([cacheK[rows, kv], s["locK"][l0:l0 + n, kv]]).double()
            V = torch.cat([cacheV[rows, kv], s["locV"][l0:l0 + n, kv]]).double()
            logit = (s["Q"][q, h].double() @ K.T * s["scale"]).masked_fill(hidden, -math.inf)
            lse[q, h] = torch.logsumexp(logit, 1)
            O[q, h] = torch.exp(logit - lse[q, h][:, None]).masked_fill(hidden, 0.0) @ V
    return {"O": O, "lse": lse}

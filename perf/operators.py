"""Cases and plain forms of four operators around attention over [nuggets ; local tokens]:

  attend_backward   gradients of ``attend`` with respect to Q, the nugget rows, the local rows and, through the
                    straight-through estimator (Eq. 16-18), the nuggets' scores
  gather_q4         selected K/V rows appended to a nugget cache held in 4 bits, and the cache read back
  expand_q4         the rows of a 4-bit nugget cache as K and V rows of a floating type
  attend_q4         attention over a 4-bit nugget cache and uncompressed local tokens

A case is one batch: per-sequence lengths as text ("205x8" is eight sequences of 205, "3,0,17" three sequences).
``run`` is one pass through one operator, as a program that serves or trains one layer calls it.

The 4-bit format: a row of one head is cut into groups of 32 features; a group keeps a bf16 minimum m (rounded down) and
a bf16 step s (the smallest bf16 number with m + 15 s >= the group's maximum), and a feature the 4-bit code
c = round((x - m) / s), ties to even: it stands for m + c s, at most half a step off.
"""
import math

import numpy as np
import torch

own = False

GROUP = 32
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_context = []


# ---- cases ------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # training, the smallest layer of the configurations: 16 fp32 queries over 52 nuggets and, causally, themselves
        dict(name="backward_tiny_f32", op="attend_backward", dtype="f32", H=4, dh=64, tq="16", nug="52", loc="16", inside=False),
        # a single query token per sequence, 205 nuggets and a 64-token window (7B heads): all traffic, no reuse
        dict(name="backward_token", op="attend_backward", dtype="bf16", H=32, dh=128, tq="1x8", nug="205x8", loc="64x8", inside=False),
        # training of the autoregressive mode: blocks of 256 tokens, the past at ratio 10, 1024 uncompressed tokens before them
        dict(name="backward_block", op="attend_backward", dtype="bf16", H=32, dh=128, tq="256x4", nug="717x4", loc="1280x4", inside=False),
        # 13B heads, nothing compressed (ratio 1): 512 queries over 16,384 rows and themselves
        dict(name="backward_long", op="attend_backward", dtype="bf16", H=40, dh=128, tq="512", nug="16384", loc="512", inside=False),
        # appending a compressed context of 8 sequences (ratio 10) to an empty 4-bit cache, then reading it back
        dict(name="gather_q4_batch", op="gather_q4", dtype="bf16", H=32, dh=128, n="2048x8", nug="205x8", used="0x8"),
        # a ragged batch, fp32 storage, appended behind rows that are already there
        dict(name="gather_q4_ragged_f32", op="gather_q4", dtype="f32", H=12, dh=64, n="16384,700,33,4097", nug="1639,70,33,1", used="5,0,64,300"),
        # a long sequence's cache (ratio 5) read back for a block of queries
        dict(name="expand_q4_long", op="expand_q4", dtype="bf16", H=40, dh=128, nug="3277", cap="3300"),
        # a small ragged cache, fp32
        dict(name="expand_q4_ragged_f32", op="expand_q4", dtype="f32", H=8, dh=64, nug="17,0,205,1", cap="32,8,205,40"),
        # single-token decode, ratio 10, 64-token window (7B heads): the smallest call that serving makes
        dict(name="attend_q4_token", op="attend_q4", dtype="bf16", H=32, dh=128, tq="1x8", nug="205x8", loc="64x8", inside=False, lse=True),
        # decode over a long uncompressed-length cache (13B heads, ratio 1)
        dict(name="attend_q4_long", op="attend_q4", dtype="bf16", H=40, dh=128, tq="1", nug="16384", loc="64", inside=False, lse=True),
        # ragged serving batch, contexts of 512 to 32768 tokens at ratio 10
        dict(name="attend_q4_ragged", op="attend_q4", dtype="bf16", H=32, dh=128, tq="1x16",
             nug="52,3277,97,1211,640,71,233,1890,410,58,133,812,2650,305,180,77", loc="64,1,127,30,90,64,0,12,100,64,3,77,128,64,5,41",
             inside=False, lse=True),
        # a block of 256 queries over a 4-bit past and 1024 + 256 uncompressed tokens
        dict(name="attend_q4_block", op="attend_q4", dtype="bf16", H=32, dh=128, tq="256x4", nug="717x4", loc="1280x4", inside=False, lse=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _text(v):
    return ",".join(str(int(x)) for x in v)


def draw(rng):
    op = rng.choice(["attend_backward", "attend_backward", "gather_q4", "expand_q4", "attend_q4", "attend_q4"])
    dtype, dh, H = rng.choice(["bf16", "bf16", "bf16", "f32"]), rng.choice([128, 128, 64]), rng.randint(1, 40)
    B = rng.randint(1, 8)
    case = dict(op=op, dtype=dtype, H=H, dh=dh)
    if op in ("gather_q4", "expand_q4"):
        hi = 16384 if B < 3 else 2048
        nug = [_log(rng, 1, hi) if rng.random() > 0.1 else 0 for _ in range(B)]
        if sum(nug) == 0:
            nug[0] = 1
        budget = (3277 if op == "expand_q4" else 1639) * 40 * 128
        while sum(nug) * H * dh > budget:
            nug = [(k + 1) // 2 for k in nug]
        if op == "expand_q4":
            case.update(nug=_text(nug), cap=_text(k + rng.randint(0, 40) for k in nug))
        else:
            ratio = rng.randint(1, 20)
            case.update(n=_text(max(k, k * ratio - rng.randint(0, ratio - 1)) for k in nug), nug=_text(nug),
                        used=_text(rng.choice([0, 0, 1, 33, 256]) for _ in nug))
        return case
    # attention: the lengths are cut until the pairs of (query, key) cost no more than the largest listed case
    tq = _log(rng, 1, 512) if op == "attend_backward" else rng.choice([1, 1, 1, 2, 5, 16, _log(rng, 32, 256)])
    tqs = [max(1, tq - rng.randint(0, tq // 3)) if tq > 1 else 1 for _ in range(B)]
    nug = [_log(rng, 1, 16384 // B) if rng.random() > 0.1 else 0 for _ in range(B)]
    loc = [t + _log(rng, 1, 1024) if rng.random() > 0.2 else t for t in tqs]
    if op == "attend_backward":
        budget = 512 * 16384 * 40 * 128 // (16 if dtype == "f32" or dh == 64 else 1)
    else:
        budget = (16384 * 40 * 128 if max(tqs) == 1 else 256 * 2000 * 32 * 128 * 4 // (8 if dtype == "f32" or dh == 64 else 1))
    while sum(t * (k + n) for t, k, n in zip(tqs, nug, loc)) * H * dh > budget:
        tqs, nug = [max(1, t * 3 // 4) for t in tqs], [k // 2 for k in nug]
        loc = [max(t, n * 3 // 4) for t, n in zip(tqs, loc)]
    case.update(tq=_text(tqs), nug=_text(nug), loc=_text(loc), inside=rng.random() < 0.25)
    if op == "attend_q4":
        case["lse"] = max(tqs) < 32
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
def _randn(g, shape, dtype, std=1.0):
    return (torch.randn(shape, generator=g, device=DEV, dtype=torch.float32) * std).to(dtype)


def _positions(g, k, span):
    """k ascending distinct positions out of [0, span)."""
    return torch.sort(torch.randperm(span, generator=g, device=DEV)[:k]).values


def _batch(case, g):
    """The host tables of an attention call and, on the device, the index tables of its padded form."""
    tq, nug, loc = _ints(case["tq"]), _ints(case["nug"]), _ints(case["loc"])
    B = len(tq)
    span = [10 * k for k in nug]                       # nuggets are chosen out of ten times as many tokens
    pos = [_positions(g, k, s) for k, s in zip(nug, span)]
    loc_pos0 = np.asarray(span, np.int32)              # local tokens follow the compressed context
    if case["inside"]:                                 # queries inside the context: some nuggets, or all, lie ahead of them
        q_pos0 = np.asarray([s * (2 * b + 1) // (2 * B + 2) for b, s in enumerate(span)], np.int32)
    else:                                              # queries are the last local tokens
        q_pos0 = np.asarray([s + n - t for s, n, t in zip(span, loc, tq)], np.int32)
    s = dict(q_off=_offsets(tq), q_pos0=q_pos0, cache_off=_offsets(nug), cache_len=np.asarray(nug, np.int32), loc_off=_offsets(loc),
             loc_len=np.asarray(loc, np.int32), loc_pos0=loc_pos0)
    s["cache_pos"] = torch.cat(pos).to(torch.int32)
    T, L = max(tq), max(k + n for k, n in zip(nug, loc))
    q_row, q_pos = np.zeros((B, T), np.int64), np.full((B, T), -1, np.int64)
    k_row, k_pos = np.zeros((B, L), np.int64), np.full((B, L), 2 ** 31 - 1, np.int64)
    at_q, at_k = np.zeros(int(s["q_off"][-1]), np.int64), np.zeros(sum(nug) + sum(loc), np.int64)
    host = s["cache_pos"].cpu().numpy()
    for b in range(B):
        q_row[b, :tq[b]] = s["q_off"][b] + np.arange(tq[b])
        q_pos[b, :tq[b]] = q_pos0[b] + np.arange(tq[b])
        at_q[s["q_off"][b]:s["q_off"][b + 1]] = b * T + np.arange(tq[b])
        k_row[b, :nug[b]] = s["cache_off"][b] + np.arange(nug[b])
        k_pos[b, :nug[b]] = host[s["cache_off"][b]:s["cache_off"][b + 1]]
        k_row[b, nug[b]:nug[b] + loc[b]] = sum(nug) + s["loc_off"][b] + np.arange(loc[b])
        k_pos[b, nug[b]:nug[b] + loc[b]] = loc_pos0[b] + np.arange(loc[b])
        at_k[s["cache_off"][b]:s["cache_off"][b + 1]] = b * L + np.arange(nug[b])
        at_k[sum(nug) + s["loc_off"][b]:sum(nug) + s["loc_off"][b + 1]] = b * L + nug[b] + np.arange(loc[b])
    for name, v in (("q_row", q_row), ("q_pos", q_pos), ("k_row", k_row), ("k_pos", k_pos), ("at_q", at_q), ("at_k", at_k)):
        s[name] = torch.from_numpy(v).to(DEV)
    return s


def _stored(x):
    """x [rows, H, dh] in the 4-bit format: codes uint8 [rows, H, dh / 2] (feature 2i in the low half of byte i) and one
    int32 word a group (step in the low 16 bits, minimum in the high ones)."""
    c, s, m = _quantise(x)
    c = c.to(torch.uint8)
    codes = c[..., 0::2] | (c[..., 1::2] << 4)
    half = lambda v: v.to(torch.bfloat16).view(torch.int16).to(torch.int32) & 0xffff  # noqa: E731
    return codes, half(s) | (half(m) << 16)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1_000_003 + 17)
    dtype, H, dh = TYPES[case["dtype"]], case["H"], case["dh"]
    s = dict(op=case["op"], dtype=dtype, H=H, dh=dh, scale=dh ** -0.5, lse=bool(case.get("lse")))
    if case["op"] == "gather_q4":
        n, nug, used = _ints(case["n"]), _ints(case["nug"]), _ints(case["used"])
        s.update(seq_off=_offsets(n), nug_off=_offsets(nug), used=np.asarray(used, np.int32),
                 cache_off=_offsets([k + u for k, u in zip(nug, used)]), pos_base=np.asarray([7 * b for b in range(len(n))], np.int32))
        s["K"], s["V"] = _randn(g, (sum(n), H, dh), dtype), _randn(g, (sum(n), H, dh), dtype)
        idx = [_positions(g, k, m) for k, m in zip(nug, n)]
        s["idx"] = torch.cat(idx).to(torch.int32)
        s["src"] = torch.cat([i + int(o) for i, o in zip(idx, s["seq_off"])])
        s["dst"] = torch.cat([torch.arange(k, device=DEV) + int(o) + u for k, o, u in zip(nug, s["cache_off"], used)])
        s["pos"] = torch.cat([i + int(p) for i, p in zip(idx, s["pos_base"])]).to(torch.int32)
        rows = int(s["cache_off"][-1])
        old = [_stored(_randn(g, (rows, H, dh), torch.float32)) for _ in range(2)]
        s["cache_q4"], s["cache_scale"] = torch.stack([old[0][0], old[1][0]], 2), torch.stack([old[0][1], old[1][1]], 2)
        s["cache_pos"] = torch.zeros(rows, dtype=torch.int32, device=DEV)
        return s
    if case["op"] == "expand_q4":
        nug, cap = _ints(case["nug"]), _ints(case["cap"])
        s.update(cache_off=_offsets(cap), cache_len=np.asarray(nug, np.int32))
        rows = int(s["cache_off"][-1])
        both = [_stored(_randn(g, (rows, H, dh), torch.float32)) for _ in range(2)]
        s["cache_q4"], s["cache_scale"] = torch.stack([both[0][0], both[1][0]], 2), torch.stack([both[0][1], both[1][1]], 2)
        s["live"] = torch.cat([torch.arange(k, device=DEV) + int(o) for k, o in zip(nug, s["cache_off"])])
        s["K"], s["V"] = torch.zeros(rows, H, dh, dtype=dtype, device=DEV), torch.zeros(rows, H, dh, dtype=dtype, device=DEV)
        return s
    s.update(_batch(case, g))
    rows, lrows, qrows = int(s["cache_off"][-1]), int(s["loc_off"][-1]), int(s["q_off"][-1])
    s["Q"] = _randn(g, (qrows, H, dh), dtype)
    s["locK"], s["locV"] = _randn(g, (lrows, H, dh), dtype), _randn(g, (lrows, H, dh), dtype)
    K, V = _randn(g, (rows, H, dh), dtype), _randn(g, (rows, H, dh), dtype)
    if case["op"] == "attend_q4":
        k4, v4 = _stored(K.float()), _stored(V.float())
        s["cache_q4"], s["cache_scale"] = torch.stack([k4[0], v4[0]], 2), torch.stack([k4[1], v4[1]], 2)
        return s
    s["cacheK"], s["cacheV"] = K, V
    # a training step has the forward's output and log-sum-exp in hand, and the gradient that arrives from the layer above
    s["O"], s["saved_lse"] = _forward(s, torch.cat([K, s["locK"]]), torch.cat([V, s["locV"]]))
    s["dO"] = _randn(g, (qrows, H, dh), dtype)
    return s


# ---- plain forms ------------------------------------------------------------------------------------------------------
def _bf16_down(x):
    """The largest bf16 numbers that are not above the fp32 numbers x (as fp32)."""
    bits = x.contiguous().view(torch.int32)
    cut = bits & -65536
    return torch.where((cut != bits) & (bits < 0), cut + 65536, cut).view(torch.float32)


def _bf16_step(s, span):
    """The next bf16 number above s wherever 15 s is still below the span (s a bf16 number >= 0, as fp32)."""
    return torch.where(15.0 * s.double() < span, (s.view(torch.int32) + 65536).view(torch.float32), s)


def _quantise(x):
    """Codes (as doubles, x's shape), steps and minima (fp32 holding bf16 numbers) of the 4-bit format."""
    g = x.unflatten(-1, (-1, GROUP))
    m = _bf16_down(g.amin(-1).float())
    span = g.amax(-1).double() - m.double()
    s = _bf16_down((span / 15.0).float())
    s = _bf16_step(_bf16_step(s, span), span)
    c = torch.round((g.double() - m.double()[..., None]) / s.double()[..., None]).clamp(0.0, 15.0)
    return torch.where(s[..., None] > 0, c, torch.zeros_like(c)).flatten(-2), s, m


def _values(codes, scale):
    """fp32 values that codes uint8 [..., dh / 2] and group words int32 [..., dh / 32] stand for."""
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).unflatten(-1, (-1, GROUP)).float()
    step = (scale << 16).view(torch.float32)
    low = (scale & -65536).view(torch.float32)
    return (c * step[..., None] + low[..., None]).flatten(-2)


def _forward(s, K, V):
    """Attention of a padded batch in fp32: O and the log-sum-exp, of the packed query rows."""
    q, k, v = s["Q"][s["q_row"]].float(), K[s["k_row"]].float(), V[s["k_row"]].float()
    see = (s["k_pos"][:, None, :] <= s["q_pos"][:, :, None])[:, None]
    x = torch.einsum("bqhd,bkhd->bhqk", q, k) * s["scale"]
    x = torch.where(see, x, torch.full_like(x, -math.inf))
    top = x.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    lse = (torch.log(total) + top)[..., 0]
    o = torch.einsum("bhqk,bkhd->bqhd", p / torch.where(total > 0, total, torch.ones_like(total)), v)
    return o.flatten(0, 1)[s["at_q"]].to(s["dtype"]), lse.transpose(1, 2).flatten(0, 1)[s["at_q"]].contiguous()


def _backward(s):
    q, o, do = (s[n][s["q_row"]].float() for n in ("Q", "O", "dO"))
    k = torch.cat([s["cacheK"], s["locK"]])[s["k_row"]].float()
    v = torch.cat([s["cacheV"], s["locV"]])[s["k_row"]].float()
    lse = s["saved_lse"][s["q_row"]].transpose(1, 2)[..., None]
    see = (s["k_pos"][:, None, :] <= s["q_pos"][:, :, None])[:, None]
    p = torch.exp(torch.einsum("bqhd,bkhd->bhqk", q, k) * s["scale"] - lse)
    p = torch.where(see, p, torch.zeros_like(p))
    delta = (do * o).sum(-1).transpose(1, 2)[..., None]
    ds = p * (torch.einsum("bqhd,bkhd->bhqk", do, v) - delta)
    dq = torch.einsum("bhqk,bkhd->bqhd", ds, k) * s["scale"]
    dk = torch.einsum("bhqk,bqhd->bkhd", ds, q) * s["scale"]
    dv = torch.einsum("bhqk,bqhd->bkhd", p, do)
    n = s["cacheK"].shape[0]
    dk, dv = (t.flatten(0, 1)[s["at_k"]].to(s["dtype"]) for t in (dk, dv))
    score = ds.sum((1, 2)).flatten()[s["at_k"]][:n]
    return {"dQ": dq.flatten(0, 1)[s["at_q"]].to(s["dtype"]), "dcacheK": dk[:n], "dcacheV": dv[:n], "dlocK": dk[n:], "dlocV": dv[n:],
            "dscore": score}


def _plain(s):
    if s["op"] == "attend_backward":
        return _backward(s)
    if s["op"] == "gather_q4":
        kv = _values(s["cache_q4"], s["cache_scale"])
        for_each = torch.stack([s["K"][s["src"]], s["V"][s["src"]]], 2)
        c, step, low = _quantise(for_each)
        kv[s["dst"]] = (c.unflatten(-1, (-1, GROUP)) * step.double()[..., None] + low.double()[..., None]).flatten(-2).float()
        pos = s["cache_pos"].clone()
        pos[s["dst"]] = s["pos"]
        return {"K": kv[:, :, 0].to(s["dtype"]), "V": kv[:, :, 1].to(s["dtype"]), "cache_pos": pos}
    kv = _values(s["cache_q4"], s["cache_scale"])
    if s["op"] == "expand_q4":
        K, V = s["K"].clone(), s["V"].clone()
        K[s["live"]], V[s["live"]] = kv[s["live"], :, 0].to(s["dtype"]), kv[s["live"], :, 1].to(s["dtype"])
        return {"K": K, "V": V}
    o, lse = _forward(s, torch.cat([kv[:, :, 0], s["locK"].float()]), torch.cat([kv[:, :, 1], s["locV"].float()]))
    return {"O": o, "lse": lse} if s["lse"] else {"O": o}


# ---- the framework's calls --------------------------------------------------------------------------------------------
def _new(s, name, shape, dtype):
    """A buffer that the program keeps from call to call."""
    if name not in s:
        s[name] = torch.empty(shape, dtype=dtype, device=DEV)
    return s[name]


def _called(s):
    from paper_2310_02409_b200 import api
    if not _context:
        _context.append(api.Dodo(0))
    dodo = _context[0]
    H, dh, dtype = s["H"], s["dh"], s["dtype"]
    if s["op"] == "gather_q4":
        used = s["used"].copy()
        dodo.gather_kv_q4(s["K"], s["V"], s["seq_off"], s["idx"], s["nug_off"], s["pos_base"], s["cache_q4"], s["cache_scale"],
                          s["cache_pos"], s["cache_off"], used)
        rows = s["cache_q4"].shape[0]
        K, V = _new(s, "outK", (rows, H, dh), dtype), _new(s, "outV", (rows, H, dh), dtype)
        dodo.expand_kv_q4(s["cache_q4"], s["cache_scale"], s["cache_off"], used, K, V)
        return {"K": K, "V": V, "cache_pos": s["cache_pos"]}
    if s["op"] == "expand_q4":
        dodo.expand_kv_q4(s["cache_q4"], s["cache_scale"], s["cache_off"], s["cache_len"], s["K"], s["V"])
        return {"K": s["K"], "V": s["V"]}
    rows = int(s["cache_off"][-1])
    if s["op"] == "attend_q4":
        ws = _new(s, "workspace", (dodo.attend_q4_workspace_bytes(H, dh, rows),) if "workspace" not in s else None, torch.uint8)
        O = _new(s, "outO", s["Q"].shape, dtype)
        lse = _new(s, "outL", s["Q"].shape[:2], torch.float32) if s["lse"] else None
        dodo.attend_q4(s["Q"], s["q_off"], s["q_pos0"], s["scale"], s["cache_q4"], s["cache_scale"], s["cache_pos"], s["cache_off"],
                       s["cache_len"], s["locK"], s["locV"], s["loc_off"][:-1], s["loc_len"], s["loc_pos0"], O, lse, ws)
        return {"O": O, "lse": lse} if s["lse"] else {"O": O}
    ws = _new(s, "workspace", (dodo.attend_backward_workspace_bytes(s["Q"].shape[0], H, dh, rows),) if "workspace" not in s else None,
              torch.uint8)
    out = {"dQ": _new(s, "dQ", s["Q"].shape, dtype), "dcacheK": _new(s, "dcK", s["cacheK"].shape, dtype),
           "dcacheV": _new(s, "dcV", s["cacheV"].shape, dtype), "dlocK": _new(s, "dlK", s["locK"].shape, dtype),
           "dlocV": _new(s, "dlV", s["locV"].shape, dtype), "dscore": _new(s, "dscore", (rows,), torch.float32)}
    dodo.attend_backward(s["Q"], s["q_off"], s["q_pos0"], s["scale"], s["cacheK"], s["cacheV"], s["cache_pos"], s["cache_off"],
                         s["cache_len"], s["locK"], s["locV"], s["loc_off"][:-1], s["loc_len"], s["loc_pos0"], s["O"], s["saved_lse"],
                         s["dO"], out["dQ"], out["dcacheK"], out["dcacheV"], out["dlocK"], out["dlocV"], out["dscore"], ws)
    return out


def run(state):
    return _called(state) if own else _plain(state)


# ---- what a pass cannot do without ------------------------------------------------------------------------------------
def work(case):
    H, dh, e = case["H"], case["dh"], 2 if case["dtype"] == "bf16" else 4
    row, row4 = H * dh * e, H * (dh // 2 + dh // GROUP * 4)        # one K (or V) row, floating and in 4 bits
    nug = sum(_ints(case["nug"]))
    if case["op"] == "gather_q4":       # rows read, stored in 4 bits, positions; the whole cache read back
        total = nug + sum(_ints(case["used"]))
        return {"bytes": nug * (2 * row + 2 * row4 + 8) + total * (2 * row4 + 2 * row), "flops": 0}
    if case["op"] == "expand_q4":
        return {"bytes": nug * (2 * row4 + 2 * row), "flops": 0}
    tq, loc = _ints(case["tq"]), _ints(case["loc"])
    pairs = 0
    for t, k, n in zip(tq, _ints(case["nug"]), loc):   # visible (query, key) pairs; inside the context about half of the nuggets
        pairs += t * k // 2 if case["inside"] else t * k + t * (n - t) + t * (t + 1) // 2
    if case["op"] == "attend_q4":
        return {"bytes": nug * (2 * row4 + 4) + sum(loc) * 2 * row + sum(tq) * 2 * row, "flops": 4 * pairs * H * dh}
    return {"bytes": (nug + sum(loc)) * 4 * row + nug * 8 + sum(tq) * (4 * row + 4 * H), "flops": 10 * pairs * H * dh}


# ---- the same in 64 bits, sequence by sequence and head by head -------------------------------------------------------
def _codes64(x):
    """Values that the 4-bit format gives to x (any shape, last axis features), from its definition."""
    f = x.double().reshape(-1, GROUP)
    lo, hi = f.min(1).values, f.max(1).values
    m = lo.float().to(torch.bfloat16)
    below = torch.nextafter(m, torch.full_like(m, -math.inf))
    m = torch.where(m.double() > lo, below, m)
    need = hi - m.double()
    s = (need / 15.0).float().to(torch.bfloat16)
    s = torch.where(15.0 * s.double() < need, torch.nextafter(s, torch.full_like(s, math.inf)), s)
    less = torch.nextafter(s, torch.zeros_like(s))
    s = torch.where(15.0 * less.double() >= need, less, s).double()
    m = m.double()
    c = torch.where(s[:, None] > 0, (f - m[:, None]) / s[:, None], torch.zeros_like(f)).round().clamp(0, 15)
    return (m[:, None] + c * s[:, None]).reshape(x.shape)


def _read64(s):
    codes, words = s["cache_q4"].to(torch.int64), s["cache_scale"].to(torch.int64) & 0xffffffff
    c = torch.zeros(codes.shape[:-1] + (2 * codes.shape[-1],), dtype=torch.float64, device=codes.device)
    c[..., 0::2], c[..., 1::2] = (codes % 16).double(), (codes // 16).double()
    to = lambda w: (w << 16).to(torch.int32).view(torch.float32).double().repeat_interleave(GROUP, -1)  # noqa: E731
    kv = to(words >> 16) + c * to(words & 0xffff)
    return kv[:, :, 0], kv[:, :, 1]


def _sequence(s, b):
    a, z = int(s["cache_off"][b]), int(s["cache_off"][b]) + int(s["cache_len"][b])
    l0, l1 = int(s["loc_off"][b]), int(s["loc_off"][b]) + int(s["loc_len"][b])
    q0, q1 = int(s["q_off"][b]), int(s["q_off"][b + 1])
    pos = torch.cat([s["cache_pos"][a:z].long(), int(s["loc_pos0"][b]) + torch.arange(l1 - l0, device=DEV)])
    qpos = int(s["q_pos0"][b]) + torch.arange(q1 - q0, device=DEV)
    return slice(a, z), slice(l0, l1), slice(q0, q1), pos[None, :] <= qpos[:, None]


def exact(case, seed):
    s = prepare(case, seed)
    if s["op"] == "gather_q4":
        K, V = _read64(s)
        K[s["dst"]], V[s["dst"]] = _codes64(s["K"][s["src"]]), _codes64(s["V"][s["src"]])
        return {"K": K, "V": V, "cache_pos": None}
    if s["op"] == "expand_q4":
        K, V = torch.zeros_like(s["K"], dtype=torch.float64), torch.zeros_like(s["V"], dtype=torch.float64)
        k, v = _read64(s)
        K[s["live"]], V[s["live"]] = k[s["live"]], v[s["live"]]
        return {"K": K, "V": V}
    cK, cV = _read64(s) if s["op"] == "attend_q4" else (s["cacheK"].double(), s["cacheV"].double())
    new = lambda t: torch.zeros(t.shape, dtype=torch.float64, device=DEV)  # noqa: E731
    O, lse = new(s["Q"]), torch.full(s["Q"].shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    dQ, dcK, dcV, dlK, dlV = new(s["Q"]), new(cK), new(cV), new(s["locK"]), new(s["locV"])
    dscore = torch.zeros(cK.shape[0], dtype=torch.float64, device=DEV)
    for b in range(len(s["q_off"]) - 1):
        c, l, q, see = _sequence(s, b)
        n = c.stop - c.start
        for h in range(s["H"]):
            Q = s["Q"][q, h].double()
            K, V = torch.cat([cK[c, h], s["locK"][l, h].double()]), torch.cat([cV[c, h], s["locV"][l, h].double()])
            logit = (Q @ K.T * s["scale"]).masked_fill(~see, -math.inf)
            if s["op"] == "attend_q4":
                lse[q, h] = torch.logsumexp(logit, 1) if logit.shape[1] else -math.inf
                P = torch.exp(logit - lse[q, h][:, None]).masked_fill(~see, 0.0)
                O[q, h] = P @ V
                continue
            P = torch.exp(logit - s["saved_lse"][q, h].double()[:, None]).masked_fill(~see, 0.0)
            dO = s["dO"][q, h].double()
            dS = P * (dO @ V.T - (dO * s["O"][q, h].double()).sum(1, keepdim=True))
            dQ[q, h] = dS @ K * s["scale"]
            dK, dV = dS.T @ Q * s["scale"], P.T @ dO
            dcK[c, h], dlK[l, h], dcV[c, h], dlV[l, h] = dK[:n], dK[n:], dV[:n], dV[n:]
            dscore[c] += dS.sum(0)[:n]
    if s["op"] == "attend_q4":
        return {"O": O, "lse": lse} if s["lse"] else {"O": O}
    return {"dQ": dQ, "dcacheK": dcK, "dcacheV": dcV, "dlocK": dlK, "dlocV": dlV, "dscore": dscore}

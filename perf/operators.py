"""Performance cases of the paged 8-bit cache: tables, append, decode, read-back and chunks.

A server that holds its sequences' keys and values in 8 bits keeps them in pages of a common pool, with one scale
per page and kv head.  Four things happen to such a cache, and each kind of case is one of them:
  tables   requests grow: the block table takes pages from the free list, and the slots of the new tokens are mapped
  step     one serving step of a layer: a token per sequence is appended, then attention over the caches
  fill     a prompt is written into the cache and what the cache holds of it is read back in bf16
  chunk    a chunk of new tokens attends to the cache and to itself
The layers are the library's own: sink + window rings (128 + 4096 tokens, 64 / 8 heads), full layers up to 131072
tokens, and a small 64-wide model.  Where `own` is false the operators are computed in plain torch.
"""
from __future__ import annotations

import math

import torch

own = False

MAX_CODE = 448.0             # largest e4m3 value
MIN_EXP = -120               # smallest exponent of a scale
F8 = torch.float8_e4m3fn


def _case(kind, B, Hq, Hkv, D, sink, window, page, n_min, n_max, T=1, block_tokens=0, layout="bhtd"):
    return {"kind": kind, "B": B, "Hq": Hq, "Hkv": Hkv, "D": D, "sink": sink, "window": window, "page": page,
            "n_min": n_min, "n_max": n_max, "T": T, "block_tokens": block_tokens, "layout": layout}


def listed():
    cases = [
        # a decoding batch between two steps: some requests cross into a new page
        ("tables_step_b64", _case("tables", 64, 64, 8, 128, 128, 4096, 64, 100, 5000)),
        # a wave of ragged prompts enters a full layer's cache: whole rows of the table, a slot for every token
        ("tables_prompts_b16", _case("tables", 16, 64, 8, 128, 0, 131072, 64, 0, 0, T=131072)),
        # a single user's step over a ring: latency
        ("step_ring_b1", _case("step", 1, 64, 8, 128, 128, 4096, 64, 131071, 131071)),
        # the library's headline serving batch, its rings in 8 bits
        ("step_ring_b16", _case("step", 16, 64, 8, 128, 128, 4096, 64, 131071, 131071)),
        # a full-attention layer at long context, every sequence at its own length: the most bytes
        ("step_full_b16", _case("step", 16, 64, 8, 128, 0, 131072, 64, 60001, 131071)),
        # a small model: short pages, an odd sink and window, sequences from a few tokens to many laps
        ("step_small_d64", _case("step", 48, 16, 4, 64, 4, 1003, 16, 5, 9000)),
        # layers without grouped queries, block-aligned window, pages of 32
        ("step_mha_b4", _case("step", 4, 32, 32, 128, 64, 2048, 32, 700, 32768, block_tokens=64)),
        # a few tokens a sequence into partly filled pages, activations as projections leave them ([B, T, H, D])
        ("fill_short_b8", _case("fill", 8, 16, 4, 64, 64, 1024, 16, 33, 2500, T=37, layout="bthd")),
        # a prompt longer than the ring: most of it is dropped, the ring is whole afterwards
        ("fill_ring_b4", _case("fill", 4, 64, 8, 128, 128, 4096, 64, 0, 0, T=6001)),
        # a prompt into a full layer without grouped queries
        ("fill_prompt_32k", _case("fill", 1, 32, 32, 128, 0, 32768, 128, 0, 0, T=32768, layout="bthd")),
        # a chunk of a long prompt against full rings
        ("chunk_1500", _case("chunk", 2, 64, 8, 128, 128, 4096, 64, 20000, 20000, T=1500)),
        # a short chunk of a small model's sequences, each at its own position
        ("chunk_ragged_d64", _case("chunk", 3, 16, 4, 64, 64, 1024, 16, 150, 4000, T=203)),
    ]
    return [dict(c, name=n) for n, c in cases]


# ------------------------------------------------------------------------------- drawn cases

_MAX_BYTES, _MAX_FLOPS = 3.2e9, 3.0e11      # of the largest listed cases


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("tables", "step", "step", "step", "fill", "fill", "chunk"))
    Hkv = rng.choice((1, 2, 4, 8, 16, 32))
    Hq = min(64, Hkv * rng.choice((1, 2, 3, 4, 8, 16)) if kind != "chunk" else Hkv * rng.choice((1, 2, 4, 8)))
    Hq -= Hq % Hkv
    D, page = rng.choice((128, 128, 64)), rng.choice((16, 32, 64, 64, 128))
    block = 0
    if kind == "chunk" or rng.random() < 0.5:
        sink, window = 64 * rng.choice((0, 1, 2)), 64 * max(1, _log_int(rng, 128, 4096) // 64)
        block = rng.choice((0, 0, 64))
    else:
        sink, window = rng.choice((0, 0, 4, 100)), _log_int(rng, 300, 131072)
    n_max = _log_int(rng, 1, 131071)
    n_min = rng.choice((n_max, 1 + n_max // 4, n_max // 50))
    if kind == "step":
        T, B = 1, _log_int(rng, 1, 64)
    elif kind == "tables":
        T, B = rng.choice((1, _log_int(rng, 2, 131072))), _log_int(rng, 1, 512)
    elif kind == "fill":
        T, B = _log_int(rng, 2, 32768), _log_int(rng, 1, 8)
    else:
        T, B = _log_int(rng, 2, 3000), rng.choice((1, 1, 2, 4))
    c = _case(kind, B, Hq, Hkv, D, sink, window, page, n_min, n_max, T, block, rng.choice(("bhtd", "bthd")))
    if kind == "chunk":
        c["layout"] = "bhtd"
    while _too_big(c):
        if c["B"] > 1:
            c["B"] //= 2
        elif c["Hkv"] > 1:
            c["Hq"], c["Hkv"] = c["Hq"] // c["Hkv"], 1
        elif c["T"] > 1:
            c["T"] //= 2
        else:
            c["window"] //= 2
            c["block_tokens"] = 0
    return c


def _too_big(c):
    w, cap = work(c), c["sink"] + c["window"]
    pool = 0 if c["kind"] == "tables" else c["B"] * cap * c["Hkv"] * c["D"] * 2.0
    scores = c["B"] * c["Hq"] * c["T"] * 4.0 * (cap + c["T"]) if c["kind"] == "chunk" else 0
    mapped = c["B"] * c["T"] * 8.0 + c["B"] * cap / c["page"] * 4.0
    return w["bytes"] > _MAX_BYTES or w["flops"] > _MAX_FLOPS or pool > 4.5e9 or scores > 9e9 or mapped > 18e6


# ----------------------------------------------------------------------------------- the work

def _before(c):
    """Tokens in each sequence's cache before the call: spread evenly over the case's range."""
    B, lo, hi = c["B"], c["n_min"], c["n_max"]
    return [hi - (hi - lo) * b // max(1, B - 1) for b in range(B)]


def _new(c):
    """New tokens of each sequence.  Steps and chunks: the same for all; prompts and tables: ragged from the second on."""
    T, B = c["T"], c["B"]
    ragged = c["kind"] in ("tables", "fill") and T > 1
    return [T - (T * 3 * b // (4 * B) if ragged else 0) for b in range(B)]


def _pages(c, n):
    return -(-min(n, c["sink"] + c["window"]) // c["page"])


def _read_back(c):
    """Positions that a fill reads back: the newest ones of each sequence, at most a window of them."""
    return min(c["window"], max(n + t for n, t in zip(_before(c), _new(c))))


def _chunk_pairs(c):
    total = 0
    for n in _before(c):
        for i in range(n, n + c["T"]):
            bs = c["block_tokens"]
            w0 = max(0, (i // bs - c["window"] // bs + 1) * bs if bs else i - c["window"] + 1)
            total += i - w0 + 1 + min(w0, c["sink"])
    return total


def work(case):
    c = case
    B, Hq, Hkv, D, T, cap = c["B"], c["Hq"], c["Hkv"], c["D"], c["T"], c["sink"] + c["window"]
    pairs = list(zip(_before(c), _new(c)))
    fresh = sum(min(t, cap) for _, t in pairs)
    if c["kind"] == "tables":
        taken = sum(_pages(c, n + t) - _pages(c, n) for n, t in pairs)
        looked = sum(_pages(c, n + t) - n % cap // c["page"] if n + t <= cap else min(_pages(c, cap), t // c["page"] + 1)
                     for n, t in pairs)
        return {"bytes": 12.0 * B + 8.0 * taken + 4.0 * looked + 8.0 * B * T, "flops": 0.0}
    if c["kind"] == "step":
        held = sum(min(n + 1, cap) for n, _ in pairs)
        pages = sum(_pages(c, n + 1) for n, _ in pairs)
        return {"bytes": held * Hkv * D * 2.0 + pages * (8.0 * Hkv + 4) + B * Hkv * D * 6.0 + B * Hq * (4.0 * D + 4) + 16.0 * B,
                "flops": 4.0 * held * Hq * D}
    if c["kind"] == "fill":
        back, read = _read_back(c), 0
        for n, t in pairs:
            read += min(back, n + t, cap)
        # new rows in, codes out; then codes in, rows out, for K and V
        return {"bytes": fresh * Hkv * D * 6.0 + read * Hkv * D * 2.0 + B * back * (Hkv * D * 4.0 + 8.0), "flops": 0.0}
    kept = sum(min(n, cap) for n, _ in pairs)
    return {"bytes": B * Hq * T * (4.0 * D + 4) + B * Hkv * T * D * 4.0 + kept * Hkv * D * 2.0,
            "flops": 4.0 * D * Hq * _chunk_pairs(c)}


# ------------------------------------------------------------------------------------ the inputs

def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)


def _pool(gen, c, num_pages, wide):
    """Pages of quantised rows: channels of unequal size, a few tokens far above the rest (K), each page with its scale."""
    Hkv, P, D = c["Hkv"], c["page"], c["D"]
    codes = torch.empty(num_pages, Hkv, P, D, dtype=F8, device="cuda")
    scale = torch.empty(num_pages, Hkv, device="cuda")
    channel = torch.exp(0.4 * _randn(gen, 1, Hkv, 1, D)) if wide else torch.ones(1, Hkv, 1, D, device="cuda")
    chunk = max(1, (1 << 27) // (Hkv * P * D))
    for a in range(0, num_pages, chunk):
        b = min(num_pages, a + chunk)
        x = _randn(gen, b - a, Hkv, P, D) * channel
        x *= 1 + 5 * (torch.rand(b - a, 1, P, 1, generator=gen, device="cuda") < 0.01)
        top = x.abs().amax((2, 3))
        e = torch.ceil(torch.log2(top / 440))
        codes[a:b] = (x * torch.exp2(-e)[..., None, None]).to(F8)
        scale[a:b] = torch.exp2(e)
    return codes, scale


def _inputs(c, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    B, Hq, Hkv, D, T, P = c["B"], c["Hq"], c["Hkv"], c["D"], c["T"], c["page"]
    before, new = _before(c), _new(c)
    after = [n + t for n, t in zip(before, new)]
    width = _pages(c, c["sink"] + c["window"])
    held = [_pages(c, n if c["kind"] in ("tables", "chunk") else n + t) for n, t in zip(before, new)]
    wanted = sum(_pages(c, n + t) for n, t in zip(before, new))
    num_pages = max(1, wanted) + max(4, wanted // 20)
    pages = torch.randperm(num_pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b in range(B):
        table[b, :held[b]] = pages[at:at + held[b]]
        at += held[b]
    s = {"table": table, "n_before": torch.tensor(before, dtype=torch.int64, device="cuda"),
         "n_after": torch.tensor(after, dtype=torch.int64, device="cuda"),
         "n_new": torch.tensor(new, dtype=torch.int32, device="cuda"), "num_pages": num_pages}
    if c["kind"] == "tables":
        s.update(free=pages, free_start=torch.tensor([at], dtype=torch.int32, device="cuda"))
        return s
    s["k_pool"], s["k_scale"] = _pool(gen, c, num_pages, True)
    s["v_pool"], s["v_scale"] = _pool(gen, c, num_pages, False)
    shape = (B, Hkv, T, D) if c["layout"] == "bhtd" else (B, T, Hkv, D)
    for x in ("k", "v"):
        s[x] = _randn(gen, *shape).to(torch.bfloat16)
        if c["layout"] != "bhtd":
            s[x] = s[x].transpose(1, 2)
    if c["kind"] == "step":
        s["q"] = (1.5 * _randn(gen, B, Hq, D)).to(torch.bfloat16)
    elif c["kind"] == "chunk":
        s["q"] = (1.5 * _randn(gen, B, Hq, T, D)).to(torch.bfloat16)
    else:
        back = _read_back(c)
        first = [max(0, a - back) for a in after]
        s["first"] = torch.tensor(first, dtype=torch.int64, device="cuda")
        s["count"] = torch.tensor([a - f for a, f in zip(after, first)], dtype=torch.int32, device="cuda")
    return s


def prepare(case, seed):
    c = case
    s = dict(_inputs(c, seed), case=c)
    B, Hq, Hkv, D, T = c["B"], c["Hq"], c["Hkv"], c["D"], c["T"]
    s["host_before"], s["back"] = _before(c), _read_back(c)
    # what a server holds anyway: where results go
    if c["kind"] == "tables":
        s["slot_map"] = torch.empty(B, T, dtype=torch.int64, device="cuda")
        s["free_next"] = torch.empty(1, dtype=torch.int32, device="cuda")
    elif c["kind"] == "fill":
        s["slot_map"] = torch.empty(B, s["back"], dtype=torch.int64, device="cuda")
        s["k_out"], s["v_out"] = (torch.empty(B, Hkv, s["back"], D, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    else:
        s["o"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(s["q"].shape[:-1], device="cuda")
    if own:
        from paper_2410_01485_b200 import binding as lg
        p = lg.paged_params(B, Hq, Hkv, D, c["sink"], c["window"], page_tokens=c["page"], num_pages=s["num_pages"],
                            block_tokens=c["block_tokens"])
        s["lg"], s["p"] = lg, p
        if c["kind"] == "step":      # a serving loop's calls: fixed buffers, arguments marshalled once
            cache = (s["k_pool"], s["v_pool"], s["k_scale"], s["v_scale"], s["table"])
            s["append"] = lg.paged_append_call(p, *cache, s["k"], s["v"], s["n_before"])
            s["decode"] = lg.paged_decode_call(p, s["q"], *cache, s["n_after"], s["o"], s["lse"], lg.paged_decode_workspace(p))
        elif c["kind"] == "chunk":
            s["ws"] = lg.paged_chunk_prefill_workspace(p, T, s["host_before"])
    return s


# ------------------------------------------------------------------------------ one pass: the library

def _run_own(s):
    lg, p, c = s["lg"], s["p"], s["case"]
    if c["kind"] == "tables":
        lg.lg_paged_table_extend(p, s["n_before"], s["n_new"], s["free"], s["free_start"], s["table"], s["free_next"])
        lg.lg_paged_slot_map(p, s["n_after"], s["n_before"], s["n_new"], s["table"], s["slot_map"])
        return s["table"], s["free_next"], s["slot_map"]
    cache = (s["k_pool"], s["v_pool"], s["k_scale"], s["v_scale"])
    if c["kind"] == "step":
        s["append"]()
        s["decode"]()
        return (s["o"], s["lse"], *cache)
    if c["kind"] == "fill":
        lg.lg_paged_append(p, *cache, s["table"], s["k"], s["v"], s["n_before"], s["n_new"])
        lg.lg_paged_slot_map(p, s["n_after"], s["first"], s["count"], s["table"], s["slot_map"])
        lg.lg_paged_gather(p, *cache, s["slot_map"], s["k_out"], s["v_out"])
        return s["k_out"], s["v_out"], s["slot_map"], s["k_scale"], s["v_scale"]
    return lg.lg_paged_chunk_prefill(p, s["q"], s["k"], s["v"], *cache, s["table"], s["host_before"], o=s["o"], lse=s["lse"],
                                     workspace=s["ws"])


# ------------------------------------------------------------------------- one pass: plain torch

def _held(c, slot, n):
    """Position of the token that a slot holds after n tokens; -1 where it holds none."""
    sink, W = c["sink"], c["window"]
    lap = torch.where(slot < sink, 0, torch.div(n - 1 - slot, W, rounding_mode="floor") * W)
    return torch.where((slot < n) & (slot < sink + W), slot + lap, -1)


def _slot_of(c, pos):
    return torch.where(pos < c["sink"], pos, c["sink"] + (pos - c["sink"]) % c["window"])


def _plain_tables(s):
    c = s["case"]
    P, cap = c["page"], c["sink"] + c["window"]
    have = (s["n_before"].clamp(max=cap) + P - 1) // P
    need = ((s["n_before"] + s["n_new"]).clamp(max=cap) + P - 1) // P
    take = need - have
    ends = torch.cumsum(take, 0) + s["free_start"]
    col = torch.arange(s["table"].shape[1], device="cuda")[None]
    at = (ends - need)[:, None] + col
    entry = torch.where(at < len(s["free"]), s["free"][at.clamp(0, len(s["free"]) - 1)], -1)
    s["table"].copy_(torch.where((col >= have[:, None]) & (col < need[:, None]), entry, s["table"]))
    s["free_next"].copy_(ends[-1:])
    _plain_slot_map(s, s["n_after"], s["n_before"], s["n_new"])
    return s["table"], s["free_next"], s["slot_map"]


def _plain_slot_map(s, n, first, count):
    c = s["case"]
    t = torch.arange(s["slot_map"].shape[1], device="cuda")[None]
    pos = first[:, None] + t
    slot = _slot_of(c, pos)
    page = torch.gather(s["table"].long(), 1, (slot // c["page"]).clamp(0, s["table"].shape[1] - 1))
    ok = (t < count[:, None]) & (_held(c, slot, n[:, None]) == pos) & (page >= 0)
    s["slot_map"].copy_(torch.where(ok, page * c["page"] + slot % c["page"], -1))


def _plain_append_one(s, x, pages, phys):
    c = s["case"]
    pool, scales = s[x + "_pool"], s[x + "_scale"]
    slot = pages[..., None] * c["page"] + torch.arange(c["page"], device="cuda")        # [B, Np, P]
    n0, n1 = s["n_before"][:, None, None], s["n_after"][:, None, None]
    pos = _held(c, slot, n1)
    fresh, live = pos >= n0, pos >= 0
    bytes_now = pool.view(torch.uint8)[phys]                                              # [B, Np, Hkv, P, D]
    old = bytes_now.view(F8).float() * scales[phys][..., None, None]
    b = torch.arange(c["B"], device="cuda")[:, None, None]
    new = s[x].transpose(1, 2)[b, (pos - n0).clamp(0, c["T"] - 1)].float().transpose(2, 3)   # [B, Np, Hkv, P, D]
    value = torch.where(fresh[:, :, None, :, None], new, old)
    value = torch.where(live[:, :, None, :, None], value, 0.0)
    mant, exp = torch.frexp(value.abs().amax((3, 4)))
    e = torch.where(mant == 0, 0, exp - 9 + (mant > 0.875)).clamp(min=MIN_EXP).float()
    coded = (value * torch.exp2(-e)[..., None, None]).to(F8).view(torch.uint8)
    coded = torch.where(live[:, :, None, :, None], coded, bytes_now)
    touched = fresh.any(2)
    pool.view(torch.uint8)[phys[touched]] = coded[touched]
    scales[phys[touched]] = torch.exp2(e)[touched]


def _plain_append(s):
    c = s["case"]
    if c["T"] == 1:
        pages = _slot_of(c, s["n_before"])[:, None] // c["page"]
    else:
        pages = torch.arange(s["table"].shape[1], device="cuda")[None].expand(c["B"], -1)
    phys = torch.gather(s["table"].long(), 1, pages).clamp(min=0)
    _plain_append_one(s, "k", pages, phys)
    _plain_append_one(s, "v", pages, phys)


def _plain_rows(s, x, phys):
    """Rows of the pages as fp32 [B, Hkv, pages * P, D]."""
    c = s["case"]
    rows = s[x + "_pool"].view(torch.uint8)[phys].view(F8).float()
    rows *= s[x + "_scale"][phys][..., None, None]
    return rows.transpose(1, 2).reshape(c["B"], c["Hkv"], -1, c["D"])


def _plain_attend(c, q, k, v, see):
    """q [B, Hkv, rows, D], k, v [B, Hkv, keys, D], see [B, rows, keys] or [B, 1, keys] -> o, lse."""
    x = (q @ k.transpose(2, 3)) * c["D"] ** -0.5
    x.masked_fill_(~see[:, None], -math.inf)
    top = x.amax(3, keepdim=True)
    x.sub_(top).exp_()
    total = x.sum(3, keepdim=True)
    return (x @ v) / total, (top + torch.log(total))[..., 0]


def _near(c, i, pos):
    bs = c["block_tokens"]
    recent = i // bs - pos // bs < c["window"] // bs if bs else i - pos < c["window"]
    return (pos >= 0) & (pos <= i) & (recent | (pos < c["sink"]))


def _plain_step(s):
    c = s["case"]
    _plain_append(s)
    slot = torch.arange(s["table"].shape[1] * c["page"], device="cuda")[None]
    n = s["n_after"][:, None]
    see = _near(c, n - 1, _held(c, slot, n))[:, None]
    phys = s["table"].long().clamp(min=0)
    k, v = _plain_rows(s, "k", phys), _plain_rows(s, "v", phys).masked_fill_(~see[..., None], 0.0)
    o, lse = _plain_attend(c, s["q"].float().view(c["B"], c["Hkv"], -1, c["D"]), k, v, see)
    s["o"].copy_(o.view_as(s["o"]))
    s["lse"].copy_(lse.view_as(s["lse"]))
    return s["o"], s["lse"], s["k_pool"], s["v_pool"], s["k_scale"], s["v_scale"]


def _plain_gather(s, x):
    c, slot = s["case"], s["slot_map"]
    page, at = slot.clamp(min=0) // c["page"], slot.clamp(min=0) % c["page"]
    rows = s[x + "_pool"].view(torch.uint8)[page, :, at].view(F8).float() * s[x + "_scale"][page][..., None]
    s[x + "_out"].copy_(torch.where(slot[..., None, None] >= 0, rows, 0.0).transpose(1, 2))


def _plain_fill(s):
    _plain_append(s)
    _plain_slot_map(s, s["n_after"], s["first"], s["count"])
    _plain_gather(s, "k")
    _plain_gather(s, "v")
    return s["k_out"], s["v_out"], s["slot_map"], s["k_scale"], s["v_scale"]


def _plain_chunk(s):
    c = s["case"]
    B, Hkv, T = c["B"], c["Hkv"], c["T"]
    slot = torch.arange(s["table"].shape[1] * c["page"], device="cuda")[None]
    n = s["n_before"][:, None]
    i = n + torch.arange(T, device="cuda")
    pos = torch.cat([_held(c, slot, n), i], 1)
    see = _near(c, i[:, :, None], pos[:, None])
    phys = s["table"].long().clamp(min=0)
    k, v = (torch.cat([_plain_rows(s, x, phys), s[x].float()], 2).masked_fill_((pos < 0)[:, None, :, None], 0.0) for x in "kv")
    G = c["Hq"] // Hkv
    q = s["q"].float().view(B, Hkv, G * T, c["D"])
    o, lse = _plain_attend(c, q, k, v, see.repeat(1, G, 1))
    s["o"].copy_(o.view_as(s["o"]))
    s["lse"].copy_(lse.view_as(s["lse"]))
    return s["o"], s["lse"]


def run(s):
    if own:
        return _run_own(s)
    return {"tables": _plain_tables, "step": _plain_step, "fill": _plain_fill, "chunk": _plain_chunk}[s["case"]["kind"]](s)


# ------------------------------------------------------- the same outputs in 64 bits

def _ring(c, n):
    """(slot, position) of what a cache holds after n tokens, in time order."""
    sink, W = c["sink"], c["window"]
    pos = torch.cat([torch.arange(min(n, sink)), torch.arange(max(sink, n - W), max(n, sink))]).cuda()
    return torch.where(pos < sink, pos, sink + (pos - sink) % W), pos


def _to_e4m3(x):
    """Nearest e4m3 value (ties to even), by its definition: 3 bits behind the leading one, none below 2^-9."""
    ulp = torch.exp2(torch.clamp(torch.frexp(x.abs())[1] - 1, min=-6).double() - 3)
    return torch.clamp(torch.round(x / ulp) * ulp, -MAX_CODE, MAX_CODE)


def _exact_append(c, s, before, new):
    for b, (n, t) in enumerate(zip(before, new)):
        slot, pos = _ring(c, n + t)
        fresh = pos >= n
        for page in torch.unique(slot[fresh] // c["page"]).tolist():
            mine = slot // c["page"] == page
            at, p, is_new = slot[mine] % c["page"], pos[mine], fresh[mine]
            phys = int(s["table"][b, page])
            for x in ("k", "v"):
                codes, scale = s[x + "_pool"][phys], s[x + "_scale"][phys]
                value = codes.double()[:, at] * scale.double()[:, None, None]
                value[:, is_new] = s[x][b, :, p[is_new] - n].double()
                top = value.abs().amax((1, 2))
                e = torch.ceil(torch.log2(top / MAX_CODE))
                e += (top > MAX_CODE * torch.exp2(e)).double() - (top <= MAX_CODE * torch.exp2(e - 1)).double()
                e = torch.where(top == 0, 0.0, e.clamp(min=MIN_EXP))
                whole = codes.double()
                whole[:, at] = _to_e4m3(value * torch.exp2(-e)[:, None, None])
                s[x + "_pool"][phys] = whole.to(F8)                  # (the values are e4m3 numbers already)
                s[x + "_scale"][phys] = torch.exp2(e).float()


def _exact_rows(c, s, b, h, slot):
    page = s["table"][b].long()[slot // c["page"]]
    at = slot % c["page"]
    return [s[x + "_pool"].view(torch.uint8)[page, h, at].view(F8).double() * s[x + "_scale"][page, h].double()[:, None]
            for x in ("k", "v")]


def exact(case, seed):
    c = case
    B, Hq, Hkv, D, T, G = c["B"], c["Hq"], c["Hkv"], c["D"], c["T"], c["Hq"] // c["Hkv"]
    if c["kind"] == "tables":
        return None                  # whole numbers
    if c["kind"] == "fill" and B * T / c["page"] > 1e4:
        return None
    s, before, new = _inputs(c, seed), _before(c), _new(c)
    if c["kind"] != "chunk":
        _exact_append(c, s, before, new)
    if c["kind"] == "fill":
        back = _read_back(c)
        out = [torch.zeros(B, Hkv, back, D, dtype=torch.float64, device="cuda") for _ in "kv"]
        for b, (n, t) in enumerate(zip(before, new)):
            slot, pos = _ring(c, n + t)
            first = max(0, n + t - back)
            there = pos >= first
            for h in range(Hkv):
                for x, rows in zip(out, _exact_rows(c, s, b, h, slot[there])):
                    x[b, h, pos[there] - first] = rows
        return out[0], out[1], None, s["k_scale"].double(), s["v_scale"].double()
    o = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(s["q"].shape[:-1], dtype=torch.float64, device="cuda")
    for b, n in enumerate(before):
        slot, pos = _ring(c, n if c["kind"] == "chunk" else n + 1)
        i = torch.arange(n, n + T, device="cuda")
        every = torch.cat([pos, i]) if c["kind"] == "chunk" else pos
        bs = c["block_tokens"]
        far = (i[:, None] // bs - every // bs >= c["window"] // bs) if bs else (i[:, None] - every >= c["window"])
        hidden = (every > i[:, None]) | (far & (every >= c["sink"]))
        for h in range(Hkv):
            k, v = _exact_rows(c, s, b, h, slot)
            if c["kind"] == "chunk":
                k, v = torch.cat([k, s["k"][b, h].double()]), torch.cat([v, s["v"][b, h].double()])
            for g in range(h * G, h * G + G):
                x = (s["q"][b, g].double().view(T, D) @ k.T / math.sqrt(D)).masked_fill(hidden, -math.inf)
                l = torch.logsumexp(x, 1)
                o[b, g] = (torch.exp(x - l[:, None]) @ v).view(o[b, g].shape)
                lse[b, g] = l.view(lse[b, g].shape)
    if c["kind"] == "chunk":
        return o, lse
    return o, lse, s["k_pool"], s["v_pool"], s["k_scale"].double(), s["v_scale"].double()

"""Cases of the paged cache's operators: what a serving program asks of them, through the public binding.

  rotate   ``qk_norm_rotate``: norms of queries and keys per head and the position rotation, dense rows in and out
  append   ``PagedCache.append``: the same pass, keys and values written into the pages of a paged cache; where the
           pages hold 8 bits, the rows just written are read back (``PagedCache.read``), so that values are returned
  read     ``PagedCache.read``: pages back into dense rows
  decode   ``PagedCache.decode``: attention of one new token per sequence over its pages

Pages as the cache documents them: keys [page][kv head][row][dim], values [page][kv head][row / g][dim][g] with g the
elements of 16 bytes, and for 8-bit pages one exponent byte per row (value = e4m3 code * 2^(exponent - 127)).
"""
from __future__ import annotations

import math

import torch

own = False

_DTYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
_EPS = 1e-6
_BASE = 500000.0
_HEAD = {"norm": True, "rotary": 1.0, "interleaved": False}      # rotary: share of the head that is rotated
_POOL = {"page_rows": 64, "page_dtype": ""}                      # page_dtype "": the rows' own type


def listed():
    return [
        # One decode step of a 7B-sized layer (32 heads of 128), batch 8 at 4096 tokens: latency alone.
        dict(_HEAD, name="rotate_step_7b_fp16", kind="rotate", batch=8, kv_heads=32, group=1, head_dim=128, dtype="fp16",
             length=1, ragged=False, start=4096),
        # A 32k-token prompt of a grouped-query layer (32 query heads on 8 kv heads).
        dict(_HEAD, name="rotate_prompt_gqa_bf16", kind="rotate", batch=1, kv_heads=8, group=4, head_dim=128, dtype="bf16",
             length=32768, ragged=False, start=0),
        # The small model of a reference run in full precision: a 512-token prompt, interleaved pairs, no norm.
        dict(_HEAD, **_POOL, name="append_tiny_fp32", kind="append", batch=1, kv_heads=8, group=1, head_dim=64, dtype="fp32",
             length=512, ragged=False, start=0) | {"norm": False, "interleaved": True, "page_rows": 16},
        # One decode step of 16 grouped-query sequences far into their contexts, 8-bit pages.
        dict(_HEAD, **_POOL, name="append_step_gqa_e4m3", kind="append", batch=16, kv_heads=8, group=4, head_dim=128,
             dtype="bf16", length=1, ragged=False, start=32701) | {"page_dtype": "e4m3"},
        # Prompts of four requests of unequal length written as 8 bits.
        dict(_HEAD, **_POOL, name="append_prompt_gqa_e4m3", kind="append", batch=4, kv_heads=8, group=4, head_dim=128,
             dtype="bf16", length=8192, ragged=True, start=0) | {"page_dtype": "e4m3"},
        # A few short sequences of the 7B layer back into rows, as a prompt that moves into another cache.
        dict(_POOL, name="read_short_7b_fp16", kind="read", batch=8, kv_heads=32, group=1, head_dim=128, dtype="fp16",
             length=300, ragged=True, start=0),
        # A whole 131k-token context of 8 kv heads out of 8-bit pages.
        dict(_POOL, name="read_long_e4m3", kind="read", batch=1, kv_heads=8, group=4, head_dim=128, dtype="bf16",
             length=131072, ragged=False, start=0) | {"page_dtype": "e4m3"},
        # The smallest: one sequence of the small fp32 model, 8 heads of 64.
        dict(_POOL, name="decode_tiny_fp32", kind="decode", batch=1, kv_heads=8, group=1, head_dim=64, dtype="fp32",
             length=513, ragged=False, sink=0, window=0) | {"page_rows": 16},
        # One user's chat on grouped-query heads.
        dict(_POOL, name="decode_chat_gqa_bf16", kind="decode", batch=1, kv_heads=8, group=4, head_dim=128, dtype="bf16",
             length=1517, ragged=False, sink=0, window=0),
        # The ordinary batch of the 7B layer, unequal lengths up to 4096.
        dict(_POOL, name="decode_7b_fp16", kind="decode", batch=8, kv_heads=32, group=1, head_dim=128, dtype="fp16",
             length=4096, ragged=True, sink=0, window=0),
        # Four 32k-token contexts on grouped-query heads in 8-bit pages.
        dict(_POOL, name="decode_gqa_e4m3", kind="decode", batch=4, kv_heads=8, group=4, head_dim=128, dtype="bf16",
             length=32768, ragged=False, sink=0, window=0) | {"page_dtype": "e4m3"},
        # The largest: batch 16 of the 7B layer, unequal lengths up to 16384.
        dict(_POOL, name="decode_wide_bf16", kind="decode", batch=16, kv_heads=32, group=1, head_dim=128, dtype="bf16",
             length=16384, ragged=True, sink=0, window=0),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        c = _draw_once(rng)
        w = work(c)
        if w["bytes"] <= 8.0e8 * (3.0 if c["kind"] == "decode" else 1.0) and w["flops"] <= 2.0e9 * (2.0 if c["kind"] == "decode" else 1.0):
            return c


def _draw_once(rng):
    kind = rng.choice(["rotate", "append", "append", "read", "decode", "decode", "decode", "decode"])
    c = {"kind": kind, "batch": rng.choice([1, 1, 2, 3, 5, 8, 16, 33, 64]), "kv_heads": rng.choice([1, 2, 4, 5, 8, 8, 16, 32]),
         "group": rng.choice([1, 1, 2, 3, 4, 4, 5, 6, 7, 8]), "head_dim": rng.choice([64, 128, 128, 128, 256]),
         "dtype": rng.choice(["bf16", "bf16", "fp16", "fp32"]), "ragged": rng.random() < 0.5}
    if kind != "rotate":
        c["page_rows"] = rng.choice([16, 32, 64, 128, 256])
        c["page_dtype"] = "e4m3" if c["dtype"] != "fp32" and rng.random() < 0.5 else ""
    if kind in ("rotate", "append"):
        c["norm"] = rng.random() < 0.6
        c["rotary"] = rng.choice([1.0, 1.0, 0.5, 0.25])
        c["interleaved"] = rng.random() < 0.3
    if kind == "decode":
        c["length"] = _log_uniform(rng, 1, 131072)
        c["sink"], c["window"] = (rng.choice([0, 1, 4, 67]), _log_uniform(rng, 1, 8192)) if rng.random() < 0.25 else (0, 0)
    else:
        c["length"] = 1 if rng.random() < 0.3 else _log_uniform(rng, 1, 32768)
        c["start"] = 0 if rng.random() < 0.4 else _log_uniform(rng, 1, 131072)
    return c


# ------------------------------------------------------------------------------------------------ sizes and work
def _counts(c):
    """Rows of every sequence: the case's length, or spread over a tenth of it and the whole."""
    n, B = c["length"], c["batch"]
    if not c["ragged"]:
        return [n] * B
    return [n] + [max(1, int(n * (0.1 + 0.9 * ((b * 0.6180339887) % 1.0)))) for b in range(1, B)]


def _starts(c):
    """Position of every sequence's first row."""
    s, B = c.get("start", 0), c["batch"]
    return [max(0, s - 37 * b) if c["ragged"] else s for b in range(B)]


def _seen(c, length):
    """Rows that a new token at the end of `length` rows attends to."""
    return length if not c["window"] else min(length, min(c["sink"], max(0, length - c["window"])) + c["window"])


def work(case):
    c = case
    e = 4.0 if c["dtype"] == "fp32" else 2.0
    D, H, Hq = c["head_dim"], c["kv_heads"], c["kv_heads"] * c["group"]
    tokens = float(sum(_counts(c)))
    row = (D + 1.0) if c.get("page_dtype") else D * e            # bytes of a row in a page
    if c["kind"] == "rotate":
        return {"bytes": tokens * 2.0 * (Hq + H) * D * e, "flops": tokens * (Hq + H) * D * 8.0}
    if c["kind"] == "append":
        back = 2.0 * H * (row + D * e) if c["page_dtype"] else 0.0
        return {"bytes": tokens * ((2.0 * Hq + 2.0 * H) * D * e + 2.0 * H * row + back), "flops": tokens * (Hq + H) * D * 8.0}
    if c["kind"] == "read":
        return {"bytes": tokens * 2.0 * H * (row + D * e), "flops": tokens * 2.0 * H * D}
    rows = float(sum(_seen(c, n) for n in _counts(c)))
    return {"bytes": rows * H * 2.0 * row + c["batch"] * Hq * D * (e + 4.0), "flops": rows * Hq * D * 4.0}


# ------------------------------------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1_000_003 * seed + 29)
    return g


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _float_of(exponent):
    """2^(exponent - 127) of exponent bytes 1..254."""
    return (exponent.to(torch.int32) << 23).view(torch.float32)


def _quantise(x):
    """e4m3 codes and exponent bytes of fp32 rows: the least power of two that brings the largest finite value to 448 or less."""
    top = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(-1)
    m, e = torch.frexp(top)
    e = (e + (m > 0.875).to(e.dtype) - 9 + 127).clamp(1, 254)
    return (x * _float_of(254 - e)[..., None]).to(torch.float8_e4m3fn), e.to(torch.uint8)


def _group(c):
    return 16 if c["page_dtype"] else 4 if c["dtype"] == "fp32" else 8


def _pages(c, g, n_pages):
    """A pool of pages full of rows: keys scaled per token by lognormal(0, 0.5), values standard normal."""
    H, R, D, dt = c["kv_heads"], c["page_rows"], c["head_dim"], _DTYPES[c["dtype"]]
    p = {}
    for name in ("k", "v"):
        store = torch.empty(n_pages, H, R, D, dtype=torch.float8_e4m3fn if c["page_dtype"] else dt, device="cuda")
        exps = torch.ones(n_pages, H, R, dtype=torch.uint8, device="cuda") if c["page_dtype"] else None
        some = max(1, (1 << 26) // (H * R * D))
        for at in range(0, n_pages, some):                       # a part at a time bounds the fp32 temporaries
            x = torch.randn(min(some, n_pages - at), H, R, D, generator=g, device="cuda")
            if name == "k":
                x = x * torch.exp(0.5 * torch.randn(x.shape[0], 1, R, 1, generator=g, device="cuda"))
            if c["page_dtype"]:
                store[at:at + some], exps[at:at + some] = _quantise(x.to(dt).float())
            else:
                store[at:at + some] = x.to(dt)
        if name == "v":
            store = store.view(n_pages, H, R // _group(c), _group(c), D).transpose(3, 4).contiguous()
        p[name + "_pages"], p[name + "_exp"] = store, exps
    return p


def prepare(case, seed):
    c, g = case, _generator(seed)
    B, H, Hq, D, dt = c["batch"], c["kv_heads"], c["kv_heads"] * c["group"], c["head_dim"], _DTYPES[c["dtype"]]
    counts, starts = _counts(c), _starts(c)
    s = {"case": c, "stream": torch.cuda.current_stream().cuda_stream, "count": _int32(counts), "start": _int32(starts)}
    if c["kind"] in ("rotate", "append"):
        n = c["length"]
        # one projection's result per token, heads of q, k and v side by side: the rows are views of it
        qkv = torch.empty(B, n, Hq + 2 * H, D, dtype=dt, device="cuda")
        for b in range(B):
            qkv[b] = torch.randn(n, Hq + 2 * H, D, generator=g, device="cuda").to(dt)
        s["q"], s["k"], s["v"] = (x.transpose(1, 2) for x in qkv.split([Hq, H, H], dim=2))
        s["q_out"] = torch.zeros(B, Hq, n, D, dtype=dt, device="cuda")
        rot = int(D * c["rotary"])
        s["inv_freq"] = _BASE ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
        for name in ("q_weight", "k_weight"):
            s[name] = (1.0 + 0.1 * torch.randn(D, generator=g, device="cuda")).to(dt) if c["norm"] else None
    if c["kind"] == "rotate":
        s["k_out"] = torch.zeros(B, H, c["length"], D, dtype=dt, device="cuda")
    else:
        R = c["page_rows"]
        first = [x // R for x in starts]                         # pages in front are not touched: they need not be there
        last = [(x + n - 1) // R + 1 for x, n in zip(starts, counts)]
        used = sum(b - a for a, b in zip(first, last))
        cols = max(last) + 1
        ids = torch.randperm(used + 1, generator=g, device="cuda").to(torch.int32).tolist()
        table, at = [], 1
        for a, b in zip(first, last):
            table.append([ids[0]] * a + ids[at:at + b - a] + [ids[0]] * (cols - b))
            at += b - a
        s["table"] = _int32(table)
        s.update(_pages(c, g, used + 1))
    if c["kind"] == "read" or (c["kind"] == "append" and c["page_dtype"]):
        s["k_out"] = torch.zeros(B, H, c["length"], D, dtype=dt, device="cuda")
        s["v_out"] = torch.zeros_like(s["k_out"])
    if c["kind"] == "decode":
        s["q"] = torch.randn(B, Hq, D, generator=g, device="cuda").to(dt)
        s["out"] = torch.empty(B, Hq, D, device="cuda")
        s["lse"] = torch.empty(B, Hq, device="cuda")
    if own:
        from paper_2410_23079_amd import PagedCache, PagedConfig, Rotary
        if "inv_freq" in s:
            s["rotary"] = Rotary(s["q_weight"], s["k_weight"], s["inv_freq"], _EPS, c["interleaved"])
        if "table" in s:
            s["cache"] = PagedCache(
                PagedConfig(B, Hq, H, D, c["dtype"], c["page_rows"], s["k_pages"].shape[0], s["table"].shape[1],
                            page_dtype=c["page_dtype"] or None, sink=c.get("sink", 0), window=c.get("window", 0)),
                pages=(s["k_pages"], s["v_pages"], s["k_exp"], s["v_exp"]))
    return s


def run(state):
    s, kind = state, state["case"]["kind"]
    if own:
        if kind == "rotate":
            from paper_2410_23079_amd import qk_norm_rotate
            qk_norm_rotate(s["q"], s["k"], s["q_out"], s["k_out"], s["rotary"], s["start"], s["count"], stream=s["stream"])
        elif kind == "append":
            s["cache"].append(s["k"], s["v"], s["table"], s["start"], s["count"], q=s["q"], q_out=s["q_out"],
                              rotary=s["rotary"], stream=s["stream"])
        elif kind == "decode":
            s["cache"].decode(s["q"], s["table"], s["count"], s["out"], s["lse"], stream=s["stream"])
        if "v_out" in s:
            s["cache"].read(s["table"], s["start"], s["count"], s["k_out"], s["v_out"], stream=s["stream"])
    else:
        {"rotate": _plain_rotate, "append": _plain_append, "read": _plain_read, "decode": _plain_decode}[kind](s)
    names = {"rotate": ["q_out", "k_out"], "read": ["k_out", "v_out"], "decode": ["out", "lse"],
             "append": ["q_out"] + (["k_out", "v_out"] if "v_out" in s else ["k_pages", "v_pages"])}[kind]
    return {name: s[name] for name in names}


# ------------------------------------------------------------------------------------------------ plain forms
def _positions(s):
    """Position of every row [B, n], and which rows are there."""
    at = torch.arange(s["case"]["length"], device="cuda")
    return s["start"][:, None].long() + at, at < s["count"][:, None]


def _norm_rotate(s, x, weight):
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + _EPS) * weight.float()
    angle = _positions(s)[0][:, None, :, None].double() * s["inv_freq"]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    half = s["inv_freq"].numel()
    if s["case"]["interleaved"]:
        a, b, rest = x[..., 0:2 * half:2], x[..., 1:2 * half:2], x[..., 2 * half:]
        return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), rest], -1)
    a, b, rest = x[..., :half], x[..., half:2 * half], x[..., 2 * half:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1)


def _keep(s, name, x):
    """Rows that are there go to the output, the others stay as they were."""
    there = _positions(s)[1][:, None, :, None]
    s[name] = torch.where(there, x.to(s[name].dtype), s[name])


def _plain_rotate(s):
    _keep(s, "q_out", _norm_rotate(s, s["q"], s["q_weight"]))
    _keep(s, "k_out", _norm_rotate(s, s["k"], s["k_weight"]))


def _plain_append(s):
    c = s["case"]
    _keep(s, "q_out", _norm_rotate(s, s["q"], s["q_weight"]))
    k, v = _norm_rotate(s, s["k"], s["k_weight"]), s["v"].float()
    pos, there = _positions(s)
    R, G = c["page_rows"], _group(c)
    page = torch.gather(s["table"].long(), 1, (pos // R).clamp(max=s["table"].shape[1] - 1))[there]
    row = (pos % R)[there]
    k, v = k.transpose(1, 2)[there], v.transpose(1, 2)[there]    # [rows, H, D]
    if c["page_dtype"]:
        k, s["k_exp"][page, :, row] = _quantise(k)
        v, s["v_exp"][page, :, row] = _quantise(v)
        # torch has no indexed writes of 8-bit floats: the codes go as bytes
        s["k_pages"].view(torch.uint8)[page, :, row] = k.view(torch.uint8)
        s["v_pages"].view(torch.uint8)[page, :, row // G, :, row % G] = v.view(torch.uint8)
        _plain_read(s)
    else:
        s["k_pages"][page, :, row] = k.to(s["k_pages"].dtype)
        s["v_pages"][page, :, row // G, :, row % G] = v.to(s["v_pages"].dtype)


def _rows(s, page, row):
    """fp32 keys and values [..., H, D] of (page, row) pairs."""
    G = _group(s["case"])
    k, v = s["k_pages"], s["v_pages"]
    if s["case"]["page_dtype"]:
        k = k.view(torch.uint8)[page, :, row].view(torch.float8_e4m3fn).float() * _float_of(s["k_exp"][page, :, row])[..., None]
        v = v.view(torch.uint8)[page, :, row // G, :, row % G].view(torch.float8_e4m3fn).float() * _float_of(s["v_exp"][page, :, row])[..., None]
        return k, v
    return k[page, :, row].float(), v[page, :, row // G, :, row % G].float()


def _plain_read(s):
    pos, there = _positions(s)
    page = torch.gather(s["table"].long(), 1, (pos // s["case"]["page_rows"]).clamp(max=s["table"].shape[1] - 1))
    k, v = _rows(s, page, pos % s["case"]["page_rows"])          # [B, n, H, D]
    _keep(s, "k_out", k.transpose(1, 2))
    _keep(s, "v_out", v.transpose(1, 2))


def _plain_decode(s):
    c = s["case"]
    B, H, G, D, R = c["batch"], c["kv_heads"], c["group"], c["head_dim"], c["page_rows"]
    j = torch.arange(c["length"], device="cuda")
    there = j < s["count"][:, None]                              # [B, n]
    if c["window"]:
        there = there & ((j >= s["count"][:, None] - c["window"]) | (j < c["sink"]))
    page = torch.gather(s["table"].long(), 1, (j // R).expand(B, -1))
    k, v = _rows(s, page, (j % R).expand(B, -1))
    k, v = k.transpose(1, 2), v.transpose(1, 2)                  # [B, H, n, D]
    q = s["q"].float().view(B, H, G, D)
    logit = torch.matmul(q, k.transpose(2, 3)) * (1.0 / math.sqrt(D))
    logit = torch.where(there[:, None, None, :], logit, -math.inf)
    top = logit.amax(-1, keepdim=True)
    p = torch.exp(logit - top)
    total = p.sum(-1, keepdim=True)
    s["out"] = (torch.matmul(p, v) / total).view(B, H * G, D)
    s["lse"] = (top + torch.log(total)).view(B, H * G)


# ------------------------------------------------------------------------------------------------ in 64 bits
def _exact_turn(s, x, weight):
    """Norm and rotation of one sequence's rows [H, n, D], pairs as complex numbers; s: its positions in "at"."""
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / x.shape[-1] + _EPS) * weight.double()
    half = s["inv_freq"].numel()
    turn = torch.polar(torch.ones_like(s["at"][:, None] * s["inv_freq"]), s["at"][:, None] * s["inv_freq"])
    head = x[..., :2 * half]
    pairs = head.unflatten(-1, (half, 2)) if s["case"]["interleaved"] else head.unflatten(-1, (2, half)).transpose(-1, -2)
    turned = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    if not s["case"]["interleaved"]:
        turned = turned.transpose(-1, -2)
    return torch.cat([turned.flatten(-2), x[..., 2 * half:]], -1)


def _exact_e4m3(x):
    """What 64-bit rows become in an 8-bit page: three mantissa bits, 2^-9 the smallest step, relative to the row's power of two."""
    top = x.abs().amax(-1, keepdim=True)
    power = torch.ceil(torch.log2(top.clamp(min=1e-300) / 448.0))
    power = torch.where(top > 448.0 * torch.exp2(power), power + 1, torch.where(top <= 448.0 * torch.exp2(power - 1), power - 1, power)).clamp(min=-126)
    y = x * torch.exp2(-power)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step * torch.exp2(power)


def exact(case, seed):
    global own
    before, own = own, False
    s = prepare(case, seed)
    own = before
    c = case
    counts, starts, D = _counts(c), _starts(c), c["head_dim"]
    R = c.get("page_rows", 1)

    def stored(b, first, n):
        """One sequence's rows [H, n, D] out of its pages, page by page in the table's order."""
        pages = s["table"][b, first // R:(first + n - 1) // R + 1].long()
        got = []
        for name in ("k", "v"):
            x = s[name + "_pages"][pages] if not c["page_dtype"] else s[name + "_pages"].view(torch.uint8)[pages].view(torch.float8_e4m3fn)
            x = x.double()
            if name == "v":
                x = x.permute(0, 1, 2, 4, 3).flatten(2, 3)
            if c["page_dtype"]:
                x = x * torch.exp2(s[name + "_exp"][pages].double() - 127.0)[..., None]
            got.append(x.transpose(0, 1).flatten(1, 2)[:, first % R:first % R + n])
        return got

    if c["kind"] == "decode":
        out, lse = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda"), torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
        for b, n in enumerate(counts):
            k, v = stored(b, 0, n)
            q = s["q"][b].double().view(c["kv_heads"], c["group"], D)
            logit = torch.matmul(q, k.transpose(1, 2)) / math.sqrt(D)
            if c["window"]:
                j = torch.arange(n, device="cuda")
                logit[..., (j < n - c["window"]) & (j >= c["sink"])] = -math.inf
            lse[b] = torch.logsumexp(logit, -1).flatten()
            out[b] = torch.matmul(torch.exp(logit - lse[b].view(c["kv_heads"], c["group"], 1)), v).view(-1, D)
        return {"out": out, "lse": lse}
    res = {name: s[name].double() for name in ("q_out", "k_out", "v_out") if name in s}
    if c["kind"] == "append" and "v_out" not in s:
        res["k_pages"], res["v_pages"] = s["k_pages"].double(), s["v_pages"].double()
    for b, (first, n) in enumerate(zip(starts, counts)):
        s["at"] = torch.arange(first, first + n, device="cuda", dtype=torch.float64)
        if c["kind"] == "read":
            res["k_out"][b, :, :n], res["v_out"][b, :, :n] = stored(b, first, n)
            continue
        res["q_out"][b, :, :n] = _exact_turn(s, s["q"][b, :, :n], s["q_weight"])
        k = _exact_turn(s, s["k"][b, :, :n], s["k_weight"])
        if c["kind"] == "rotate":
            res["k_out"][b, :, :n] = k
        elif c["page_dtype"]:
            res["k_out"][b, :, :n], res["v_out"][b, :, :n] = _exact_e4m3(k), _exact_e4m3(s["v"][b, :, :n].double())
        else:
            v, g = s["v"][b, :, :n].double(), _group(c)
            at = torch.arange(first, first + n, device="cuda")
            flat = s["table"][b].long()[torch.div(at, R, rounding_mode="floor")] * R + at % R   # rows numbered through the pool
            kp = res["k_pages"].transpose(1, 2).flatten(0, 1).clone()
            kp[flat] = k.transpose(0, 1)
            res["k_pages"] = kp.unflatten(0, (-1, R)).transpose(1, 2).contiguous()
            vp = res["v_pages"].permute(0, 2, 4, 1, 3).flatten(0, 2).clone()
            vp[flat] = v.transpose(0, 1)
            res["v_pages"] = vp.unflatten(0, (-1, R // g, g)).permute(0, 3, 1, 4, 2).contiguous()
    return res

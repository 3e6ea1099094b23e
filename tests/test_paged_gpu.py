"""The paged cache and the position rotation on the GPU against plain computations in 64 bits.

Tolerances count roundings.  u = 2^-24 is half a step of fp32; a result in type t may be off by eps(t) / 2 of its value more.
  norm + rotation   the sum of squares adds at most 8 + 6 terms one after the other (14 u, halved by the root), mean, root,
                    division, two products 5 u; cosine and sine are right to 4 u, two products and a sum 3 u more: at most 20 u
                    of |x| + |y| of the pair after the norm
  8-bit rows        half a step of e4m3 (2^-4 of the value's power of two, at least 2^-10 of the row's) on top of the above
  decode            logits: D products summed in at most D + 8 steps, (D + 8) u of scale * sum |q_i k_i|, twice (numerator and
                    sum), and 2 u of the logit for its product with log2 e; exp2 2 u; weights of 22 bits (2^-23, twice); sums
                    over N keys in at most N / 16 + 64 steps.  All of it of sum_j p_j |v_j|
"""
import math

import numpy as np
import pytest
import torch

from paper_2410_23079_amd import BuzzCache, BuzzConfig, BuzzError, PagedCache, PagedConfig, Rotary, qk_norm_rotate

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
PAGES = [("fp32", None), ("fp16", None), ("bf16", None), ("fp16", "e4m3"), ("bf16", "e4m3")]


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(g, *shape, dtype="fp32", scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(DT[dtype])


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def half_step(dtype):
    return torch.finfo(DT[dtype]).eps / 2


# ------------------------------------------------------------------------------------------------ the oracle
def turned(x, pos, weight, rot):
    """(norm and rotation in 64 bits, the sum of magnitudes that an element's error is measured by); x [..., n, D], pos [n]."""
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt(x.pow(2).mean(-1, keepdim=True) + rot.c.eps) * weight.double()
    y, mag = x.clone(), x.abs()
    if rot is not None and rot.inv_freq is not None:
        f = rot.inv_freq
        a = torch.tensor(pos, dtype=torch.float64, device="cuda")[:, None] * f
        h = f.numel()
        i, j = (slice(0, 2 * h, 2), slice(1, 2 * h, 2)) if rot.c.interleaved else (slice(0, h), slice(h, 2 * h))
        y[..., i] = x[..., i] * a.cos() - x[..., j] * a.sin()
        y[..., j] = x[..., j] * a.cos() + x[..., i] * a.sin()
        mag = mag.clone()
        mag[..., i] = mag[..., j] = x[..., i].abs() + x[..., j].abs()
    return y, mag


def assert_within(got, want, tol, what=""):
    got, want = got.double(), want.double()
    assert torch.equal(got.isnan(), want.isnan()), f"{what}: NaN in other places"
    if got.numel() == 0:
        return
    far = ((got - want).abs() - tol).nan_to_num(nan=-1.0)
    assert float(far.max()) <= 0, f"{what}: {float((got - want).abs().nan_to_num().max())} off, {float(far.max())} more than it may be"


def v_rows(pages):
    """Values [page][head][row][dim] of pages [page][head][row / g][dim][g]."""
    p = pages.view(torch.uint8) if pages.dtype == torch.float8_e4m3fn else pages
    n, H, R, D, g = p.shape
    p = p.transpose(3, 4).reshape(n, H, R * g, D)
    return p.view(torch.float8_e4m3fn) if pages.dtype == torch.float8_e4m3fn else p


def in_v_order(rows, g):
    """The inverse."""
    n, H, R, D = rows.shape
    p = rows.view(torch.uint8) if rows.dtype == torch.float8_e4m3fn else rows
    p = p.view(n, H, R // g, g, D).transpose(3, 4).contiguous()
    return p.view(torch.float8_e4m3fn) if rows.dtype == torch.float8_e4m3fn else p


def values(cache):
    """Keys and values of all pages in 64 bits, [page][head][row][dim]."""
    k, v = cache.k_pages.float().double(), v_rows(cache.v_pages).float().double()
    if cache.k_exp is not None:
        k = k * torch.exp2(cache.k_exp.double() - 127)[..., None]
        v = v * torch.exp2(cache.v_exp.double() - 127)[..., None]
    return k, v


def exponents(top):
    """The least e in 1 .. 254 with top <= 448 * 2^(e - 127), by trying."""
    e = torch.full_like(top, 1, dtype=torch.int64)
    for x in range(2, 255):
        e = torch.where(top > 448.0 * 2.0 ** (x - 1 - 127), x, e)
    return e


def pool(B, H, G, D, dtype, page_dtype, R, n_pages, cols, fill="nan", **kw):
    c = PagedCache(PagedConfig(B, H * G, H, D, dtype, R, n_pages, cols, page_dtype=page_dtype, **kw))
    for t in (c.k_pages, c.v_pages):
        t.view(torch.uint8).fill_(0xff)            # NaN in every type
    if c.k_exp is not None:
        c.k_exp.fill_(255)
        c.v_exp.fill_(255)
    return c


def tables(seed, lengths, R, n_pages, cols, first=None):
    """A page table with pages of their own, in random order, for tokens first .. length - 1; the rest are no pages."""
    ids = np.random.RandomState(seed).permutation(n_pages).tolist()
    none = [-1, n_pages, 2 ** 31 - 1, -2 ** 31]
    t = [[none[(b + c) % 4] for c in range(cols)] for b in range(len(lengths))]
    for b, n in enumerate(lengths):
        for c in range((first[b] if first else 0) // R, (n + R - 1) // R):
            t[b][c] = ids.pop()
    return t


# ------------------------------------------------------------------------------------------------ norm and rotation
@pytest.mark.parametrize("dtype,D,rot,interleaved,norm,n,B,Hq,Hkv", [
    ("fp32", 64, 64, False, True, 1, 1, 4, 4), ("fp32", 128, 32, True, False, 37, 2, 3, 1), ("fp32", 256, 256, False, True, 16, 1, 9, 2),
    ("fp16", 64, 16, False, False, 50, 3, 2, 2), ("fp16", 128, 128, False, True, 1, 8, 32, 8), ("fp16", 256, 64, True, True, 33, 1, 5, 5),
    ("bf16", 64, 64, True, True, 129, 1, 17, 1), ("bf16", 128, 64, False, True, 100, 2, 40, 10), ("bf16", 256, 0, False, True, 5, 2, 2, 1),
    ("bf16", 128, 112, False, False, 31, 1, 1, 1)])
def test_norm_and_rotation(dtype, D, rot, interleaved, norm, n, B, Hq, Hkv):
    g = gen(n * 7 + D)
    qkv = randn(g, B, n, Hq + 2 * Hkv, D, dtype=dtype)                         # rows are slices of one projection's result
    q, k = qkv[:, :, :Hq].transpose(1, 2), qkv[:, :, Hq:Hq + Hkv].transpose(1, 2)
    w = [randn(g, D, dtype=dtype) if norm else None for _ in range(2)]
    r = Rotary(*w, inv_freq=10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / max(rot, 1)) if rot else None,
               eps=1e-5, interleaved=interleaved)
    start = [(0, 131071, 77, 5)[b % 4] * (b + 1) for b in range(B)]
    count = [n - (3 * b) % (n + 1) for b in range(B)]
    q_out, k_out = torch.full((B, Hq, n, D), 7.0, dtype=DT[dtype], device="cuda"), torch.full((B, n, Hkv, D), 7.0, dtype=DT[dtype], device="cuda").transpose(1, 2)
    print("norm_rotate", dtype, D, rot, n, flush=True)
    qk_norm_rotate(q, k, q_out, k_out, r, ints(start), ints(count))
    for x, out, weight in ((q, q_out, w[0]), (k, k_out, w[1])):
        for b in range(B):
            want, mag = turned(x[b, :, :count[b]], [start[b] + t for t in range(count[b])], weight, r)
            assert_within(out[b, :, :count[b]], want, 20 * U * mag + half_step(dtype) * want.abs() + (2.0 ** -25 if dtype == "fp16" else 0), f"sequence {b}")
            assert bool((out[b, :, count[b]:] == 7.0).all())                   # rows that are not there


def test_rotation_in_place_without_starts_and_of_one_kind_only():
    g = gen(1)
    q = randn(g, 2, 6, 40, 128, dtype="bf16")
    r = Rotary(inv_freq=torch.rand(64, generator=g, device="cuda", dtype=torch.float64))
    apart, here = torch.empty_like(q), q.clone()
    qk_norm_rotate(q, None, apart, None, r)
    qk_norm_rotate(here, None, here, None, r)
    assert torch.equal(apart, here)
    k = torch.empty_like(q)
    qk_norm_rotate(None, q, None, k, r, ints([0, 0]))
    assert torch.equal(apart, k)
    assert torch.equal(apart[:, :, 0], q[:, :, 0])                             # position 0 does not turn


def test_rows_of_a_sequence_with_a_negative_start_stay_and_counts_are_clamped():
    q = randn(gen(2), 3, 2, 5, 64)
    out = torch.full_like(q, 3.0)
    r = Rotary(q_weight=torch.ones(64, device="cuda"), eps=0.0)
    qk_norm_rotate(q, None, out, None, r, ints([-1, 4, 2 ** 31 - 1]), ints([5, 99, -3]))
    assert bool((out[0] == 3.0).all()) and bool((out[2] == 3.0).all())
    want, mag = turned(q[1], [4 + t for t in range(5)], r.q_weight, r)
    assert_within(out[1], want, 20 * U * mag + half_step("fp32") * want.abs())


def test_a_far_position_keeps_its_phase():
    """2^31 - 9 .. 2^31: in 32 bits the angle itself would be off by tens of turns' fractions."""
    q = torch.ones(1, 1, 9, 64, device="cuda")
    r = Rotary(inv_freq=torch.linspace(1.0, 0.01, 32, dtype=torch.float64, device="cuda"))
    out = torch.empty_like(q)
    qk_norm_rotate(q, None, out, None, r, ints([2 ** 31 - 9]))
    want, mag = turned(q, [2 ** 31 - 9 + t for t in range(9)], None, r)
    # both sides form the angle in 64 bits: 2^31 radians to 2^-22 each
    assert_within(out, want, (20 * U + 2 * 2.0 ** -22) * mag)


# ------------------------------------------------------------------------------------------------ append and read
@pytest.mark.parametrize("dtype,page_dtype", PAGES)
@pytest.mark.parametrize("D,H,G,R,n,starts,counts", [
    (64, 2, 1, 16, 1, [0, 15, 16, 100], [1, 1, 1, 0]), (128, 3, 4, 32, 45, [0, 3, 31, 90], [45, 44, 1, 17]),
    (256, 1, 2, 64, 70, [7, 64, 0], [70, 16, 65]), (128, 9, 1, 256, 33, [250], [33]), (64, 17, 2, 128, 16, [16, 1], [16, 15])])
def test_append_and_read(dtype, page_dtype, D, H, G, R, n, starts, counts):
    g, B = gen(D + n), len(starts)
    lengths = [s + c for s, c in zip(starts, counts)]
    cols = max((x + R - 1) // R for x in lengths) + 1
    n_pages = sum((x + R - 1) // R for x in lengths) + 2
    table = tables(n, lengths, R, n_pages, cols, starts)
    c = pool(B, H, G, D, dtype, page_dtype, R, n_pages, cols)
    k, v, q = randn(g, B, n, H, D, dtype=dtype).transpose(1, 2), randn(g, B, H, n, D, dtype=dtype, scale=3.0), randn(g, B, H * G, n, D, dtype=dtype)
    v[0, 0, 0] = 0.0
    v[:, :, n // 2, 3] = float("inf")
    v[:, :, n // 3, 5] = float("nan")
    rot = D // 2
    r = Rotary(q_weight=randn(g, D, dtype=dtype), k_weight=randn(g, D, dtype=dtype),
               inv_freq=torch.rand(rot // 2, generator=g, device="cuda", dtype=torch.float64))
    q_out = torch.full_like(q, 9.0)
    before = [t.clone() if t is not None else None for t in (c.k_pages, c.v_pages, c.k_exp, c.v_exp)]
    print("append", dtype, page_dtype, D, R, flush=True)
    c.append(k, v, ints(table), ints(starts), ints(counts), q=q, q_out=q_out, rotary=r)
    kp, vp = values(c)
    touched = torch.zeros(n_pages, R, dtype=torch.bool, device="cuda")
    for b in range(B):
        pos = list(range(starts[b], starts[b] + counts[b]))
        want, mag = turned(q[b, :, :counts[b]], pos, r.q_weight, r)
        assert_within(q_out[b, :, :counts[b]], want, 20 * U * mag + half_step(dtype) * want.abs() + (2.0 ** -25 if dtype == "fp16" else 0), "queries")
        assert bool((q_out[b, :, counts[b]:] == 9.0).all())
        want_k, mag = turned(k[b, :, :counts[b]], pos, r.k_weight, r)
        for t, p in enumerate(pos):
            page, row = table[b][p // R], p % R
            touched[page, row] = True
            x, y = kp[page, :, row], want_k[:, t]
            if page_dtype:
                top = y.abs().amax(-1)
                e = c.k_exp[page, :, row].long()
                slack = 20 * U * mag[:, t].amax(-1)
                assert bool((e >= exponents(top - slack)).all()) and bool((e <= exponents(top + slack)).all())
                unit = torch.exp2(e.double() - 127)[:, None]
                step = torch.exp2(torch.floor(torch.log2(torch.maximum(x.abs(), y.abs()).div(unit).clamp(min=2.0 ** -6))) - 3) * unit
                assert_within(x, y, step / 2 + 20 * U * mag[:, t], f"key {t}")
            else:
                assert_within(x, y, 20 * U * mag[:, t] + half_step(dtype) * y.abs() + (2.0 ** -25 if dtype == "fp16" else 0), f"key {t}")
            y = v[b, :, t].double()
            if page_dtype:                                                     # values are stored as they are: exactly known
                fine = torch.where(y.isfinite(), y, 0.0)
                e = exponents(fine.abs().amax(-1))
                assert torch.equal(c.v_exp[page, :, row].long(), e)
                y = torch.where(y.isfinite(), y, math.nan)
                code = (y * torch.exp2(127.0 - e.double())[:, None]).float().to(torch.float8_e4m3fn).double()
                y = code * torch.exp2(e.double() - 127)[:, None]
            assert torch.equal(vp[page, :, row].nan_to_num(nan=1e30), y.nan_to_num(nan=1e30)), f"value {t}"
    # nothing else was written
    rest = ~touched
    assert torch.equal(c.k_pages.view(torch.uint8).transpose(1, 2)[rest], before[0].view(torch.uint8).transpose(1, 2)[rest])
    assert torch.equal(v_rows(c.v_pages).view(torch.uint8).transpose(1, 2)[rest], v_rows(before[1]).view(torch.uint8).transpose(1, 2)[rest])
    if page_dtype:
        for now, then in ((c.k_exp, before[2]), (c.v_exp, before[3])):
            assert torch.equal(now.transpose(1, 2)[rest], then.transpose(1, 2)[rest])
    # and back: the stored values, rounded to the rows' type once
    k_back, v_back = torch.full_like(v, 9.0), torch.full((B, n, H, D), 9.0, dtype=DT[dtype], device="cuda").transpose(1, 2)
    c.read(ints(table), ints(starts), ints(counts), k_back, v_back)
    for b in range(B):
        for t in range(n):
            if t >= counts[b]:
                assert bool((k_back[b, :, t] == 9.0).all()) and bool((v_back[b, :, t] == 9.0).all())
                continue
            page, row = table[b][(starts[b] + t) // R], (starts[b] + t) % R
            assert torch.equal(k_back[b, :, t], kp[page, :, row].to(DT[dtype]))
            assert torch.equal(v_back[b, :, t].nan_to_num(nan=77.0), vp[page, :, row].to(DT[dtype]).nan_to_num(nan=77.0))


def test_eight_bit_rows_at_the_ends_of_the_range():
    """The largest and smallest magnitudes, powers of two and borders of the exponent rule, ties and subnormal codes."""
    tops = torch.tensor([0.0, 1.0, 448.0, 448.25, 449.0, 1.75, 1.7578125, 65504.0, 2.0 ** -24, 0.875, 3.0, 3.3e38, 1e-38, 2.0 ** -126])
    v = torch.zeros(1, 1, 16, 64)
    v[0, 0, :14, 0] = tops
    v[0, 0, :, 1] = v[0, 0, :, 0] / 16 * 1.0625                                # a tie between two codes for powers of two
    v[0, 0, :, 2] = -v[0, 0, :, 0] / 1000
    v[0, 0, :, 3] = v[0, 0, :, 0] / 2 ** 17
    v[0, 0, 14] = float("inf")
    v[0, 0, 15] = -float("nan")
    v = v.to(torch.bfloat16).cuda()
    c = pool(1, 1, 1, 64, "bf16", "e4m3", 16, 1, 1)
    c.append(v, v, ints([[0]]))
    y = v[0, 0].double()
    e = exponents(torch.where(y.isfinite(), y.abs(), 0.0).amax(-1))
    code = (torch.where(y.isfinite(), y, math.nan) * torch.exp2(127.0 - e.double())[:, None]).float().to(torch.float8_e4m3fn).double()
    want = (code * torch.exp2(e.double() - 127)[:, None]).nan_to_num(nan=-5.0)
    for pages, exp in ((c.k_pages, c.k_exp), (v_rows(c.v_pages), c.v_exp)):
        assert torch.equal(exp[0, 0].long(), e)
        assert torch.equal((pages[0, 0].float().double() * torch.exp2(exp[0, 0].double() - 127)[:, None]).nan_to_num(nan=-5.0), want)


def test_rows_without_a_page_are_dropped_and_read_as_nan():
    c = pool(2, 1, 1, 64, "fp16", None, 16, 3, 3)
    x = randn(gen(3), 2, 1, 40, 64, dtype="fp16")
    table = ints([[0, -1, 3], [2 ** 31 - 1, 1, 2]])
    print("bad pages", flush=True)
    c.append(x, x, table, ints([0, 16]), ints([40, 40]))                       # positions 48 .. 55 lie beyond the table
    k, v = torch.zeros_like(x), torch.zeros_like(x)
    c.read(table, ints([0, 16]), ints([40, 40]), k, v)
    for got in (k, v):
        assert torch.equal(got[0, 0, :16], x[0, 0, :16]) and bool(got[0, 0, 16:].isnan().all())
        assert torch.equal(got[1, 0, :32], x[1, 0, :32]) and bool(got[1, 0, 32:].isnan().all())


# ------------------------------------------------------------------------------------------------ decode
def attention(cache, q, table, lengths, scale=None):
    """(out, lse, how far each may be off) in 64 bits for cache.cfg's mask."""
    c, (k, v) = cache.cfg, values(cache)
    H, G, D, R = c.n_kv_heads, c.n_q_heads // c.n_kv_heads, c.head_dim, c.page_rows
    scale = scale or 1.0 / math.sqrt(D)
    out, lse = torch.zeros(len(lengths), H * G, D, dtype=torch.float64, device="cuda"), torch.full((len(lengths), H * G), -math.inf, dtype=torch.float64, device="cuda")
    tol_o, tol_l = torch.zeros_like(out), torch.zeros_like(lse)
    for b, n in enumerate(lengths):
        js = [j for j in range(n) if c.window == 0 or j >= n - c.window or j < c.sink]
        if not js:
            continue
        pages, rows = [table[b][j // R] for j in js], [j % R for j in js]
        kb, vb = k[pages, :, rows].transpose(0, 1), v[pages, :, rows].transpose(0, 1)          # [H, N, D]
        qb = q[b].double().view(H, G, D)
        s = torch.matmul(qb, kb.transpose(1, 2)) * scale
        top = s.amax(-1, keepdim=True)
        p = torch.exp(s - top)
        total = p.sum(-1, keepdim=True)
        out[b] = (torch.matmul(p, vb) / total).view(-1, D)
        lse[b] = (top + total.log()).flatten()
        ds = (D + 8) * U * scale * torch.matmul(qb.abs(), kb.abs().nan_to_num(posinf=0.0).transpose(1, 2)) + 2 * U * s.abs().nan_to_num(posinf=0.0, neginf=0.0)
        ds = torch.where(p > 0, ds, 0.0).amax(-1, keepdim=True)
        sums = (len(js) / 16 + 64) * U
        tol_o[b] = ((2 * ds + 2.0 ** -22 + sums + 4 * U) * torch.matmul(p, vb.abs()) / total).view(-1, D)
        tol_l[b] = (ds + sums + 4 * U + 4 * U * (top + total.log()).abs()).flatten()
    return out, lse, tol_o, tol_l


def filled(seed, lengths, H, G, D, dtype, page_dtype, R, spread=0.5, cols=None, spare=2, **kw):
    """A pool in which the sequences' tokens, and nothing else, hold numbers; with its page table."""
    g, B = gen(seed), len(lengths)
    need = [(n + R - 1) // R for n in lengths]
    cols = cols or max(need) + 1
    table = tables(seed, lengths, R, sum(need) + spare, cols)
    c = pool(B, H, G, D, dtype, page_dtype, R, sum(need) + spare, cols, **kw)
    n = max(max(lengths), 1)
    k = randn(g, B, H, n, D) * torch.exp(spread * randn(g, B, 1, n, 1))
    c.append(k.to(DT[dtype]), randn(g, B, H, n, D, dtype=dtype), ints(table), None, ints(lengths))
    return c, table, randn(g, B, H * G, D, dtype=dtype)


def check_decode(c, table, q, lengths, what, **kw):
    B = len(lengths)
    out, lse = torch.full((B, c.cfg.n_q_heads, c.cfg.head_dim), 5.0, device="cuda"), torch.full((B, c.cfg.n_q_heads), 5.0, device="cuda")
    print("decode", what, flush=True)
    c.decode(q, ints(table), ints(lengths), out, lse)
    want, want_l, tol, tol_l = attention(c, q, table, lengths, **kw)
    assert_within(out, want, tol, what)
    empty = ints(lengths) == 0
    assert bool((lse[empty] == -math.inf).all()) and bool((out[empty] == 0).all())
    assert_within(lse[~empty], want_l[~empty], tol_l[~empty], what + " lse")
    return out, lse


LENGTHS = [[1], [0, 1, 2], [15, 16, 17, 0, 64], [63, 64, 65, 128, 33, 1], [300, 5, 1111, 32], [4099]]


@pytest.mark.parametrize("dtype,page_dtype", PAGES)
@pytest.mark.parametrize("D,H,G", [(64, 2, 1), (128, 3, 4), (256, 1, 8), (128, 1, 7)])
@pytest.mark.parametrize("lengths", LENGTHS, ids=str)
def test_decode(dtype, page_dtype, D, H, G, lengths):
    R = (16, 32, 64, 128, 256)[(D // 64 + H + G + len(lengths)) % 5]
    c, table, q = filled(len(lengths) * 31 + D, lengths, H, G, D, dtype, page_dtype, R)
    check_decode(c, table, q, lengths, f"{dtype} {page_dtype} D {D} G {G} R {R} {lengths}")


@pytest.mark.parametrize("dtype,page_dtype", PAGES)
@pytest.mark.parametrize("R", [16, 256])
def test_decode_long(dtype, page_dtype, R):
    """One long sequence beside short ones: its blocks are many, its partial results are added up by the last of them."""
    lengths = [40001, 17, 0, 2500]
    c, table, q = filled(5, lengths, 2, 3, 64, dtype, page_dtype, R)
    check_decode(c, table, q, lengths, f"long {dtype} {page_dtype} R {R}")


@pytest.mark.parametrize("dtype,page_dtype", [("fp32", None), ("bf16", None), ("fp16", "e4m3")])
def test_decode_of_many_sequences(dtype, page_dtype):
    """More sequences than lanes in a wave, more pairs than blocks."""
    lengths = [int(x) for x in np.random.RandomState(1).randint(0, 90, size=391)]
    c, table, q = filled(6, lengths, 3, 2, 64, dtype, page_dtype, 32)
    check_decode(c, table, q, lengths, f"many {dtype} {page_dtype}")


@pytest.mark.parametrize("B,H,G,D,dtype,page_dtype,longest,mask", [
    (70, 40, 1, 64, "bf16", None, 60, {}),                     # more pairs than waves, each a wave's; two lengths to a lane
    (64, 8, 2, 128, "fp16", None, 480, {}), (70, 8, 1, 128, "bf16", None, 768, {}),   # two to a block, a wave's up to 24 tiles
    (70, 8, 1, 128, "bf16", None, 769, {}), (70, 8, 1, 128, "bf16", None, 1025, {}),  # whole for a block up to 32; cut
    (70, 9, 2, 128, "fp16", "e4m3", 740, dict(sink=7, window=300)), (35, 60, 1, 64, "fp32", None, 700, {}),   # a wave's
    (40, 8, 1, 64, "bf16", "e4m3", 2500, {}),                  # blocks with parts of several pairs
    (33, 8, 3, 256, "bf16", None, 900, {}), (20, 8, 2, 128, "fp32", None, 1500, {}), (66, 4, 5, 256, "fp16", "e4m3", 400, {}),
    (48, 4, 8, 128, "fp16", "e4m3", 3000, dict(sink=100, window=1000)), (90, 3, 4, 128, "bf16", None, 1300, dict(sink=7, window=300)),
    (2, 60, 1, 128, "bf16", None, 5000, {}), (3, 30, 2, 64, "fp16", None, 9000, {})])   # few pairs: a unit to every block
def test_shares_of_blocks(B, H, G, D, dtype, page_dtype, longest, mask):
    lengths = [int(x) for x in np.random.RandomState(B + H).randint(0, longest + 1, size=B)]
    lengths[B // 2] = longest
    c, table, q = filled(B * 100 + H, lengths, H, G, D, dtype, page_dtype, 64, **mask)
    check_decode(c, table, q, lengths, f"shares {B} {H} {D} {dtype} {page_dtype} {longest}")


@pytest.mark.parametrize("dtype,page_dtype", PAGES)
@pytest.mark.parametrize("sink,window", [(0, 1), (4, 8), (1, 64), (70, 33), (500, 100), (16, 1000)])
def test_decode_with_sink_and_window(dtype, page_dtype, sink, window):
    """Tokens that the mask hides have no pages: they are not looked at."""
    lengths, R = [1, 9, 77, 129, 700, 0, 701], 32
    c, table, q = filled(7, lengths, 2, 2, 128, dtype, page_dtype, R, sink=sink, window=window)
    for b, n in enumerate(lengths):
        for col in range(len(table[b])):
            if all(j >= sink and j < n - window for j in range(col * R, col * R + R)):
                table[b][col] = -7
    check_decode(c, table, q, lengths, f"sink {sink} window {window} {dtype} {page_dtype}")


@pytest.mark.parametrize("dtype,page_dtype", PAGES)
def test_a_page_that_is_none_gives_nan_for_its_sequence_alone(dtype, page_dtype):
    lengths = [100, 4000, 90, 100]
    c, table, q = filled(8, lengths, 2, 2, 64, dtype, page_dtype, 16)
    good = check_decode(c, table, q, lengths, "good")
    table[0][6], table[1][200] = c.cfg.n_pages, -1
    out, lse = torch.empty_like(good[0]), torch.empty_like(good[1])
    c.decode(q, ints(table), ints(lengths), out, lse)
    for got, want in ((out, good[0]), (lse, good[1])):
        assert bool(got[:2].isnan().all()) and torch.equal(got[2:], want[2:])


def test_lengths_that_are_none_give_nan_for_their_sequence_alone():
    lengths = [60, 64, 10, 64]
    c, table, q = filled(9, lengths, 1, 2, 64, "bf16", None, 16, cols=4)
    good = check_decode(c, table, q, lengths, "good")
    out, lse = torch.empty_like(good[0]), torch.empty_like(good[1])
    c.decode(q, ints(table), ints([60, 65, 10, -1]), out, lse)
    for got, want in ((out, good[0]), (lse, good[1])):
        assert bool(got[1::2].isnan().all()) and torch.equal(got[::2], want[::2])
    c.decode(q, ints(table), ints([-2 ** 31, 2 ** 31 - 1, 0, 0]), out, lse)
    assert bool(out[:2].isnan().all()) and bool((out[2:] == 0).all()) and bool((lse[2:] == -math.inf).all())


@pytest.mark.parametrize("dtype,page_dtype", PAGES)
def test_shared_pages_strided_queries_scale_and_far_logits(dtype, page_dtype):
    """Two sequences on the same pages; queries out of a wider row; logits that leave the range of exp in 32 bits."""
    lengths = [200, 150, 200]
    c, table, _ = filled(10, lengths, 2, 4, 64, dtype, page_dtype, 32, softmax_scale=1.7)
    table[2], table[1] = table[0], table[0]
    wide = randn(gen(11), 3, 2, 8, 64, dtype=dtype, scale=12.0)
    check_decode(c, table, wide[:, 1], lengths, "strided", scale=float(np.float32(1.7)))


@pytest.mark.parametrize("dtype", ["fp32", "fp16", "bf16"])
def test_infinite_keys_and_nan_values(dtype):
    """A logit of -infinity takes no part, one of +infinity or NaN makes its heads NaN, a NaN value its column."""
    lengths, D = [70, 70, 70, 70], 64
    c, table, _ = filled(12, lengths, 1, 1, D, dtype, None, 16)
    q = torch.ones(4, 1, D, dtype=DT[dtype], device="cuda")
    c.k_pages[table[0][0], 0, 3, 5] = -math.inf
    c.k_pages[table[1][4], 0, 2, 5] = math.inf
    c.k_pages[table[2][1], 0, 1, 9] = math.nan
    g = c.v_pages.shape[-1]
    c.v_pages[table[3][2], 0, 8 // g, 6, 8 % g] = math.nan
    out, lse = torch.empty(4, 1, D, device="cuda"), torch.empty(4, 1, device="cuda")
    c.decode(q, ints(table), ints(lengths), out, lse)
    want, want_l, tol, tol_l = attention(c, q, table, lengths)
    assert_within(out[0], want[0], tol[0])
    assert_within(lse[0], want_l[0], tol_l[0])
    assert bool(out[1].isnan().all()) and bool(out[2].isnan().all()) and bool(lse[2].isnan().all())
    assert bool(out[3, 0, 6].isnan()) and bool(out[3, 0, :6].isfinite().all()) and bool(out[3, 0, 7:].isfinite().all())


def test_without_lse_on_another_stream_with_fewer_sequences_and_the_same_bits_twice():
    lengths = [5000, 300, 0]
    c, table, q = filled(13, lengths, 4, 2, 128, "bf16", None, 64)
    out, lse = check_decode(c, table, q, lengths, "first")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    again = torch.full_like(out, 1.0)
    c.decode(q, ints(table), ints(lengths), again, stream=s)
    s.synchronize()
    assert torch.equal(again, out)
    few = torch.full_like(out, 1.0)
    c.decode(q[:2], ints(table)[:2], ints(lengths)[:2], few[:2])
    assert bool((few[2] == 1.0).all())
    # fewer sequences, other shares of the blocks: another order of the same sums
    want, _, tol, _ = attention(c, q[:2], table, lengths[:2])
    assert_within(few[:2], want, tol)


def test_two_captured_graphs_share_a_cache():
    """Two steps captured apart, replayed in turn with eager calls in between; the lengths change between replays."""
    lengths = [3000, 100, 1500]
    c, table, q = filled(14, lengths, 2, 4, 128, "bf16", "e4m3", 64)
    t, q2 = ints(table), randn(gen(15), 3, 8, 128, dtype="bf16")
    n = ints(lengths)
    outs = [torch.zeros(3, 8, 128, device="cuda") for _ in range(3)]
    graphs = []
    for x, out in ((q, outs[0]), (q2, outs[1])):
        c.decode(x, t, n, out)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.decode(x, t, n, out)
        graphs.append(g)
    for step, now in enumerate(([3000, 100, 1500], [1, 0, 1499], [2999, 64, 0], [3000, 100, 1500])):
        n.copy_(ints(now))
        for i, x in enumerate((q, q2)):
            outs[i].fill_(3.0)
            graphs[i].replay()
            c.decode(x, t, n, outs[2])
            torch.cuda.synchronize()
            assert torch.equal(outs[i], outs[2]), (step, i)
    want, _, tol, _ = attention(c, q, table, lengths)
    assert_within(outs[0], want, tol)


def test_offsets_beyond_32_bits():
    """A pool of more than 4 GiB in which the sequence's pages are the last ones."""
    R, D, H = 256, 256, 8
    n_pages = (5 << 30) // (R * D * H * 2)
    c = PagedCache(PagedConfig(1, H, H, D, "bf16", R, n_pages, 3))
    g = gen(16)
    k, v = randn(g, 1, H, 700, D, dtype="bf16"), randn(g, 1, H, 700, D, dtype="bf16")
    table = [[n_pages - 1, 0, n_pages - 2]]
    c.append(k, v, ints(table))
    k_back, v_back = torch.empty_like(k), torch.empty_like(v)
    c.read(ints(table), None, None, k_back, v_back)
    assert torch.equal(k, k_back) and torch.equal(v, v_back)
    assert torch.equal(c.k_pages[n_pages - 2, :, :188], k[0, :, 512:])
    q = randn(g, 1, H, D, dtype="bf16")
    out = torch.empty(1, H, D, device="cuda")
    c.decode(q, ints(table), ints([700]), out)
    p = torch.softmax(torch.matmul(k[0].double(), q[0].double()[..., None])[..., 0] / 16, -1)
    want = (p[..., None] * v[0].double()).sum(1)
    assert_within(out[0], want, (2 * 264 * U * 64 + 2.0 ** -22 + 108 * U) * (p[..., None] * v[0].double().abs()).sum(1))


# ------------------------------------------------------------------------------------------------ all of them together
@pytest.mark.parametrize("dtype,page_dtype", [("bf16", None), ("fp16", "e4m3"), ("fp32", None)])
def test_prompts_steps_and_the_move_into_a_bounded_cache(dtype, page_dtype):
    """As a server uses them: prompts of unequal length in two chunks, decode steps, then one sequence's rows leave the pages for a
    bounded cache that keeps them all, whose own step must give what the paged one gives."""
    g, B, H, G, D, R, steps = gen(20), 3, 2, 4, 128, 32, 9
    prompts = [75, 1, 140]
    cols = (max(prompts) + steps + R - 1) // R
    lengths = [p + steps for p in prompts]
    table = tables(21, lengths, R, 3 * cols, cols)
    c = pool(B, H, G, D, dtype, page_dtype, R, 3 * cols, cols)
    r = Rotary(randn(g, D, dtype=dtype), randn(g, D, dtype=dtype), 10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64, device="cuda") / D))
    t, seen = ints(table), [0] * B
    for chunk in (64, 100):
        n = [min(chunk, p - s) for p, s in zip(prompts, seen)]
        k, v = randn(g, B, H, chunk, D, dtype=dtype), randn(g, B, H, chunk, D, dtype=dtype)
        c.append(k, v, t, ints(seen), ints(n), rotary=r)
        seen = [s + x for s, x in zip(seen, n)]
    assert seen == prompts
    q_in, q_now, out = randn(g, steps, B, H * G, 1, D, dtype=dtype), torch.empty(B, H * G, 1, D, dtype=DT[dtype], device="cuda"), torch.empty(B, H * G, D, device="cuda")
    start, length = ints(seen), ints([s + 1 for s in seen])
    for step in range(steps):
        k, v = randn(g, B, H, 1, D, dtype=dtype), randn(g, B, H, 1, D, dtype=dtype)
        c.append(k, v, t, start, q=q_in[step], q_out=q_now, rotary=r)
        c.decode(q_now[:, :, 0], t, length, out)
        start += 1
        length += 1
        seen = [s + 1 for s in seen]
        want, _, tol, _ = attention(c, q_now[:, :, 0], table, seen)
        assert_within(out, want, tol, f"step {step}")
    # sequence 2 into a bounded cache with room for all of it; the last token goes in by a decode step
    N = seen[2]
    k_rows, v_rows_ = (torch.empty(1, H, N, D, dtype=DT[dtype], device="cuda") for _ in range(2))
    c.read(t[2:], None, None, k_rows, v_rows_)
    b = BuzzCache(BuzzConfig(1, H * G, H, D, dtype, 4, 200, 16, 2, 16, N + 8))
    b.prefill(k_rows[:, :, :N - 1].contiguous(), v_rows_[:, :, :N - 1].contiguous())
    bounded = torch.empty(1, H * G, D, device="cuda")
    b.decode_step(q_now[2:, :, 0].contiguous(), k_rows[:, :, N - 1].contiguous(), v_rows_[:, :, N - 1].contiguous(), bounded)
    if page_dtype is None or dtype == "bf16":
        assert_within(bounded[0], out[2], 2 * tol[2], "bounded cache")
    else:                                                                      # rows come back rounded to fp16 where e4m3 reaches below it
        assert float((bounded[0] - out[2]).abs().max()) <= 2.0 ** -10 * float(out[2].abs().max())
    b.close()
    c.close()


def test_refusals_leave_the_outputs_alone():
    c, table, q = filled(22, [40, 40], 1, 2, 64, "bf16", None, 16)
    out = torch.full((2, 2, 64), 2.0, device="cuda")
    with pytest.raises(BuzzError):
        c.decode(q, ints(table), ints([40]), out)
    with pytest.raises(BuzzError):
        c.decode(q.float(), ints(table), ints([40, 40]), out)
    with pytest.raises(BuzzError) as e:
        c.decode(torch.zeros(2 * 2 * 64 + 8, dtype=torch.bfloat16, device="cuda")[1:257].view(2, 2, 64), ints(table), ints([40, 40]), out)
    assert e.value.code == -5                                                  # rows on 2-byte boundaries
    torch.cuda.synchronize()
    assert bool((out == 2.0).all())

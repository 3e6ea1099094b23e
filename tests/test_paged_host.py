"""Host-side checks of the paged cache and of the position rotation that need no GPU: what is refused, in which order,
and the arithmetic by which the kernels place their work (pages, tiles, shares of blocks) compiled for the host."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

from paper_2410_23079_amd import (FLAG_DRY_RUN, BuzzError, PagedCache, PagedConfig, Rotary, load_library,
                                  paged_workspace_bytes, qk_norm_rotate)
from paper_2410_23079_amd.binding import _Pages, _pack_rows, _Rotary

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HERE = os.path.join(ROOT, "tests")


def cfg(**kw):
    base = dict(batch=3, n_q_heads=8, n_kv_heads=2, head_dim=128, dtype="bf16", page_rows=32, n_pages=40, table_cols=12)
    base.update(kw)
    return PagedConfig(**base)


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc not on PATH")
def test_the_arithmetic_that_places_the_work(tmp_path):
    exe = str(tmp_path / "paged_schedule")
    subprocess.run(["hipcc", "-x", "hip", "--cuda-host-only", "-std=c++17", "-O1", "-Xarch_host", "-fsanitize=undefined",
                    "-Xarch_host", "-fno-sanitize-recover=undefined", "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2410_23079_amd", "csrc"), os.path.join(HERE, "paged_schedule.cpp"), "-o", exe],
                   check=True, capture_output=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "paged_schedule ok" in r.stdout, r.stderr


@pytest.mark.parametrize("bad,code", [
    (dict(batch=0), -1), (dict(n_q_heads=7), -1), (dict(n_kv_heads=0), -1), (dict(n_pages=0), -1), (dict(table_cols=0), -1),
    (dict(page_rows=0), -1), (dict(sink=-1), -1), (dict(window=-1), -1), (dict(flags=1), -1), (dict(softmax_scale=float("nan")), -1),
    (dict(softmax_scale=-1.0), -1), (dict(softmax_scale=float("inf")), -1), (dict(page_dtype="fp16"), -1),
    (dict(head_dim=96), -5), (dict(n_q_heads=18), -5), (dict(dtype="fp32", page_dtype="e4m3"), -5), (dict(page_rows=24), -5),
    (dict(page_rows=8), -5), (dict(page_rows=512), -5), (dict(table_cols=(1 << 28) // 32 + 1), -5), (dict(batch=65536), -5),
])
def test_configurations_that_are_refused(bad, code):
    with pytest.raises(BuzzError) as e:
        paged_workspace_bytes(cfg(**bad))
    assert e.value.code == code


def test_the_workspace_holds_what_the_largest_step_leaves():
    c = cfg(n_q_heads=64, n_kv_heads=8, head_dim=256, batch=100)
    # two partial results (max, sum, output) of 8 heads and their counters for each of 512 blocks, one counter for each pair
    assert paged_workspace_bytes(c) >= 2 * 512 * 8 * (256 + 2) * 4 + 100 * 8 * 4 + 2 * 512 * 4


def rows(ptr=0x1000, seq=4096, head=1024, row=128):
    return _pack_rows(ptr or 0, seq, head, row)


def dry(**kw):
    return PagedCache(cfg(flags=FLAG_DRY_RUN, **kw))


def test_creation_is_refused_before_anything_is_touched():
    lib, h, p = load_library(), ctypes.c_void_p(), _Pages(0x1000, 0x2000, None, None)
    create = lambda c, pages, ws, n: lib.buzz_paged_create(c.to_c(), pages, ws, n, None, ctypes.byref(h))
    big = 1 << 40
    assert create(cfg(), None, 0x1000, big) == -1
    assert create(cfg(), _Pages(None, 0x2000, None, None), 0x1000, big) == -1
    assert create(cfg(), _Pages(0x1008, 0x2000, None, None), 0x1000, big) == -1                # misaligned
    assert create(cfg(), p, None, big) == -1 and create(cfg(), p, 0x1010, big) == -1
    assert create(cfg(), _Pages(0x1000, 0x2000, 0x3000, 0x4000), 0x1000, big) == -1            # exponents of 16-bit pages
    assert create(cfg(page_dtype="e4m3"), p, 0x1000, big) == -1                                # 8-bit pages without them
    assert create(cfg(), p, 0x1000, 4096) == -2
    assert h.value is None
    assert lib.buzz_paged_destroy(None) == 0
    assert lib.buzz_paged_workspace_bytes(None, None) == -1


def test_calls_that_are_refused():
    lib = load_library()
    c = dry()
    h, r = c._h, rows()
    ref = lambda s: None if s is None else ctypes.byref(s)
    append = lambda n=4, batch=3, rot=None, q=None, q_out=None: lib.buzz_paged_append(h, ref(rot), q, r, r, q_out, batch, n, 0x1000, None, None, None)
    assert append() == 0 and append(n=0) == 0 and append(batch=0) == 0
    assert append(n=-1) == -1 and append(batch=-1) == -1
    assert append(batch=4) == -2 and append(n=12 * 32 + 1) == -2                               # capacity
    assert append(q=r) == -1 and append(q_out=r) == -1                                         # half a pair
    assert append(rot=_Rotary(None, None, None, 1e-6, 64, 0, 0)) == -1                         # no frequencies
    assert append(rot=_Rotary(None, None, 0x1000, 1e-6, 130, 0, 0)) == -1
    assert append(rot=_Rotary(None, None, 0x1000, 1e-6, -16, 0, 0)) == -1
    assert append(rot=_Rotary(None, None, 0x1000, 1e-6, 24, 0, 0)) == -5
    assert append(rot=_Rotary(None, None, 0x1000, 1e-6, 64, 2, 0)) == -1
    assert append(rot=_Rotary(None, None, 0x1000, 1e-6, 64, 0, 1)) == -1
    assert append(rot=_Rotary(0x1000, None, None, -1.0, 0, 0, 0)) == -1
    assert append(rot=_Rotary(0x1000, None, None, float("nan"), 0, 0, 0)) == -1
    assert append(rot=_Rotary(0x1008, None, None, 1e-6, 0, 0, 0)) == -5
    assert append(rot=_Rotary(0x1000, 0x1000, 0x1008, 1e-6, 128, 1, 0)) == 0
    read = lambda n=4, batch=3: lib.buzz_paged_read(h, r, r, batch, n, 0x1000, None, None, None)
    assert read() == 0 and read(n=-1) == -1 and read(batch=4) == -2 and read(n=12 * 32 + 1) == -2
    decode = lambda batch=3: lib.buzz_paged_decode(h, r, batch, 0x1000, 0x1000, 0x1000, None, None)
    assert decode() == 0 and decode(-1) == -1 and decode(4) == -2
    for call in (lib.buzz_paged_append(None, None, None, r, r, None, 1, 1, 0x1000, None, None, None),
                 lib.buzz_paged_read(None, r, r, 1, 1, 0x1000, None, None, None),
                 lib.buzz_paged_decode(None, r, 1, 0x1000, 0x1000, 0x1000, None, None)):
        assert call == -1
    c.close()


def test_rows_that_are_refused():
    """Everything is looked at before a launch: these calls return without one, though the pointers are made up."""
    lib, rot = load_library(), _Rotary(None, None, 0x1000, 1e-6, 64, 0, 0)

    def call(q=None, k=None, q_out=None, k_out=None, dtype=2, D=128, Hq=8, Hkv=2, rotary=rot, batch=2, n=4):
        return lib.buzz_qk_norm_rotate(dtype, D, Hq, Hkv, None if rotary is None else ctypes.byref(rotary), q, k, q_out, k_out, batch, n, None, None, None)
    r = rows()
    assert call() == 0 and call(r, r, r, r, batch=0) == 0 and call(r, r, r, r, n=0) == 0       # nothing to do
    assert call(r) == -1 and call(k=r) == -1 and call(q_out=r) == -1
    assert call(r, None, r, rotary=None) == -1
    assert call(r, None, r, dtype=3) == -1 and call(r, None, r, D=96) == -5 and call(r, None, r, Hq=0) == -1
    assert call(r, None, r, batch=-1) == -1 and call(r, None, r, n=-1) == -1
    assert call(r, None, r, batch=65536) == -5 and call(r, None, r, n=(1 << 27) + 1) == -5
    assert call(rows(ptr=None), None, r) == -1
    for crooked in (rows(ptr=0x1008), rows(seq=4100), rows(head=1028), rows(row=132)):
        assert call(crooked, None, r) == -5 and call(r, None, crooked) == -5
        assert call(None, crooked, None, r) == -5


def test_the_binding_looks_at_tensors_before_their_addresses_are_used():
    t = torch.zeros
    k = t(3, 2, 4, 128, dtype=torch.bfloat16)
    table = t(3, 12, dtype=torch.int32)
    c = dry()
    c.append(k, k, table)
    c.append(k.transpose(1, 2).contiguous().transpose(1, 2), k, table, t(3, dtype=torch.int32))
    c.read(table, None, None, k, None)
    q, out = t(3, 8, 128, dtype=torch.bfloat16), t(3, 8, 128)
    c.decode(q, table, t(3, dtype=torch.int32), out)
    bad = [lambda: c.append(k.float(), k, table), lambda: c.append(k, k[:, :1], table), lambda: c.append(k, k, table.long()),
           lambda: c.append(k, k, table[:, :11]), lambda: c.append(k, k, table[:2]), lambda: c.append(k, k, table, t(3)),
           lambda: c.append(k, k, table, None, t(2, dtype=torch.int32)), lambda: c.append(k, k, table, q=k),
           lambda: c.append(k[..., ::2], k, table), lambda: c.append(k, k, table, rotary=Rotary(t(128))),
           lambda: c.append(k, k, table, rotary=Rotary(t(64, dtype=torch.bfloat16))),
           lambda: c.read(table, None, None, None, None), lambda: c.read(table, None, None, k, k[:, :, :3]),
           lambda: c.decode(q, table, t(3, dtype=torch.int32), out.double()), lambda: c.decode(q[:, :4], table, t(3, dtype=torch.int32), out),
           lambda: c.decode(q, table, t(3, dtype=torch.int32), out, t(3, 4)), lambda: c.decode(q, table, t(4, dtype=torch.int32), out),
           lambda: c.decode(q, table, t(3, dtype=torch.int32), out.transpose(0, 1).contiguous().transpose(0, 1)),
           lambda: Rotary(inv_freq=t(32)), lambda: Rotary(q_weight=t(128, dtype=torch.float64)), lambda: Rotary(t(2, 64)),
           lambda: qk_norm_rotate(None, None, None, None, Rotary()),
           lambda: qk_norm_rotate(k, None, k, None, Rotary()),                                 # not on the GPU
           lambda: PagedCache(cfg(), device="cpu"),
           lambda: PagedCache(cfg(), pages=(t(40, 2, 32, 128, dtype=torch.bfloat16), t(40, 2, 4, 128, 8, dtype=torch.bfloat16), None, None))]
    for i, call in enumerate(bad):
        with pytest.raises(BuzzError) as e:
            call()
        assert e.value.code == -1, i

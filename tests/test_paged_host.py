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


# ------------------------------------------------------------------------------------------------ what is enqueued
@pytest.fixture(scope="module")
def recorded(tmp_path_factory):
    """The library's objects linked against a recorder that takes kernel launches in place of the HIP runtime."""
    if shutil.which("hipcc") is None:
        pytest.skip("hipcc not on PATH")
    from paper_2410_23079_amd.build import CSRC, SOURCES, build
    objs = [os.path.join(CSRC, stem + ".o") for _, stem, _ in SOURCES]
    if not all(os.path.exists(o) for o in objs):
        build()
    tmp = tmp_path_factory.mktemp("recorder")
    rec, so = str(tmp / "launch_recorder.o"), str(tmp / "libbuzz_recorded.so")
    subprocess.run(["hipcc", "-x", "hip", "--cuda-host-only", "-std=c++17", "-O1", "-fPIC", "-I", os.path.join(ROOT, "include"),
                    "-I", CSRC, "-c", os.path.join(HERE, "launch_recorder.cpp"), "-o", rec], check=True, capture_output=True)
    subprocess.run(["g++", "-shared", "-Wl,-Bsymbolic", "-Wl,--no-undefined", "-o", so, rec, *objs], check=True, capture_output=True)
    lib, real = ctypes.CDLL(so), load_library()
    for name in ("buzz_qk_norm_rotate", "buzz_paged_create", "buzz_paged_destroy", "buzz_paged_append", "buzz_paged_read", "buzz_paged_decode"):
        getattr(lib, name).argtypes = getattr(real, name).argtypes
    lib.rec_kernel.restype = ctypes.c_char_p
    lib.rec_value.restype = ctypes.c_longlong
    lib.rec_value.argtypes = [ctypes.c_int, ctypes.c_char_p]
    return lib


def made(lib, **kw):
    c, h = cfg(**kw), ctypes.c_void_p()
    exps = (0x300000, 0x400000) if c.page_dtype else (None, None)
    lib.rec_reset(-1)
    assert lib.buzz_paged_create(c.to_c(), _Pages(0x100000, 0x200000, *exps), 0x500000, 1 << 40, None, ctypes.byref(h)) == 0
    assert lib.rec_count() == 1 and b"clear" in lib.rec_kernel(0)          # the counters, by a kernel
    lib.rec_reset(-1)
    return h


def test_every_call_is_one_launch_and_a_launch_that_fails_is_told(recorded):
    lib, r, rot = recorded, rows(), _Rotary(None, None, 0x1000, 1e-6, 64, 0, 0)
    h = made(lib)
    calls = [lambda: lib.buzz_paged_append(h, ctypes.byref(rot), r, r, r, r, 3, 40, 0x1000, 0x1000, None, None),
             lambda: lib.buzz_paged_read(h, r, r, 3, 40, 0x1000, None, None, None),
             lambda: lib.buzz_paged_decode(h, r, 3, 0x1000, 0x1000, 0x1000, None, None),
             lambda: lib.buzz_qk_norm_rotate(2, 128, 8, 2, ctypes.byref(rot), r, r, r, r, 3, 40, None, None, None)]
    for call in calls:
        lib.rec_reset(-1)
        assert call() == 0 and lib.rec_count() == 1
        lib.rec_reset(0)
        assert call() == -4
    lib.rec_reset(-1)
    assert lib.buzz_paged_append(h, None, None, r, r, None, 0, 40, 0x1000, None, None, None) == 0
    assert lib.buzz_paged_append(h, None, None, r, r, None, 3, 0, 0x1000, None, None, None) == 0
    assert lib.buzz_paged_read(h, None, None, 3, 40, 0x1000, None, None, None) == 0
    assert lib.buzz_paged_decode(h, r, 0, 0x1000, 0x1000, 0x1000, None, None) == 0
    assert lib.rec_count() == 0                                            # nothing to do
    assert lib.buzz_paged_append(h, None, None, r, None, None, 3, 40, 0x1000, None, None, None) == -1
    assert lib.buzz_paged_append(h, None, None, r, r, None, 3, 40, None, None, None, None) == -1
    assert lib.buzz_paged_decode(h, rows(ptr=0x1008), 3, 0x1000, 0x1000, 0x1000, None, None) == -5
    assert lib.buzz_paged_decode(h, r, 3, 0x1000, 0x1000, 0x1004, None, None) == -5
    assert lib.buzz_paged_decode(h, r, 3, 0x1000, None, 0x1000, None, None) == -1
    assert lib.rec_count() == 0
    assert lib.buzz_paged_destroy(h) == 0
    c, x = cfg(), ctypes.c_void_p()
    lib.rec_reset(0)
    assert lib.buzz_paged_create(c.to_c(), _Pages(0x1000, 0x2000, None, None), 0x1000, 1 << 40, None, ctypes.byref(x)) == -4
    assert x.value is None
    lib.rec_reset(-1)


@pytest.mark.parametrize("kw,batch,most", [
    (dict(batch=1, n_q_heads=1, n_kv_heads=1, table_cols=1), 1, 1), (dict(table_cols=64), 3, 2 * 3 * 64 // 4),
    (dict(batch=64, table_cols=4096), 64, 512), (dict(batch=4, page_dtype="e4m3", table_cols=64), 4, 512),
    (dict(dtype="fp32", table_cols=2), 3, 6)])
def test_the_decode_grid_has_no_more_blocks_than_there_can_be_work(recorded, kw, batch, most):
    h = made(recorded, **kw)
    assert recorded.buzz_paged_decode(h, rows(), batch, 0x1000, 0x1000, 0x1000, None, None) == 0
    assert 1 <= recorded.rec_value(0, b"grid_x") <= most and recorded.rec_value(0, b"grid_y") == recorded.rec_value(0, b"grid_z") == 1
    assert recorded.rec_value(0, b"block_x") == 512
    recorded.buzz_paged_destroy(h)


@pytest.mark.parametrize("n,batch,D,dtype", [(1, 3, 128, "bf16"), (17, 2, 64, "fp32"), (300, 1, 256, "fp16"), (20000, 3, 128, "bf16"), (2, 1, 128, "fp32")])
def test_the_row_grids_cover_every_tile_of_every_sequence(recorded, n, batch, D, dtype):
    """16 positions to a tile, wherever the first row stands; as many blocks per tile as jobs."""
    h, r, rot = made(recorded, head_dim=D, dtype=dtype, table_cols=1000, page_rows=32), rows(), _Rotary(None, None, 0x1000, 1e-6, 64, 0, 0)
    assert recorded.buzz_paged_append(h, ctypes.byref(rot), r, r, r, r, batch, n, 0x1000, 0x1000, None, None) == 0
    assert recorded.buzz_paged_read(h, r, r, batch, n, 0x1000, 0x1000, None, None) == 0
    assert recorded.buzz_paged_read(h, r, None, batch, n, 0x1000, 0x1000, None, None) == 0
    for i, least in ((0, 3), (1, 2), (2, 1)):                              # q, k and v; k and v; k: a job each at least
        assert recorded.rec_value(i, b"grid_x") == (n + 14) // 16 + 1 and recorded.rec_value(i, b"grid_z") == batch
        assert least <= recorded.rec_value(i, b"grid_y") <= 8 + 2 + 2
    recorded.buzz_paged_destroy(h)

"""The operators of 4-bit paged caches without a GPU: refusals on the host, and the addresses and shares of csrc/lpq_paged_index.h that only they use, compiled for the host:
groups of cells stay in the pool, and the shares are the same numbers with 32-bit and with 64-bit divisions."""
import ctypes
import os
import subprocess

import pytest

import paper_2403_01136_amd as lpq

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000          # never dereferenced: every call below must fail validation first
NULL, SHAPE, ALIGN, UNSUPPORTED = 1, 4, 5, 8

HARNESS = r'''
#include "lpq_paged_index.h"
using namespace lpq;
extern "C" {
int t_group_bytes(int d) { return cell_group_bytes(d); }
int64_t t_group(int page, int h, int kv, int shift, int g, int d) { return cell_group(page, h, kv, shift, g, d); }
int t_small(int64_t u, int W) { return stream_small(u, W); }
int64_t t_begin(int64_t u, int w, int W) { return stream_begin(u, w, W); }
int t_worker(int64_t units, int64_t u, int W) { return stream_worker(units, u, W); }
}
'''


@pytest.fixture(scope="module")
def idx(tmp_path_factory):
    d = tmp_path_factory.mktemp("cells_index")
    src, so = str(d / "h.cpp"), str(d / "h.so")
    open(src, "w").write(HARNESS)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-shared", "-fPIC",
                           "-I" + os.path.join(ROOT, "paper_2403_01136_amd", "csrc"), src, "-o", so])
    L = ctypes.CDLL(so)
    L.t_group.restype = L.t_begin.restype = ctypes.c_int64
    L.t_small.argtypes, L.t_begin.argtypes = [ctypes.c_int64, ctypes.c_int], [ctypes.c_int64, ctypes.c_int, ctypes.c_int]
    L.t_worker.argtypes = [ctypes.c_int64, ctypes.c_int64, ctypes.c_int]
    return L


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("shift", [4, 5, 6, 7, 8])
def test_groups_of_cells_stay_in_the_pool(idx, d, shift):
    assert idx.t_group_bytes(d) == 16 * (d // 2 + 4)
    for kv, pages in ((1, 3), (3, 2), (8, 5)):
        seen = sorted(idx.t_group(p, h, kv, shift, g, d) for p in range(pages) for h in range(kv) for g in range(1 << (shift - 4)))
        assert seen == [i * idx.t_group_bytes(d) for i in range(len(seen))]
        assert len(seen) * idx.t_group_bytes(d) == pages * kv * lpq.lpq_cell_page_bytes(1 << shift, d)
    assert idx.t_group(2**31 // (1 << shift) - 1, 127, 128, shift, (1 << (shift - 4)) - 1, d) == (2**31 // (1 << shift) * 128 * (1 << (shift - 4)) - 1) * idx.t_group_bytes(d)


def test_shares_on_both_sides_of_32_bits(idx):
    """The product of units and workers decides which division is taken; the numbers are floor(units * w / W) and the worker that has a unit either way."""
    for W in (1, 3, 1024, 2048):
        edge = (2**32 - 1) // W
        for units in (1, W, 1000003, edge - 1, edge, edge + 1, edge + 12345, 2**32 - 1, 2**32, 2**40 + 7):
            assert bool(idx.t_small(units, W)) == (units < 2**32 and units * W < 2**32)
            for w in {0, 1, W // 3, W - 1, W}:
                assert idx.t_begin(units, w, W) == units * w // W
            if units < W:
                continue
            for w in {0, 1 % W, W // 2, W - 1}:
                for u in {units * w // W, max(units * w // W, units * (w + 1) // W - 1)}:
                    assert idx.t_worker(units, u, W) == w


def cfg(heads=8, kv=2, d=64, dtype=0):
    return ctypes.byref(lpq.lpq_attn_cfg(heads, kv, d, dtype))


def pool(page=16, n=10, width=4, table=FAKE, ring=FAKE, counters=FAKE):
    return ctypes.byref(lpq.lpq_page_pool(page, n, width, table, ring, counters))


def turn(dim=64, pairs=0, max_pos=10, eps=1e-6, table=FAKE, q=None, k=None):
    return ctypes.byref(lpq.lpq_rotary(dim, pairs, max_pos, eps, table, q, k))


BAD_CFGS = [(cfg(heads=0), SHAPE), (cfg(kv=0), SHAPE), (cfg(heads=8, kv=3), SHAPE), (cfg(d=96), SHAPE), (cfg(dtype=2), UNSUPPORTED), (cfg(dtype=-1), UNSUPPORTED)]
BAD_POOLS = [pool(page=8), pool(page=48), pool(page=512), pool(page=0), pool(n=0), pool(n=-1), pool(page=256, n=1 << 23)]


def test_page_bytes():
    for d in (64, 128):
        for page in (16, 32, 64, 128, 256):
            assert lpq.lpq_cell_page_bytes(page, d) == page * (d // 2 + 4)
    for page, d in ((8, 64), (48, 64), (512, 64), (0, 64), (-16, 64), (16, 96), (16, 0), (16, -64), (16, 256)):
        assert lpq.load_library().lpq_cell_page_bytes(page, d) == 0
        with pytest.raises(ValueError):
            lpq.lpq_cell_page_bytes(page, d)


def test_rotary_refusals():
    L = lpq.load_library()
    OUT = FAKE + (1 << 30)
    call = lambda x=FAKE, c=cfg(), r=turn(), p=FAKE, s=None, M=1, o=OUT: L.lpq_qk_norm_rotary(x, c, r, p, s, M, o, None)
    assert call(x=None) == call(c=None) == call(r=None) == call(p=None) == call(o=None) == call(r=turn(table=None)) == NULL
    for c, status in BAD_CFGS:
        assert call(c=c) == status
    for r in (turn(dim=-16), turn(dim=8), turn(dim=24), turn(dim=80), turn(max_pos=0), turn(max_pos=-1), turn(q=FAKE, eps=0.0), turn(k=FAKE, eps=-1.0), turn(q=FAKE, eps=float("nan"))):
        assert call(r=r) == SHAPE
    assert call(r=turn(pairs=2)) == call(r=turn(pairs=-1)) == UNSUPPORTED
    assert call(M=0) == call(M=-1) == call(M=(1 << 24) + 1) == SHAPE                 # 8 heads: M * heads is at most 2^27
    assert call(x=FAKE + 2) == call(o=OUT + 8) == call(p=FAKE + 2) == call(s=FAKE + 1) == ALIGN
    assert call(r=turn(table=FAKE + 8)) == call(r=turn(q=FAKE + 8)) == call(r=turn(k=FAKE + 4)) == ALIGN
    row = 12 * 64 * 2
    for M, off in ((1, 16), (1, row - 16), (4, row), (4, 4 * row - 16)):             # another buffer that overlaps the rows, from either side
        assert call(M=M, o=FAKE + off) == call(M=M, x=FAKE + off, o=FAKE) == SHAPE


def test_append_and_load_refusals():
    L = lpq.load_library()
    append = lambda x=FAKE, c=cfg(), p=pool(), k=FAKE, v=FAKE, s=FAKE, M=1: L.lpq_paged_append4(x, c, p, k, v, s, M, None)
    load = lambda x=FAKE, c=cfg(), p=pool(), k=FAKE, v=FAKE, s=FAKE, M=1: L.lpq_paged_load4(k, v, c, p, s, M, x, None)
    for call in (append, load):
        assert call(x=None) == call(c=None) == call(p=None) == call(k=None) == call(v=None) == call(s=None) == NULL
        for c, status in BAD_CFGS:
            assert call(c=c) == status
        for p in BAD_POOLS:
            assert call(p=p) == SHAPE
        assert call(M=0) == call(M=(1 << 24) + 1) == SHAPE
        assert call(x=FAKE + 8) == call(k=FAKE + 2) == call(v=FAKE + 4) == call(s=FAKE + 2) == ALIGN


def test_attention_refusals():
    L = lpq.load_library()
    call = lambda x=FAKE, c=cfg(), p=pool(), k=FAKE, v=FAKE, a=None, cu=FAKE, kv=FAKE, n=1, M=1, mq=1, mk=1, o=FAKE: L.lpq_paged_attention4(
        x, c, p, k, v, a, cu, kv, n, M, mq, mk, o, None)
    assert call(x=None) == call(c=None) == call(cu=None) == call(o=None) == call(p=None) == call(k=None) == call(v=None) == call(kv=None) == call(p=pool(table=None)) == NULL
    for c, status in BAD_CFGS:
        assert call(c=c) == status
    for p in BAD_POOLS + [pool(width=0), pool(page=256, width=(1 << 22) + 1)]:
        assert call(p=p) == SHAPE
    assert call(M=0) == call(n=0) == call(n=2049) == call(mq=0) == call(M=1 << 26) == call(mk=0) == SHAPE
    assert call(x=FAKE + 2) == call(o=FAKE + 8) == call(a=FAKE + 2) == call(cu=FAKE + 1) == call(k=FAKE + 8) == call(v=FAKE + 8) == call(kv=FAKE + 2) == call(p=pool(table=FAKE + 2)) == ALIGN
    many = cfg(heads=8192, kv=8192)                                   # M * heads is 2^24 and allowed; 2048 sequences of 8192 K/V heads are not
    assert call(c=many, n=2048, M=2048) == SHAPE


def test_binding_refuses_host_tensors():
    import torch
    x, i = torch.zeros((1, 256), dtype=torch.float16), torch.zeros(2, dtype=torch.int32)
    pages = torch.zeros((1, 1, lpq.lpq_cell_page_bytes(16, 64)), dtype=torch.uint8)
    with pytest.raises(ValueError):
        lpq.lpq_qk_norm_rotary(x, i[:1], 2, 1, cos_sin=torch.zeros((4, 64)))
    with pytest.raises(ValueError):
        lpq.lpq_paged_append4(x, pages, pages, i[:1])
    with pytest.raises(ValueError):
        lpq.lpq_paged_load4(pages, pages, i[:1], x)
    with pytest.raises(ValueError):
        lpq.lpq_paged_attention4(x, pages, pages, i.view(1, 2), i, i[:1])

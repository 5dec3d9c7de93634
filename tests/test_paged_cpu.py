"""The paged and packed operators without a GPU: refusals on the host, and the index arithmetic that every kernel address goes through
(csrc/lpq_paged_index.h), compiled for the host and checked by brute force: bad page ids, slots, offsets and lengths stay inside their buffers,
and every row tile, key tile and work unit is somebody's exactly once."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import paper_2403_01136_amd as lpq

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000          # never dereferenced: every call below must fail validation first
NULL, SHAPE, ALIGN, UNSUPPORTED = 1, 4, 5, 8

HARNESS = r'''
#include "lpq_paged_index.h"
using namespace lpq;
extern "C" {
void t_row_span(int c0, int c1, int M, int* out) { const RowSpan r = row_span(c0, c1, M); out[0] = r.first; out[1] = r.end; }
int t_page_entry(int g, int shift, int max_pages) { return page_entry(g, shift, max_pages); }
int t_page_checked(int id, int n) { return page_checked(id, n); }
int t_slot_checked(int s, int n, int shift) { return slot_checked(s, n, shift); }
int64_t t_page_element(int p, int h, int kv, int shift, int d) { return page_element(p, h, kv, shift, d); }
int t_keys_of(int kv, int mp, int shift) { return keys_of(kv, mp, shift); }
int t_token_position(int kv, int q, int t) { return token_position(kv, q, t); }
int t_tile_start(int f, int g, int s, int rows) { return tile_start(f, g, s, rows); }
int64_t t_tile_bound(int M, int g, int n, int rows) { return tile_bound(M, g, n, rows); }
void t_key_split(int tiles, int splits, int least, int sp, int* out) { const KeySplit k = key_split(tiles, splits, least, sp); out[0] = k.begin; out[1] = k.end; out[2] = k.used; }
int64_t t_stream_begin(int64_t u, int w, int W) { return stream_begin(u, w, W); }
int t_stream_worker(int64_t units, int64_t u, int W) { return stream_worker(units, u, W); }
int t_key_steps(int ctx) { return stream_key_steps(ctx); }
}
'''


@pytest.fixture(scope="module")
def idx(tmp_path_factory):
    d = tmp_path_factory.mktemp("paged_index")
    src, so = str(d / "h.cpp"), str(d / "h.so")
    open(src, "w").write(HARNESS)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-shared", "-fPIC",
                           "-I" + os.path.join(ROOT, "paper_2403_01136_amd", "csrc"), src, "-o", so])
    L = ctypes.CDLL(so)
    for f in ("t_page_element", "t_tile_bound", "t_stream_begin"):
        getattr(L, f).restype = ctypes.c_int64
    L.t_stream_begin.argtypes = [ctypes.c_int64, ctypes.c_int, ctypes.c_int]
    L.t_stream_worker.argtypes = [ctypes.c_int64, ctypes.c_int64, ctypes.c_int]
    return L


INTS = (-2**31, -7, -1, 0, 1, 15, 16, 17, 100, 2**20, 2**31 - 1)


def test_spans_stay_in_the_batch(idx):
    out = (ctypes.c_int * 2)()
    for M in (1, 16, 99):
        for a in INTS:
            for b in INTS:
                idx.t_row_span(a, b, M, out)
                assert 0 <= out[0] <= out[1] <= M
                if 0 <= a <= b <= M:
                    assert (out[0], out[1]) == (a, b)


def test_pages_and_slots_stay_in_the_pool(idx):
    for n in (1, 5, 1000):
        for v in INTS:
            assert idx.t_page_checked(v, n) == (v if 0 <= v < n else -1)
            for shift in (4, 6, 8):
                assert idx.t_slot_checked(v, n, shift) == (v if 0 <= v < n << shift else -1)
    for shift in (4, 5, 8):
        for g in range(40):
            e = g * 16 >> shift
            assert idx.t_page_entry(g, shift, 3) == (e if e < 3 else -1)
    # past 32 bits: the last page of a pool of 2^31 - 2^8 positions, 64 heads of 128
    assert idx.t_page_element(2**23 - 2, 63, 64, 8, 128) == (((2**23 - 2) * 64 + 63) << 8) * 128


def test_lengths(idx):
    for kv in INTS:
        for pages, shift in ((1, 4), (100, 6), (1 << 22, 8)):
            k = idx.t_keys_of(kv, pages, shift)
            assert k == min(max(kv, 0), pages << shift)
    assert [idx.t_token_position(10, 3, t) for t in range(3)] == [7, 8, 9]
    assert idx.t_token_position(2, 5, 0) == -3 and idx.t_token_position(-4, 5, 0) == -5
    assert [idx.t_key_steps(c) for c in (0, 1, 32, 33, 1 << 30)] == [1, 1, 1, 2, 1 << 25]


def test_every_row_tile_has_a_place(idx):
    r = np.random.default_rng(5)
    for _ in range(300):
        n, group = int(r.integers(1, 9)), int(r.choice([1, 2, 3, 7, 8, 16, 200]))
        lens = r.choice([0, 1, 2, 5, 16, 17, 127, 128, 129, 400], n)
        cu = np.concatenate([[0], np.cumsum(lens)])
        M = int(cu[-1] + r.integers(0, 5)) or 1
        for rows in (128, 256):
            starts = [idx.t_tile_start(int(c), group, s, rows) for s, c in enumerate(cu)]
            assert all(b > a for a, b in zip(starts, starts[1:]))        # the search for a tile's sequence goes by this
            for s in range(n):
                tiles = -(-int(lens[s]) * group // rows)
                assert tiles <= starts[s + 1] - starts[s] <= tiles + 1
            assert starts[-1] <= idx.t_tile_bound(M, group, n, rows)


def test_splits_cover_the_keys_once(idx):
    out = (ctypes.c_int * 3)()
    for tiles in list(range(1, 70)) + [1000, 16384]:
        for splits in (1, 2, 3, 7, 16):
            for least in (1, 4):
                nxt = 0
                for sp in range(splits):
                    idx.t_key_split(tiles, splits, least, sp, out)
                    b, e, used = out
                    assert 1 <= used <= splits
                    if sp < used:
                        assert b == nxt and e > b
                        nxt = e
                    else:
                        assert b == e == tiles
                assert nxt == tiles


def test_workers_share_the_units_evenly(idx):
    for units in (1, 2, 511, 512, 513, 6256, 2**33 + 7, 2**50):
        for W in sorted({1, min(units, 2), min(units, 512)}):
            begins = [idx.t_stream_begin(units, w, W) for w in range(W + 1)]
            assert begins[0] == 0 and begins[-1] == units
            sizes = [b - a for a, b in zip(begins, begins[1:])]
            assert min(sizes) >= 1 and max(sizes) - min(sizes) <= 1
            for w in {0, W // 2, W - 1}:
                for u in {begins[w], begins[w + 1] - 1}:
                    assert idx.t_stream_worker(units, u, W) == w


def cfg(heads=8, kv=2, d=64, dtype=0):
    return ctypes.byref(lpq.lpq_attn_cfg(heads, kv, d, dtype))


def pool(page=16, n=10, width=4, table=FAKE, ring=FAKE, counters=FAKE):
    return ctypes.byref(lpq.lpq_page_pool(page, n, width, table, ring, counters))


BAD_CFGS = [(cfg(heads=0), SHAPE), (cfg(kv=0), SHAPE), (cfg(heads=8, kv=3), SHAPE), (cfg(d=96), SHAPE), (cfg(dtype=2), UNSUPPORTED), (cfg(dtype=-1), UNSUPPORTED)]
BAD_POOLS = [pool(page=8), pool(page=48), pool(page=512), pool(page=0), pool(n=0), pool(n=-1), pool(page=256, n=1 << 23)]


def test_plan_refusals():
    L = lpq.load_library()
    out = lambda **k: ctypes.byref(lpq.lpq_page_plan(*[k.get(f, FAKE) for f in ("counters", "cu_q", "kv_lens", "slots", "positions", "info")]))
    call = lambda p=pool(), past=FAKE, q=FAKE, n=1, M=1, o=out(): L.lpq_paged_plan(p, past, q, n, M, o, None)
    assert call(p=None) == call(past=None) == call(q=None) == call(o=None) == NULL
    for f in ("counters", "cu_q", "kv_lens", "slots", "positions", "info"):
        assert call(o=out(**{f: None})) == NULL and call(o=out(**{f: FAKE + 2})) == ALIGN
    for k in ("table", "ring", "counters"):
        assert call(p=pool(**{k: None})) == NULL and call(p=pool(**{k: FAKE + 1})) == ALIGN
    for p in BAD_POOLS + [pool(width=0), pool(width=-3), pool(page=256, width=(1 << 22) + 1)]:
        assert call(p=p) == SHAPE
    for n, M in ((0, 1), (-1, 1), (2049, 1), (1, 0), (1, -5), (1, (1 << 27) + 1)):
        assert call(n=n, M=M) == SHAPE
    assert call(past=FAKE + 2) == call(q=FAKE + 3) == ALIGN


def test_append_refusals():
    L = lpq.load_library()
    call = lambda x=FAKE, c=cfg(), p=pool(), k=FAKE, v=FAKE, s=FAKE, M=1: L.lpq_paged_append(x, c, p, k, v, s, M, None)
    assert call(x=None) == call(c=None) == call(p=None) == call(k=None) == call(v=None) == call(s=None) == NULL
    for c, status in BAD_CFGS:
        assert call(c=c) == status
    for p in BAD_POOLS:
        assert call(p=p) == SHAPE
    assert call(M=0) == call(M=(1 << 24) + 1) == SHAPE                # 8 heads: M * heads is at most 2^27
    assert call(x=FAKE + 8) == call(k=FAKE + 2) == call(v=FAKE + 4) == call(s=FAKE + 2) == ALIGN


def test_attention_refusals():
    L = lpq.load_library()
    paged = lambda x=FAKE, c=cfg(), p=pool(), k=FAKE, v=FAKE, a=None, cu=FAKE, kv=FAKE, n=1, M=1, mq=1, mk=1, o=FAKE: L.lpq_paged_attention(
        x, c, p, k, v, a, cu, kv, n, M, mq, mk, o, None)
    packed = lambda x=FAKE, c=cfg(), a=None, cu=FAKE, n=1, M=1, mq=1, o=FAKE: L.lpq_packed_attention(x, c, a, cu, n, M, mq, o, None)
    for call in (paged, packed):
        assert call(x=None) == call(c=None) == call(cu=None) == call(o=None) == NULL
        for c, status in BAD_CFGS:
            assert call(c=c) == status
        assert call(M=0) == call(n=0) == call(n=2049) == call(mq=0) == call(M=1 << 26) == SHAPE
        assert call(x=FAKE + 2) == call(o=FAKE + 8) == call(a=FAKE + 2) == call(cu=FAKE + 1) == ALIGN
    assert paged(p=None) == paged(k=None) == paged(v=None) == paged(kv=None) == paged(p=pool(table=None)) == NULL
    for p in BAD_POOLS + [pool(width=0), pool(page=256, width=(1 << 22) + 1)]:
        assert paged(p=p) == SHAPE
    assert paged(mk=0) == SHAPE
    assert paged(k=FAKE + 8) == paged(v=FAKE + 8) == paged(kv=FAKE + 2) == paged(p=pool(table=FAKE + 2)) == ALIGN


def test_more_tiles_than_a_launch_has_threads_for_are_refused():
    L = lpq.load_library()
    many = cfg(heads=8192, kv=8192)                                   # M * heads is 2^24 and allowed; 2048 sequences of 8192 K/V heads are not
    assert L.lpq_paged_attention(FAKE, many, pool(), FAKE, FAKE, None, FAKE, FAKE, 2048, 2048, 1, 1, FAKE, None) == SHAPE
    assert L.lpq_packed_attention(FAKE, many, None, FAKE, 2048, 2048, 1, FAKE, None) == SHAPE


def test_binding_refuses_host_tensors():
    import torch
    x, pages, i = torch.zeros((1, 256), dtype=torch.float16), torch.zeros((1, 1, 16, 64), dtype=torch.float16), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        lpq.lpq_packed_attention(x, i, 2, 1)
    with pytest.raises(ValueError):
        lpq.lpq_paged_append(x, pages, pages, i[:1])
    with pytest.raises(ValueError):
        lpq.lpq_paged_attention(x, pages, pages, i.view(1, 2), i, i[:1])
    with pytest.raises(ValueError):
        lpq.lpq_paged_plan(i[:1], i[:1], i.view(1, 2), i, i, 16, 1)

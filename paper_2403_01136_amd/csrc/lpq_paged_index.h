// Index arithmetic of the paged and packed operators: which rows, pages, slots and work units a workgroup touches.  Plain functions for both
// sides, so that they can be checked without a GPU; every address that a kernel forms from a caller's integers goes through them.
#pragma once
#include <stdint.h>
#if defined(__HIPCC__)
#define LPQ_BOTH __host__ __device__ __forceinline__
#else
#define LPQ_BOTH inline
#endif

namespace lpq {

enum { PAGED_MAX_SEQS = 2048,            // sequences of a call: the plan keeps four numbers of each in LDS
       STREAM_ROWS = 16,                 // rows (tokens x query heads of a K/V head) of a column tile of the streaming kernel
       STREAM_KEYS = 32,                 // keys of its work unit: a step of one wave
       TILE_ROWS_Q = 128, TILE_KEYS = 64 };  // rows of a workgroup of the tile kernel; keys of a step

LPQ_BOTH int clamp_int(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }

// Rows [first, end) of sequence s, whatever the offsets say: within the M rows of the batch, end >= first.
struct RowSpan { int first, end; };
LPQ_BOTH RowSpan row_span(int cu0, int cu1, int M)
{
    RowSpan r;
    r.first = clamp_int(cu0, 0, M);
    r.end = clamp_int(cu1, r.first, M);
    return r;
}

// The page of group g of 16 positions: -1 if the sequence's row of the table has no entry for it.
LPQ_BOTH int page_entry(int g, int page_shift, int max_pages) { const int e = g >> (page_shift - 4); return e < max_pages ? e : -1; }
// A page id as a page of the pool: -1 if it is none.
LPQ_BOTH int page_checked(int id, int n_pages) { return (uint32_t)id < (uint32_t)n_pages ? id : -1; }
// Slots are page * page_size + offset; a slot outside the pool is none (-1).
LPQ_BOTH int slot_checked(int slot, int n_pages, int page_shift) { return slot >= 0 && (slot >> page_shift) < n_pages ? slot : -1; }
// First element of head h of a page (pages are [kv heads][page_size][d]).
LPQ_BOTH int64_t page_element(int page, int h, int kv_heads, int page_shift, int d) { return (((int64_t)page * kv_heads + h) << page_shift) * d; }

// Keys that exist for a sequence: [0, ctx).  kv_len may be anything.
LPQ_BOTH int keys_of(int kv_len, int max_pages, int page_shift)
{
    const int64_t cap = (int64_t)max_pages << page_shift;
    return kv_len < 0 ? 0 : kv_len > cap ? (int)cap : kv_len;
}
// The position of token t of q_len new ones; below zero where kv_len is less than q_len.
LPQ_BOTH int token_position(int kv_len, int q_len, int t) { return (kv_len < 0 ? 0 : kv_len) - q_len + t; }

// ---- the tile kernel's list: virtual tile v of tile_rows rows; sequence s starts at v = floor(first row * group / tile_rows) + s, which leaves every
// sequence room for its tiles (and at most one more, which has no rows), whatever the lengths, without a prefix sum.
LPQ_BOTH int tile_start(int first_row, int group, int s, int tile_rows) { return (int)((int64_t)first_row * group / tile_rows) + s; }
LPQ_BOTH int64_t tile_bound(int M, int group, int n_seqs, int tile_rows) { return (int64_t)M * group / tile_rows + n_seqs; }
// Key tiles [begin, end) of split `sp` out of `splits` for a row tile that sees `tiles` of them; used: splits that have any (at least one).
struct KeySplit { int begin, end, used; };
LPQ_BOTH KeySplit key_split(int tiles, int splits, int least, int sp)
{
    int per = (tiles + splits - 1) / splits;
    per = per < least ? least : per;
    KeySplit k;
    k.used = tiles > per ? (tiles + per - 1) / per : 1;
    const int64_t b = (int64_t)sp * per, e = b + per;
    k.begin = b < tiles ? (int)b : tiles;
    k.end = e < tiles ? (int)e : tiles;
    return k;
}

// ---- the streaming kernel's list: units of 32 keys, ordered sequence, K/V head, row tile, keys.  A sequence with rows but no keys has one unit per
// row tile (its rows are set to zero).
LPQ_BOTH int stream_row_tiles(int rows, int tile_rows) { return (rows + tile_rows - 1) / tile_rows; }
LPQ_BOTH int stream_key_steps(int ctx) { return ctx > STREAM_KEYS ? (ctx + STREAM_KEYS - 1) / STREAM_KEYS : 1; }
// Unit at which worker w of W begins, out of `units`.
LPQ_BOTH int64_t stream_begin(int64_t units, int w, int W) { return units / W * w + units % W * w / W; }
// The worker that has unit u.
LPQ_BOTH int stream_worker(int64_t units, int64_t u, int W)
{
    int w = (int)(u * W / units);            // begin(w) <= u * ... : at most one off either way
    while (w > 0 && stream_begin(units, w, W) > u) --w;
    while (w + 1 < W && stream_begin(units, w + 1, W) <= u) ++w;
    return w;
}

}  // namespace lpq

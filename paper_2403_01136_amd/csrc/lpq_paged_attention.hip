// Causal attention of new tokens of many sequences at once, over paged caches or over the packed rows themselves, with any number of query
// heads per K/V head:
//     out[row] = sum_j w_j v_j / sum_j w_j,   w_j = exp(q . k_j / sqrt(D) + slope (j - p)),   j <= p, p the row's position
// and zero where no key is visible.  The rows of a sequence and K/V head are its new tokens times the head's `group` query heads, row = token * group +
// g: all of them read the same keys, so a tile of rows is one product whatever the layout, and the diagonal of a group is narrow.
//
// Two kernels.  The streaming kernel (few rows per sequence: decode) reads the pages once, straight into registers, as fast as the memory gives them.
// The tile kernel (prompts and chunks) shares tiles of keys through LDS between 128 rows and is bound by the matrix and vector units.
// Both keep a running reference (about the largest score) and sum per row in fp32 and take exponents to base 2.  Weights are rounded to the inputs' type for the matrix units, and the sum
// that divides is of the rounded ones (pairs of them by one v_dot2, exact for subnormal weights too): what rounding does to a weight that outweighs the
// others then cancels.  (One prompt of 5801 tokens in bf16 with sums of unrounded weights: 2.2e-3 from 64 bits; so 2.1e-3; the output's rounding alone 1.6e-3.)
//
// In fp16 a weight of 2^-25 beside 1 would be zero, and lost the tens of thousands of them that a long context may have: there a row's largest weight is 2^15 (tile
// kernel: 2^7 to 2^15) beside a smallest one of 2^-24.
//
// Keys that no row may see (behind the sequence's end, pages that are not in the pool) are read from page 0 or a stale page, their scores are replaced and
// their values set to zero.  A value that only some rows of a tile see stays in the products, at weight zero for the others, and must be finite: what is not is
// set to zero too and added afterwards to the rows that see it (any weight of an infinity is one, of a NaN is one).  Such keys lie within the tokens of a tile,
// at the diagonal, so only the tiles there are looked through (by v_dot2 with zeros: NaN if anything is not finite), at up to 1 % of a call's time.  A prompt of 3000
// tokens, 8 heads over 2, one feature infinite in the first value row 58 us, in every row 91, without 58.
#include <algorithm>
#include <mutex>
#include <type_traits>

#include "lpq_common.h"
#include "lpq_device.h"
#include "lpq_lanes.h"
#include "lpq_paged_index.h"

namespace lpq {

namespace {

typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

template <int DT> struct Elem;
template <> struct Elem<LPQ_DT_FP16> {
    typedef _Float16 t;
    typedef h8 v8;
    static __device__ __forceinline__ f16x mfma32(v8 a, v8 b, f16x c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ f4 mfma16(v8 a, v8 b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ uint32_t pack(float a, float b) { const h2 p = {(_Float16)a, (_Float16)b}; return __builtin_bit_cast(uint32_t, p); }
    static __device__ __forceinline__ float add_pair(uint32_t p, float c) { return __builtin_amdgcn_fdot2(__builtin_bit_cast(h2, p), h2{1, 1}, c, false); }
    static __device__ __forceinline__ float probe_pair(uint32_t p, float c) { return __builtin_amdgcn_fdot2(__builtin_bit_cast(h2, p), h2{0, 0}, c, false); }
    enum { EXPONENT_STEP = 0x04000400 };                                        // one in the exponents' last places
    enum { TOP = 15 };                                                          // log2 of the largest weight
};
template <> struct Elem<LPQ_DT_BF16> {
    typedef __bf16 t;
    typedef bf8 v8;
    static __device__ __forceinline__ f16x mfma32(v8 a, v8 b, f16x c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ f4 mfma16(v8 a, v8 b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ uint32_t pack(float a, float b) { const bf2 p = {(__bf16)a, (__bf16)b}; return __builtin_bit_cast(uint32_t, p); }
    static __device__ __forceinline__ float add_pair(uint32_t p, float c) { return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf2, p), bf2{1.0f, 1.0f}, c, false); }
    static __device__ __forceinline__ float probe_pair(uint32_t p, float c) { return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf2, p), bf2{0.0f, 0.0f}, c, false); }
    enum { EXPONENT_STEP = 0x00800080 };
    enum { TOP = 0 };
};

// What a launch is about.  Pointers are to 16-bit elements.
struct AttnArgs {
    const uint16_t* qkv;                 // [M][(heads + 2 kv_heads) * D]
    const uint16_t *kp, *vp;             // pages; null: keys are the rows themselves
    const int32_t *table, *cu_q, *kv_lens;
    const float* slopes;
    uint16_t* out;                       // [M][heads * D]
    float* part;                         // partial results, or null: nothing is split
    int32_t n_seqs, M, heads, kv_heads, group, shift, n_pages, max_pages;
    int32_t rows_from, rows_to;          // sequences with rows_from <= rows < rows_to are this launch's
    int32_t workers;                     // streaming kernel: waves
    int32_t splits, least, tiles;        // tile kernel: K splits at most, key tiles of one at least; virtual row tiles
};

// A sequence as a kernel sees it.
struct Seq {
    int s, first, len, rows;             // rows of the batch [first, first + len); rows = len * group
    int pos0, ctx;                       // position of its first new token; keys that exist
};
__device__ __forceinline__ Seq make_seq(const AttnArgs& a, int s, int cu0, int cu1, int kv_len)
{
    const RowSpan r = row_span(cu0, cu1, a.M);
    Seq q;
    q.s = s;
    q.first = r.first;
    q.len = r.end - r.first;
    q.rows = q.len * a.group;
    const int kv = a.kv_lens ? kv_len : q.len;
    q.pos0 = token_position(kv, q.len, 0);
    q.ctx = a.kv_lens ? keys_of(kv, a.max_pages, a.shift) : q.len;
    return q;
}
__device__ __forceinline__ Seq load_seq(const AttnArgs& a, int s) { return make_seq(a, s, a.cu_q[s], a.cu_q[s + 1], a.kv_lens ? a.kv_lens[s] : 0); }
__device__ __forceinline__ bool takes(const AttnArgs& a, int rows) { return rows > 0 && rows >= a.rows_from && rows < a.rows_to; }

__device__ __forceinline__ int page_of_group(const AttnArgs& a, int s, int g)
{
    const int e = page_entry(g, a.shift, a.max_pages);
    return e < 0 ? -1 : page_checked(a.table[(size_t)s * a.max_pages + e], a.n_pages);
}

// Which of a pair of elements are infinite or NaN: bit 15 and bit 31.  An exponent of all ones carries into the sign's place.
template <int DT> __device__ __forceinline__ uint32_t not_finite(uint32_t pair) { return ((pair & 0x7fff7fffu) + (uint32_t)Elem<DT>::EXPONENT_STEP) & 0x80008000u; }
// What scores are taken from so that the largest, mx, has weight 2^top; without that factor where it would be lost beside the score.
__device__ __forceinline__ float reference(float mx, int top) { return top == 0 || !(__builtin_fabsf(mx) < 0x1p20f) ? mx : mx - (float)top; }
// The pair without the elements that `odd`, the above, names.
__device__ __forceinline__ uint32_t without(uint32_t pair, uint32_t odd) { return pair & ~(odd | (odd - (odd >> 15))); }
// Element e of a pair if it is infinite or NaN and `seen`, else zero.
template <int DT> __device__ __forceinline__ float odd_element(uint32_t pair, int e, bool seen)
{
    const float v = (float)__builtin_bit_cast(typename Elem<DT>::t, (uint16_t)(pair >> (16 * e)));
    return seen && !__builtin_isfinite(v) ? v : 0.0f;
}
// The value row of key j of a sequence and K/V head (the same for the whole wave): null if it has no page, or if all of it is finite.
template <int DT, int D>
__device__ __forceinline__ const uint16_t* odd_value_row(const AttnArgs& a, const Seq& q, int h, int j)
{
    const uint16_t* row;
    if (a.kp) {
        const int page = __builtin_amdgcn_readfirstlane(page_of_group(a, q.s, j >> 4));
        if (page < 0) return nullptr;
        row = a.vp + page_element(page, h, a.kv_heads, a.shift, D) + (size_t)(j & ((1 << a.shift) - 1)) * D;
    } else row = a.qkv + (size_t)(q.first + j) * ((a.heads + 2 * a.kv_heads) * D) + (a.heads + a.kv_heads + h) * D;
    const uint32_t pair = reinterpret_cast<const uint32_t*>(row)[threadIdx.x % (D / 2)];
    return __any(not_finite<DT>(pair) != 0) ? row : nullptr;
}

// ---- streaming kernel ---------------------------------------------------------------------------
// Bound by the memory: 4 D bytes per key and K/V head.  A persistent launch whose workers are single waves, four to a compute unit: the units of 32 keys of
// all (sequence, head, row tile) are one list, cut into equal shares, so contexts of any lengths fill the chip evenly.  A wave walks its share by itself:
// nothing waits for another wave.  Two units (K and V of 8 KB each at D = 128) have register buffers, and the next unit's K or V is asked for as soon as
// a buffer's contents are used up.
//
// Products on 16x16x32 matrix instructions, columns = rows of the problem (16 per column tile), so that scores land where the weights are wanted:
//   S^T = K . Q^T    A = K: lane (i = lane % 16, q = lane / 16) holds key i, features 32 step + 8 q + 0..7, loaded as they lie;
//                    register r of the result: key 4 q + r, column i.
//   O^T = V^T . P^T  over 32 keys: lane quarter q contracts over keys {4 q + 0..3, 16 + 4 q + 0..3}: its own scores of the two key tiles, so
//                    the weights go from result to operand in place.  V is read in whole rows (lane i: features F i .. F i + F - 1, F = D / 16, of the quarter's
//                    eight keys); V^T operand e, features F i + e, is one v_perm per register, no LDS.  Register r of result e: feature F (4 q + r) + e.
// A row tile that a share's border cuts is left in parts (unnormalised sums, maximum, sum), two slots per worker, which stream_combine_kernel adds up in the
// order of the keys; the worker in whose share it begins says so in its entry of `cuts`.
// (With workgroups of four waves as workers, units of 128 keys, the waves' sums added through LDS where a row tile ends, and a combining kernel that found
// the cut tiles by the same search: 16 sequences of 40 heads 36.5 + 18.3 us, 61 of 8 K/V heads 89.0 + 20.6, one of 90001 positions 61.4 + 27.5.)
constexpr int CUTS_PER_WG = 16;          // of the combining kernel
struct Cut { int32_t parts, first, row0, head_rows; };   // parts: 0: none; first row of the sequence; first row of the tile; K/V head * 64 + rows of the tile

__device__ __forceinline__ int64_t uniform64(int64_t v)
{
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)v), hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ int64_t shfl64(int64_t v, int from)
{
    const int lo = __shfl((int)(uint32_t)v, from), hi = __shfl((int)(v >> 32), from);
    return (int64_t)((uint64_t)(uint32_t)hi << 32 | (uint32_t)lo);
}
__device__ __forceinline__ int64_t scan64(int64_t v)                              // inclusive, over the wave
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t o = shfl64(v, lane - d);
        if (lane >= d) v += o;
    }
    return v;
}

__device__ __forceinline__ int64_t seq_units(const AttnArgs& a, int s, int tile_rows)
{
    if (s >= a.n_seqs) return 0;
    const Seq q = load_seq(a, s);
    return takes(a, q.rows) ? (int64_t)a.kv_heads * stream_row_tiles(q.rows, tile_rows) * stream_key_steps(q.ctx) : 0;
}

// A wave's share: units [u, end), the sequence that has unit u and the units before that sequence.
struct Share { int64_t u, end, units, seq_begin; int workers, s; };
struct ShareSmem { int64_t scan[4], begin[4]; int seq[4]; };
__device__ __forceinline__ Share find_share(const AttnArgs& a, int block, int tile_rows, ShareSmem& sm)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t first = seq_units(a, tid, tile_rows);                          // the usual batch has no more than 256 sequences: one pass
    int64_t mine = first;
    for (int s = tid + 256; s < a.n_seqs; s += 256) mine += seq_units(a, s, tile_rows);
    int64_t sum = scan64(mine);
    if (lane == 63) sm.scan[wave] = sum;
    __syncthreads();
    Share r;
    r.units = uniform64(sm.scan[0] + sm.scan[1] + sm.scan[2] + sm.scan[3]);
    r.workers = (int)min<int64_t>(a.workers, r.units);
    const int w0 = 4 * block;
    int64_t carry = 0;
    for (int s0 = 0; s0 < a.n_seqs; s0 += 256) {
        if (a.n_seqs > 256) {
            mine = s0 == 0 ? first : seq_units(a, s0 + tid, tile_rows);
            sum = scan64(mine);
            __syncthreads();
            if (lane == 63) sm.scan[wave] = sum;
            __syncthreads();
        }
        int64_t before = carry + sum - mine;
        for (int w = 0; w < 4; ++w) {
            if (w < wave) before += sm.scan[w];
            carry += sm.scan[w];
        }
        for (int w = 0; w < 4; ++w) {
            if (w0 + w >= r.workers) break;
            const int64_t u = stream_begin(r.units, w0 + w, r.workers);
            if (u >= before && u < before + mine) sm.seq[w] = s0 + tid, sm.begin[w] = before;
        }
    }
    __syncthreads();
    const int w = __builtin_amdgcn_readfirstlane(w0 + wave);
    r.u = r.end = r.seq_begin = 0;
    r.s = 0;
    if (w < r.workers) {
        r.u = stream_begin(r.units, w, r.workers);
        r.end = stream_begin(r.units, w + 1, r.workers);
        r.s = __builtin_amdgcn_readfirstlane(sm.seq[wave]);
        r.seq_begin = uniform64(sm.begin[wave]);
    }
    return r;
}

// One wave per SIMD, two units under way: few, long, contiguous streams suit the memory.  Waves per SIMD / units, us, 61 sequences of 8 K/V heads and one of 90001
// positions: 1 / 1 77.8, 66.0; 1 / 2 76.9, 63.2; 1 / 3 77.6, 62.7; 2 / 1 80.4, 66.4; 2 / 2 81.6, 66.5; 3 / 1 85.0, 72.4.
constexpr int STREAM_WAVES = 1, DEPTH = 2;

template <int DT, int D, int NT, bool ALIBI>
__device__ __forceinline__ void stream_block(const AttnArgs& a, int block, ShareSmem& sm)
{
    typedef typename Elem<DT>::v8 V8;
    constexpr int KJ = D / 32, F = D / 16, TILE_ROWS = STREAM_ROWS * NT;         // feature steps of S^T; features of a lane's V chunk
    constexpr int SLOT = TILE_ROWS * (D + 2);
    typedef uint32_t vchunk __attribute__((ext_vector_type(F / 2)));
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, quarter = lane >> 4;
    const float c = LOG2E / sqrtf((float)D);
    const int cols = (a.heads + 2 * a.kv_heads) * D, page_mask = (1 << a.shift) - 1;

    const Share share = find_share(a, block, TILE_ROWS, sm);
    const int w = 4 * block + wave;
    int64_t u = share.u, s_begin = share.seq_begin;
    int s = share.s;
    Cut cut{0, 0, 0, 0};
    int64_t s_units = u < share.end ? seq_units(a, s, TILE_ROWS) : 0;

    while (u < share.end) {
        if (u >= s_begin + s_units) {                  // the next sequence with units, 64 looked at together: there is one, u is below the total
            s_begin += s_units;
            uint64_t found = 0;
            int64_t mine = 0;
            for (++s; !found && s < a.n_seqs; s += found ? 0 : 64) {
                mine = seq_units(a, s + lane, TILE_ROWS);
                found = __ballot(mine > 0);
            }
            if (!found) break;                         // lengths that change under the kernel
            const int k = __builtin_ctzll(found);
            s = __builtin_amdgcn_readfirstlane(s + k);
            s_units = uniform64(shfl64(mine, k));
        }
        const Seq q = load_seq(a, s);
        const int steps = stream_key_steps(q.ctx), tiles = stream_row_tiles(q.rows, TILE_ROWS);
        const int64_t at = u - s_begin, tile = at >> 31 ? at / steps : (int64_t)((uint32_t)at / (uint32_t)steps), first = s_begin + tile * steps;
        const int h = tiles == 1 ? (int)tile : (int)(tile / tiles), rt = tiles == 1 ? 0 : (int)(tile % tiles);
        if (!a.part && first < u) {                    // nowhere to leave parts: a worker takes the row tiles that begin in its share, whole
            u = first + steps;
            continue;
        }
        const int n0 = (int)(u - first), n1 = a.part ? (int)min<int64_t>(steps, share.end - first) : steps;
        const int row0 = rt * TILE_ROWS, n_rows = min(TILE_ROWS, q.rows - row0);
        const int t_first = row0 / a.group, t_last = (row0 + n_rows - 1) / a.group;
        const int key_end = min(q.ctx, q.pos0 + t_last + 1);                     // no row sees a key from here on (may be below 1)
        const int all_see = min(key_end, q.pos0 + t_first + 1);                 // every row sees the keys below
        const int n_last = max(n0, min(n1, (key_end + STREAM_KEYS - 1) / STREAM_KEYS));

        // pages: lane 2 n + i holds the page of 16-key group i of step k + n, 32 steps at a time
        int ids = 0;
        auto load_ids = [&](int k) { ids = k + lane / 2 < n_last ? page_of_group(a, s, 2 * k + lane) : -1; };
        if (n0 < n_last) load_ids(n0);
        // the lane's column(s): query row, position, slope
        V8 qf[NT][KJ];
        int p[NT];
        float slope[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int r = row0 + min(STREAM_ROWS * t + col, n_rows - 1), tok = r / a.group, head = h * a.group + r % a.group;
            const uint16_t* qp = a.qkv + (size_t)(q.first + tok) * cols + head * D + 8 * quarter;
#pragma unroll
            for (int j = 0; j < KJ; ++j) qf[t][j] = *reinterpret_cast<const V8*>(qp + 32 * j);
            p[t] = q.pos0 + tok;
            slope[t] = ALIBI ? a.slopes[head] * LOG2E : 0.0f;
        }
        float m[NT], l[NT];
        f4 o[NT][F];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            m[t] = -INFINITY;
            l[t] = 0.0f;
#pragma unroll
            for (int e = 0; e < F; ++e) o[t][e] = f4{0.0f, 0.0f, 0.0f, 0.0f};
        }

        const uint32_t koff = (uint32_t)(col * D + 8 * quarter) * 2u, voff = (uint32_t)(4 * quarter * D + F * col) * 2u;
        V8 kf[DEPTH][2][KJ];
        vchunk vf[DEPTH][2][4];
        uint32_t bad_of[DEPTH];                        // of the buffers' steps: bit i: 16-key group i has no page
        uint64_t bad_ids = 0;                          // bit l: lane l's group has none
        bool odd = false;                              // a step that not every row sees had values that are not finite
        int ids_from = n0;
        // step n's loads from the pages `from`: an address is a scalar base and a 32-bit lane offset
        auto page_bytes = [&](const uint16_t* pages, int n, int i) {
            const int id = max(__builtin_amdgcn_readlane(ids, 2 * (n - ids_from) + i), 0);
            return reinterpret_cast<const uint8_t*>(pages + (size_t)page_element(id, h, a.kv_heads, a.shift, D) + (size_t)((STREAM_KEYS * n + 16 * i) & page_mask) * D);
        };
        auto load_k = [&](int n, int x) {
            if (n - ids_from == 32) {
                ids_from = n;
                load_ids(n);
                bad_ids = __ballot(ids < 0);
            }
            bad_of[x] = (uint32_t)(bad_ids >> (2 * (n - ids_from))) & 3u;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint8_t* b = page_bytes(a.kp, n, i);
#pragma unroll
                for (int j = 0; j < KJ; ++j) kf[x][i][j] = __builtin_nontemporal_load(reinterpret_cast<const V8*>(b + koff + 64 * j));
            }
        };
        auto load_v = [&](int n, int x) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint8_t* b = page_bytes(a.vp, n, i);
#pragma unroll
                for (int r = 0; r < 4; ++r) vf[x][i][r] = __builtin_nontemporal_load(reinterpret_cast<const vchunk*>(b + voff + 2 * D * r));
            }
        };
        if (n0 < n_last) bad_ids = __ballot(ids < 0);
#pragma unroll
        for (int x = 0; x < DEPTH; ++x)
            if (n0 + x < n_last) {
                load_k(n0 + x, x);
                load_v(n0 + x, x);
            }
        auto step = [&](int n, int x) {
#pragma clang fp contract(off)                         // an exponent is a rounded score less the largest rounded score: at most zero, whatever their size
            const int key0 = STREAM_KEYS * n;
            const uint32_t bad = bad_of[x];
            const bool plain = bad == 0 && key0 + STREAM_KEYS <= all_see, more = n + DEPTH < n_last;
            f4 sc[NT][2];
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    sc[t][i] = f4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int j = 0; j < KJ; ++j) sc[t][i] = Elem<DT>::mfma16(kf[x][i][j], qf[t][j], sc[t][i]);
                }
            __builtin_amdgcn_sched_barrier(0);
            if (more) load_k(n + DEPTH, x);
            __builtin_amdgcn_sched_barrier(0);
            V8 pf[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                float mx = -INFINITY;
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int key = key0 + 16 * i + 4 * quarter + r;
                        float v = sc[t][i][r] * c;
                        if constexpr (ALIBI) v = __builtin_fmaf(slope[t], (float)(key - p[t]), v);
                        if (!plain) v = (bad >> i & 1) || key > p[t] || key >= key_end ? -INFINITY : v;
                        sc[t][i][r] = v;
                        mx = fmaxf(mx, v);
                    }
                f2 z = both_rows(mx);
                z = both_halves(fmaxf(z[0], z[1]));
                mx = fmaxf(z[0], z[1]);
                if (__any(mx - m[t] > (float)Elem<DT>::TOP)) {
                    const float mn = fmaxf(m[t], reference(mx, Elem<DT>::TOP)), alpha = __builtin_amdgcn_exp2f(m[t] - (mn == -INFINITY ? 0.0f : mn));
                    l[t] *= alpha;
#pragma unroll
                    for (int e = 0; e < F; ++e) o[t][e] *= alpha;
                    m[t] = mn;
                }
                const float ms = m[t] == -INFINITY ? 0.0f : m[t];
                u32x4 pk;
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int r = 0; r < 4; r += 2) {
                        pk[2 * i + r / 2] = Elem<DT>::pack(__builtin_amdgcn_exp2f(sc[t][i][r] - ms), __builtin_amdgcn_exp2f(sc[t][i][r + 1] - ms));
                        l[t] = Elem<DT>::add_pair(pk[2 * i + r / 2], l[t]);
                    }
                pf[t] = __builtin_bit_cast(V8, pk);
            }
            if (!plain)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if ((bad >> i & 1) || key0 + 16 * i + 4 * quarter + r >= key_end) vf[x][i][r] = vchunk{};
            if (all_see < key_end && key0 + STREAM_KEYS > all_see) {             // the diagonal of more than one token
                float probe = 0.0f;                    // NaN once a value has been infinite or NaN
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
#pragma unroll
                        for (int e = 0; e < F / 2; ++e) probe = Elem<DT>::probe_pair(vf[x][i][r][e], probe);
                if (__builtin_expect(__any(probe != probe), 0)) {
                    odd = true;
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
#pragma unroll
                            for (int e = 0; e < F / 2; ++e) vf[x][i][r][e] = without(vf[x][i][r][e], not_finite<DT>(vf[x][i][r][e]));
                }
            }
#pragma unroll
            for (int e = 0; e < F; ++e) {
                u32x4 vt;                              // element e of the lane's chunks of the quarter's eight keys
                const uint32_t sel = e & 1 ? 0x07060302u : 0x05040100u;
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int r = 0; r < 4; r += 2) vt[2 * i + r / 2] = __builtin_amdgcn_perm(vf[x][i][r + 1][e / 2], vf[x][i][r][e / 2], sel);
#pragma unroll
                for (int t = 0; t < NT; ++t) o[t][e] = Elem<DT>::mfma16(__builtin_bit_cast(V8, vt), pf[t], o[t][e]);
            }
            __builtin_amdgcn_sched_barrier(0);
            if (more) load_v(n + DEPTH, x);
            __builtin_amdgcn_sched_barrier(0);
        };
        for (int n = n0; n < n_last; n += DEPTH)
#pragma unroll
            for (int x = 0; x < DEPTH; ++x)            // buffers by name
                if (n + x < n_last) step(n + x, x);

        if (__builtin_expect(odd, 0))
#pragma unroll 1
            for (int j = max(STREAM_KEYS * n0, all_see / STREAM_KEYS * STREAM_KEYS); j < min(STREAM_KEYS * n_last, key_end); ++j) {
                const uint16_t* row = odd_value_row<DT, D>(a, q, h, j);
                if (!row) continue;
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const vchunk x = *reinterpret_cast<const vchunk*>(row + F * (4 * quarter + g));
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int e = 0; e < F; ++e) o[t][e][g] += odd_element<DT>(x[e / 2], e % 2, j <= p[t]);
                }
            }

        // a whole row tile's results, or a part's sums
        const bool whole = n0 == 0 && n1 == steps;
        float* const slot = a.part + (size_t)(2 * w + (first < share.u ? 0 : 1)) * SLOT;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int ri = STREAM_ROWS * t + col, r = row0 + min(ri, n_rows - 1), tok = r / a.group, head = h * a.group + r % a.group;
            f2 z = both_rows(l[t]);
            z = both_halves(z[0] + z[1]);
            const float L = z[0] + z[1];
            if (ri < n_rows) {
                if (whole) {
                    const float inv = L == 0.0f ? 0.0f : 1.0f / L;
                    uint16_t* op = a.out + (size_t)(q.first + tok) * a.heads * D + head * D;
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        vchunk y;
#pragma unroll
                        for (int e = 0; e < F; e += 2) y[e / 2] = Elem<DT>::pack(o[t][e][g] * inv, o[t][e + 1][g] * inv);
                        *reinterpret_cast<vchunk*>(op + F * (4 * quarter + g)) = y;
                    }
                } else {
#pragma unroll
                    for (int g = 0; g < 4; ++g)
#pragma unroll
                        for (int e = 0; e < F; e += 4)
                            *reinterpret_cast<f4*>(slot + ri * D + F * (4 * quarter + g) + e) = f4{o[t][e][g], o[t][e + 1][g], o[t][e + 2][g], o[t][e + 3][g]};
                    if (quarter == 0) *reinterpret_cast<f2*>(slot + TILE_ROWS * D + 2 * ri) = f2{m[t], L};
                }
            }
        }
        if (!whole && first >= share.u)                // it begins here and ends in another worker's share
            cut = Cut{stream_worker(share.units, first + steps - 1, share.workers) - w + 1, q.first, row0, 64 * h + n_rows};
        u = first + n1;
    }
    if (a.part && lane == 0) reinterpret_cast<Cut*>(a.part + (size_t)2 * a.workers * SLOT)[w] = cut;
}

template <int DT, int D, int NT, bool ALIBI>
__global__ __launch_bounds__(256, STREAM_WAVES) void stream_attention_kernel(AttnArgs a)
{
    __shared__ ShareSmem sm;
    stream_block<DT, D, NT, ALIBI>(a, (int)blockIdx.x, sm);
}

// Adds up the parts of the row tiles that the entries of `cuts` name, 16 entries a workgroup; blockIdx.y: rows and, if LONG, slices of 32 features.  Many
// short lists of parts: a wave takes a row of a cut, D / 4 lanes of four features each for every (256 / D)-th part.  LONG, for few lists of hundreds of parts:
// the workgroup takes a slice, 8 lanes for every 32nd part, the sums added through LDS.  Either is right for any list.
template <int DT, int D, int NT, bool LONG>
__global__ __launch_bounds__(256) void stream_combine_kernel(AttnArgs a)
{
    constexpr int TILE_ROWS = STREAM_ROWS * NT, SLOT = TILE_ROWS * (D + 2), SLICES = LONG ? D / 32 : 1, LANES = D / SLICES / 4, WAYS = (LONG ? 256 : 64) / LANES;
    __shared__ __attribute__((aligned(16))) float red[4][36];                    // LONG only: a wave's sums
    const Cut* cuts = reinterpret_cast<const Cut*>(a.part + (size_t)2 * a.workers * SLOT);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), team = LONG ? (int)threadIdx.x : lane;
    const int f = 32 * ((int)blockIdx.y % SLICES) + 4 * (team % LANES), way = team / LANES, row_step = (int)gridDim.y / SLICES;
    const int w0 = CUTS_PER_WG * (int)blockIdx.x;
    Cut mine{0, 0, 0, 0};
    if (lane < CUTS_PER_WG && w0 + lane < a.workers) mine = cuts[w0 + lane];
    uint64_t todo = __ballot(mine.parts != 0);
    for (int i = 0; todo; ++i, todo &= todo - 1) {
        if (!LONG && i % 4 != wave) continue;
        const int k0 = __builtin_ctzll(todo), w = w0 + k0;
        const int parts = __builtin_amdgcn_readlane(mine.parts, k0), first = __builtin_amdgcn_readlane(mine.first, k0);
        const int row0 = __builtin_amdgcn_readlane(mine.row0, k0), hr = __builtin_amdgcn_readlane(mine.head_rows, k0), h = hr >> 6;
        for (int ri = (int)blockIdx.y / SLICES; ri < (hr & 63); ri += row_step) {
            float m = -INFINITY, l = 0.0f;
            f4 v = {0.0f, 0.0f, 0.0f, 0.0f};
            auto add = [&](float km, float kl, const f4& kv) {
                const float mn = fmaxf(m, km), ms = mn == -INFINITY ? 0.0f : mn, x = __builtin_amdgcn_exp2f(m - ms), y = __builtin_amdgcn_exp2f(km - ms);
                m = mn;
                l = l * x + kl * y;
                v = v * x + kv * y;
            };
#pragma unroll 4
            for (int k = way; k < parts; k += WAYS) {  // part k: worker w + k; the first is in its slot 1, the others, which begin inside the row tile, in their slot 0
                const float* ps = a.part + (size_t)(2 * (w + k) + (k == 0 ? 1 : 0)) * SLOT;
                const f2 ml = *reinterpret_cast<const f2*>(ps + TILE_ROWS * D + 2 * ri);
                const f4 o = *reinterpret_cast<const f4*>(ps + ri * D + f);
                add(ml[0], ml[1], o);
            }
#pragma unroll
            for (int d = LANES; d < 64; d *= 2) add(__shfl_xor(m, d), __shfl_xor(l, d), f4{__shfl_xor(v[0], d), __shfl_xor(v[1], d), __shfl_xor(v[2], d), __shfl_xor(v[3], d)});
            if constexpr (LONG) {
                __syncthreads();                       // the last row's sums are read
                if (lane < LANES) {
                    *reinterpret_cast<f4*>(&red[wave][4 * lane]) = v;
                    if (lane == 0) red[wave][32] = m, red[wave][33] = l;
                }
                __syncthreads();
                if (way != 0) continue;
#pragma unroll
                for (int k = 1; k < 4; ++k) add(red[k][32], red[k][33], *reinterpret_cast<const f4*>(&red[k][4 * lane]));
            }
            if (way != 0) continue;
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;
            const int r = row0 + ri, tok = r / a.group, head = h * a.group + r % a.group;
            *reinterpret_cast<u32x2*>(a.out + (size_t)(first + tok) * a.heads * D + head * D + f) =
                u32x2{Elem<DT>::pack(v[0] * inv, v[1] * inv), Elem<DT>::pack(v[2] * inv, v[3] * inv)};
        }
    }
}

// ---- tile kernel ----------------------------------------------------------------------------------
// Bound by the matrix and vector units together.  A workgroup takes 128 rows (token, head of the group) of one sequence and K/V head, each of its four
// waves 32 of them, and walks the visible keys 64 at a time; K and V tiles are shared through LDS (two buffers each, filled by global-to-LDS loads
// while the tile before is multiplied; 64 KB at D = 128, two workgroups per compute unit).
// Both products are transposed, on 32x32x16: S^T = K . Q^T, O^T = V^T . P^T; a lane holds scores of one row (column lane % 32), so the softmax needs
// one exchange between the halves of the wave.  Register v of a score tile is key 8 (v / 4) + 4 half + v % 4; registers 8 c .. 8 c + 7 of a lane go as they are
// into the weights' operand of 16-key step c, which contracts half h over keys {4 h + 0..3, 8 + 4 h + 0..3}.  V^T operands in that order are read from row-major
// tiles by the transposing LDS read: each 16 lanes fetch four keys x 16 features and lane i gets feature i of the four.
// 16-byte chunks are swizzled: K's by the row (16 lanes read 16 rows), V's by the row modulo 4 in steps of four chunks (32 lanes read four rows x 64 bytes).
// Workgroup ids go round-robin over the 8 XCDs; a head of keys, or a class of row tiles of it where there are fewer than eight, stays on one of them.
template <int D> __device__ __forceinline__ int k_swizzle(int row) { return D == 128 ? row & 15 : (row >> 1) & 7; }
template <int D> __device__ __forceinline__ int v_swizzle(int row) { return D == 128 ? 4 * (row & 3) : 4 * ((row >> 1) & 1); }

// log2 of what a row's maximum may lag behind its largest score: sums are then at most 2^8 larger.  Renewed with every larger score there is hardly a
// tile without 32 rows' sums being multiplied: one prompt of 5801 tokens 684 us, so 655; its error in bf16 1.9e-3, so 2.1e-3; in fp16 2.2e-4 and 2.3e-4.
constexpr int LAZY = 8;
constexpr float LARGE_SCORE = 0x1p22f;                 // half of the last place of scores below: at most a quarter
// Of a split.  At least 4 / 8 key tiles, us: 64 tokens behind 6000 positions 23 + 9 / 22 + 7, 512 tokens of 16 heads over 2 behind 4000 32 + 9 / 30 + 7; 16: 33 + 5 both.
constexpr int LEAST_KEY_TILES = 8, LONG_KEY_TILES = 48;

// The sequence of virtual tile v: false if it is nobody's.  Every wave for itself.  Up to 63 sequences: one load of every lane's has all that is needed.
// More: two rounds of 64 candidates, then the one found.
__device__ __forceinline__ bool tile_sequence(const AttnArgs& a, int v, Seq* q)
{
    const int lane = threadIdx.x & 63;
    auto begins = [&](int cu, int s) { return s < a.n_seqs && tile_start(clamp_int(cu, 0, a.M), a.group, s, TILE_ROWS_Q) <= v; };
    if (a.n_seqs < 64) {
        const int cu = a.cu_q[min(lane, a.n_seqs)], kv = a.kv_lens ? a.kv_lens[min(lane, a.n_seqs - 1)] : 0;
        const int s = __popcll(__ballot(begins(cu, lane))) - 1;
        if (s >= 0) *q = make_seq(a, s, __builtin_amdgcn_readlane(cu, s), __builtin_amdgcn_readlane(cu, s + 1), __builtin_amdgcn_readlane(kv, s));
        return s >= 0;
    }
    auto begins_at = [&](int s) { return s < a.n_seqs && begins(a.cu_q[s], s); };
    const int stride = (a.n_seqs + 63) / 64, block = __popcll(__ballot(begins_at(lane * stride))) - 1;
    if (block < 0) return false;
    const int s = block * stride + __popcll(__ballot(lane < stride && begins_at(block * stride + lane))) - 1;
    if (s < 0) return false;
    *q = load_seq(a, __builtin_amdgcn_readfirstlane(s));
    return true;
}

// What a workgroup of the tile kernel, or of its combining kernel, is about.
struct Tile { Seq q; int row0, n_rows, key_end, key_tiles; };
__device__ __forceinline__ bool tile_of(const AttnArgs& a, int v, Tile* t)
{
    if (!tile_sequence(a, v, &t->q)) return false;
    t->row0 = TILE_ROWS_Q * (v - tile_start(t->q.first, a.group, t->q.s, TILE_ROWS_Q));
    if (!takes(a, t->q.rows) || t->row0 < 0 || t->row0 >= t->q.rows) return false;
    t->n_rows = min((int)TILE_ROWS_Q, t->q.rows - t->row0);
    t->key_end = max(0, min(t->q.ctx, t->q.pos0 + (t->row0 + t->n_rows - 1) / a.group + 1));
    t->key_tiles = max(1, (t->key_end + TILE_KEYS - 1) / TILE_KEYS);
    return true;
}

// Where a split leaves its sums ([rows][D], then maximum and sum of each row), or null: there is only one.
template <int D>
__device__ __forceinline__ float* tile_part(const AttnArgs& a, const KeySplit& ks, int h, int v, int split)
{
    return ks.used == 1 ? nullptr : a.part + (((size_t)h * a.tiles + v) * a.splits + split) * ((size_t)TILE_ROWS_Q * (D + 2));
}

// The results (part null) or sums of 32 rows of a tile from row wr on: a lane has row wr + lane % 32 = (tok, head) and its features 32 d + 8 i + 4 (lane / 32) +
// 0 .. 3 in registers 4 i .. 4 i + 3 of o[d], the maximum m and the sum l.
template <int DT, int D>
__device__ __forceinline__ void store_rows(const AttnArgs& a, const Tile& tl, int h, const KeySplit& ks, float* part, const f16x (&o)[D / 32], float m, float l,
                                           int wr, int tok, int head)
{
    constexpr int DTL = D / 32;
    const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
    const bool store = wr + col < tl.n_rows;
    float* const ml = part + (size_t)TILE_ROWS_Q * D;
    if (part) {
        if (store) {
#pragma unroll
            for (int d = 0; d < DTL; ++d)
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                    *reinterpret_cast<f4*>(part + (size_t)(wr + col) * D + 32 * d + 2 * i + 4 * half) = f4{o[d][i], o[d][i + 1], o[d][i + 2], o[d][i + 3]};
            if (half == 0) *reinterpret_cast<f2*>(ml + 2 * (wr + col)) = f2{m, l};
        }
    } else {                                           // the halves trade so that each stores 16 bytes
        uint16_t* const orow = a.out + (size_t)(tl.q.first + tok) * a.heads * D + head * D;
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
        for (int d = 0; d < DTL; ++d)
#pragma unroll
            for (int b = 0; b < 4; b += 2) {
                u32x4 x;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const u32x2 t = __builtin_amdgcn_permlane32_swap(Elem<DT>::pack(o[d][4 * b + 2 * i] * inv, o[d][4 * b + 2 * i + 1] * inv),
                                                                     Elem<DT>::pack(o[d][4 * b + 4 + 2 * i] * inv, o[d][4 * b + 5 + 2 * i] * inv), false, false);
                    x[i] = t[0];
                    x[2 + i] = t[1];
                }
                if (store) *reinterpret_cast<u32x4*>(orow + 8 * half + 32 * d + 8 * b) = x;
            }
    }
}

extern __shared__ __attribute__((aligned(16))) uint8_t smem_raw[];              // K, K, V, V, a word per wave (dynamic: ahead of a read of a named array the compiler waits for every load into it)

template <int DT, int D, bool ALIBI, bool PAGED>
__device__ __forceinline__ void tile_block(const AttnArgs& a, int block)
{
    typedef typename Elem<DT>::v8 V8;
    constexpr int CH = D / 8, KS = D / 16, DTL = D / 32, ROWS = 512 / D, FILLS = 16 / ROWS;       // chunks of a row; feature steps; feature tiles; keys per load; loads of a wave's 16 keys
    constexpr int TILE_BYTES = TILE_KEYS * D * 2;
    constexpr bool BACKWARD = ALIBI;                   // biases grow towards the diagonal: from there on the first tiles have the maximum
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
    // (head, split, row tile) of this workgroup: the last row tiles, with the longest walks, first
    const int classes = a.kv_heads % 8 == 0 ? 1 : a.kv_heads % 4 == 0 ? 2 : a.kv_heads % 2 == 0 ? 4 : 8;
    const int per_xcd = a.kv_heads * classes / 8, per_class = (a.tiles + classes - 1) / classes;
    const int slot = block >> 3, combo = (block & 7) + 8 * (slot % per_xcd), rest = slot / per_xcd;
    const int h = combo % a.kv_heads, split = rest / per_class, v = a.tiles - 1 - ((rest % per_class) * classes + combo / a.kv_heads);
    Tile tl;
    if (v < 0 || !tile_of(a, v, &tl)) return;
    const KeySplit ks = key_split(tl.key_tiles, a.splits, a.least, split);
    if (split >= ks.used) return;
    const Seq& q = tl.q;
    const int cols = (a.heads + 2 * a.kv_heads) * D;
    const int wr0 = 32 * wave;                                                  // this wave's first row of the tile
    const bool active = wr0 < tl.n_rows;
    const int r = tl.row0 + min(wr0 + col, tl.n_rows - 1), tok = r / a.group, head = h * a.group + r % a.group, p = q.pos0 + tok;
    const float c = LOG2E / sqrtf((float)D);
    const float slope = ALIBI ? a.slopes[head] * LOG2E : 0.0f;
    const int all_see = min(tl.key_end, q.pos0 + (tl.row0 + min(wr0, tl.n_rows - 1)) / a.group + 1);        // keys below: every row of the wave sees them
    const int my_end = active ? min(ks.end, (max(0, min(q.ctx, q.pos0 + (tl.row0 + min(wr0 + 31, tl.n_rows - 1)) / a.group + 1)) + TILE_KEYS - 1) / TILE_KEYS) : 0;

    // fills: this wave brings keys 16 wave .. 16 wave + 15 of a tile, of one page
    int ids = 0, ids_from = 0;
    uint64_t bad_ids = 0;
    auto load_ids = [&](int j) {                       // of 16 tiles, j and those that come behind it
        ids_from = BACKWARD ? max(j - 15, 0) : j;
        const int g = 4 * ids_from + lane;
        ids = 16 * g < tl.key_end ? page_of_group(a, q.s, g) : -1;
        bad_ids = __ballot(ids < 0);
    };
    const uint32_t kl = (uint32_t)((lane / CH) * (PAGED ? D : cols) + 8 * ((lane % CH) ^ k_swizzle<D>(lane / CH))) * 2u;
    const uint32_t vl = (uint32_t)((lane / CH) * (PAGED ? D : cols) + 8 * ((lane % CH) ^ v_swizzle<D>(lane / CH))) * 2u;
    // asks for tile j; which of its 16-key groups have no page
    auto fill = [&](int j, int buf) -> uint32_t {
        uint8_t *ks_ = smem_raw + buf * TILE_BYTES + 16 * wave * D * 2, *vs_ = ks_ + 2 * TILE_BYTES;
        uint32_t bad = 0;
        if constexpr (PAGED) {
            if ((uint32_t)(j - ids_from) >= 16u) load_ids(j);
            const int id = max(__builtin_amdgcn_readlane(ids, 4 * (j - ids_from) + wave), 0);
            bad = (uint32_t)(bad_ids >> (4 * (j - ids_from))) & 15u;
            const size_t at = (size_t)page_element(id, h, a.kv_heads, a.shift, D) + (size_t)((TILE_KEYS * j + 16 * wave) & ((1 << a.shift) - 1)) * D;
            const uint8_t *kb = reinterpret_cast<const uint8_t*>(a.kp + at), *vb = reinterpret_cast<const uint8_t*>(a.vp + at);
#pragma unroll
            for (int i = 0; i < FILLS; ++i) {
                const uint32_t ko = kl ^ (uint32_t)(k_swizzle<D>(ROWS * i) * 16);
                __builtin_amdgcn_global_load_lds((gptr_t)(kb + ROWS * i * D * 2 + ko), (lptr_t)(ks_ + 1024 * i), 16, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < FILLS; ++i) __builtin_amdgcn_global_load_lds((gptr_t)(vb + ROWS * i * D * 2 + vl), (lptr_t)(vs_ + 1024 * i), 16, 0, 0);
        } else {
            const int k0 = TILE_KEYS * j + 16 * wave;
            const uint8_t* base = reinterpret_cast<const uint8_t*>(a.qkv + (size_t)q.first * cols + (a.heads + h) * D);
            if (TILE_KEYS * (j + 1) <= q.len) {
#pragma unroll
                for (int i = 0; i < FILLS; ++i) {
                    const uint8_t* kb = base + (size_t)(k0 + ROWS * i) * cols * 2;
                    const uint32_t ko = kl ^ (uint32_t)(k_swizzle<D>(ROWS * i) * 16);
                    __builtin_amdgcn_global_load_lds((gptr_t)(kb + ko), (lptr_t)(ks_ + 1024 * i), 16, 0, 0);
                    __builtin_amdgcn_global_load_lds((gptr_t)(kb + a.kv_heads * D * 2 + vl), (lptr_t)(vs_ + 1024 * i), 16, 0, 0);
                }
            } else {                                   // rows behind the sequence's last: that one, in their place
#pragma unroll
                for (int i = 0; i < FILLS; ++i) {
                    const int row = ROWS * i + lane / CH;
                    const uint8_t* kb = base + (size_t)min(k0 + row, q.len - 1) * cols * 2;
                    __builtin_amdgcn_global_load_lds((gptr_t)(kb + 16 * ((lane % CH) ^ k_swizzle<D>(row))), (lptr_t)(ks_ + 1024 * i), 16, 0, 0);
                    __builtin_amdgcn_global_load_lds((gptr_t)(kb + a.kv_heads * D * 2 + 16 * ((lane % CH) ^ v_swizzle<D>(row))), (lptr_t)(vs_ + 1024 * i), 16, 0, 0);
                }
            }
        }
        return bad;
    };

    V8 qf[KS];                                         // Q^T operands: lane (row col, features 16 k + 8 half ..)
    {
        const uint16_t* qp = a.qkv + (size_t)(q.first + tok) * cols + head * D + 8 * half;
#pragma unroll
        for (int k = 0; k < KS; ++k) qf[k] = *reinterpret_cast<const V8*>(qp + 16 * k);
    }
    f16x o[DTL];
#pragma unroll
    for (int d = 0; d < DTL; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
    float m = -INFINITY, l = 0.0f;                     // the maximum in use of the lane's row; this lane's part of its sum
    constexpr int TOP = Elem<DT>::TOP ? Elem<DT>::TOP - LAZY : 0;
    bool large = false;                                // the maximum of some row of the wave is
    // operand reads, bytes within a buffer
    uint32_t ka[KS], va[DTL];
#pragma unroll
    for (int k = 0; k < KS; ++k) ka[k] = (uint32_t)(col * D * 2 + 16 * ((2 * k + half) ^ k_swizzle<D>(col)));
#pragma unroll
    for (int d = 0; d < DTL; ++d) {
        const int row = 4 * half + (lane & 15) / 4, chunk = 4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
        va[d] = (uint32_t)(2 * TILE_BYTES + row * D * 2 + 16 * (chunk ^ v_swizzle<D>(row)) + 8 * (lane & 1));
    }

    // keys from here on are not seen by every row of the tile; and whether a wave has set values of theirs to zero, in LDS behind the tiles
    const int first_hidden = min(tl.key_end, q.pos0 + tl.row0 / a.group + 1);
    uint32_t* const odd_values = reinterpret_cast<uint32_t*>(smem_raw + 4 * TILE_BYTES);
    if (lane == 0) odd_values[wave] = 0;

    float near[ALIBI ? 16 : 1];                        // bias of a register's key within its 32
    if constexpr (ALIBI)
#pragma unroll
        for (int i = 0; i < 16; ++i) near[i] = slope * (float)(8 * (i / 4) + i % 4);

    const int tiles = ks.end - ks.begin, j_first = BACKWARD ? ks.end - 1 : ks.begin;
    if constexpr (PAGED) load_ids(j_first);
    uint32_t bad = 0, bad_next = fill(j_first, 0);
    for (int n = 0; n < tiles; ++n) {
        const int j = BACKWARD ? j_first - n : j_first + n, buf = n & 1, j0 = TILE_KEYS * j;
        bad = bad_next;
        __builtin_amdgcn_s_waitcnt(0x0F70);            // vmcnt(0): this wave's part of tile j has landed
        if (bad != 0 || j0 + TILE_KEYS > tl.key_end) { // values of keys that no row sees: zero, like their weights
#pragma unroll
            for (int i = 0; i < FILLS; ++i) {
                const int row = 16 * wave + ROWS * i + lane / CH;
                if ((bad >> wave & 1) || j0 + row >= tl.key_end) *reinterpret_cast<u32x4*>(smem_raw + 2 * TILE_BYTES + buf * TILE_BYTES + (16 * wave + ROWS * i) * D * 2 + 16 * lane) = u32x4{};
            }
        }
        if (j0 + 16 * wave + 16 > first_hidden && first_hidden < tl.key_end) {      // the wave's keys are not seen by every row: none of their values may be infinite or NaN
            u32x4* const at = reinterpret_cast<u32x4*>(smem_raw + (2 + buf) * TILE_BYTES + 16 * wave * D * 2 + 16 * lane);
            float probe = 0.0f;
#pragma unroll
            for (int i = 0; i < FILLS; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) probe = Elem<DT>::probe_pair(at[64 * i][e], probe);
            if (__builtin_expect(__any(probe != probe), 0)) {
#pragma unroll 1
                for (int i = 0; i < FILLS; ++i) {
                    u32x4 x = at[64 * i];
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = without(x[e], not_finite<DT>(x[e]));
                    at[64 * i] = x;
                }
                odd_values[wave] = 1;
            }
        }
        __syncthreads();                               // everybody's part has landed, and the tile before is no longer read
        if (n + 1 < tiles) bad_next = fill(BACKWARD ? j - 1 : j + 1, buf ^ 1);
        if (j >= my_end) continue;
        // Operands are read a batch ahead of the matrix instructions that take them, and the wait for a batch stands ahead of the next batch's issue:
        // with global-to-LDS loads under way the compiler waits for every LDS read at each use.
        auto wait_reads = [] { __builtin_amdgcn_s_waitcnt(0xC07F); __builtin_amdgcn_sched_barrier(0); };
        const uint8_t* tile = smem_raw + buf * TILE_BYTES;
        V8 ra[8], rb[8];
        auto read_k = [&](V8 (&x)[8], int kt) {
#pragma unroll
            for (int k = 0; k < KS; ++k) x[k] = *reinterpret_cast<const V8*>(tile + ka[k] + 32 * kt * D * 2);
        };
        auto read_v = [&](V8 (&x)[8], int d0) {        // features 32 d0 .. 32 d0 + 63, the tile's four 16-key steps
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint8_t* at = tile + va[d0 + i / 4] + 16 * (i % 4) * D * 2;
                typedef __attribute__((address_space(3))) s16x4* tr_t;
                const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_t)at), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_t)(at + 8 * D * 2));
                x[i] = __builtin_bit_cast(V8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
            }
        };
        f16x s[2];
        constexpr f16x zero = {};
        read_k(ra, 0);
        wait_reads();
        read_k(rb, 1);
#pragma unroll
        for (int k = 0; k < KS; ++k) s[0] = Elem<DT>::mfma32(ra[k], qf[k], k == 0 ? zero : s[0]);
        wait_reads();
        read_v(ra, 0);
#pragma unroll
        for (int k = 0; k < KS; ++k) s[1] = Elem<DT>::mfma32(rb[k], qf[k], k == 0 ? zero : s[1]);
        __builtin_amdgcn_sched_barrier(0);
        float base[2] = {0.0f, 0.0f};                  // bias of a 32-key tile's first key; the others' are in near[]
        if constexpr (ALIBI)                           // to base 2, with the bias within the 32 keys
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                base[kt] = slope * (float)(j0 + 32 * kt + 4 * half - p);
#pragma unroll
                for (int i = 0; i < 16; ++i) s[kt][i] = __builtin_fmaf(s[kt][i], c, near[i]);
            }
        if (bad != 0 || j0 + TILE_KEYS > all_see) {    // some key of the tile is not for some row of the wave
            const int rel = min(p, tl.key_end - 1) - j0 - 4 * half;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    s[kt][i] = 32 * kt + 8 * (i / 4) + i % 4 <= rel && !(bad >> (2 * kt + i / 8) & 1) ? s[kt][i] : -INFINITY;
        }
        float mk[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int i = 0; i < 16; ++i) mk[kt] = fmaxf(mk[kt], s[kt][i]);
        float mx = ALIBI ? fmaxf(mk[0] + base[0], mk[1] + base[1]) : fmaxf(mk[0], mk[1]) * c;
        const f2 m2 = both_halves(mx);
        mx = fmaxf(m2[0], m2[1]);
        // An exponent is c s - m by one FMA, m the rounded product of a largest s (or s + base - m, likewise): up to half of m's last place off.  Where that is much,
        // products are rounded first (0 to 1.5 % of a call's time for asking).
        if (__builtin_expect(__any(mx - m > TOP + LAZY) || large, 0)) {
#pragma clang fp contract(off)
            const float mn = fmaxf(m, reference(mx, TOP)), alpha = __builtin_amdgcn_exp2f(m - (mn == -INFINITY ? 0.0f : mn));
            m = mn;
            l *= alpha;
#pragma unroll
            for (int d = 0; d < DTL; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= alpha;
            large = __any(__builtin_fabsf(m) >= LARGE_SCORE && m != -INFINITY);
            if (__builtin_expect(large, 0))
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[kt][i] = (ALIBI ? s[kt][i] + base[kt] : s[kt][i] * c) - (m == -INFINITY ? 0.0f : m);
        }
        const float ms = m == -INFINITY ? 0.0f : m, by = large ? 1.0f : c;
        const float from[2] = {large ? 0.0f : ms - base[0], large ? 0.0f : ms - base[1]};
        V8 pf[4];                                      // P^T operands of the four 16-key steps
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int i = 0; i < 16; i += 8) {
                u32x4 x;
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const float e0 = __builtin_amdgcn_exp2f(ALIBI ? s[kt][i + e] - from[kt] : __builtin_fmaf(s[kt][i + e], by, -from[kt]));
                    const float e1 = __builtin_amdgcn_exp2f(ALIBI ? s[kt][i + e + 1] - from[kt] : __builtin_fmaf(s[kt][i + e + 1], by, -from[kt]));
                    x[e / 2] = Elem<DT>::pack(e0, e1);
                    l = Elem<DT>::add_pair(x[e / 2], l);
                }
                pf[2 * kt + i / 8] = __builtin_bit_cast(V8, x);
            }
#pragma unroll
        for (int d0 = 0; d0 < DTL; d0 += 2) {
            V8 (&cur)[8] = (d0 & 2) ? rb : ra;
            wait_reads();
            if (d0 + 2 < DTL) read_v((d0 & 2) ? ra : rb, d0 + 2);
#pragma unroll
            for (int i = 0; i < 8; ++i) o[d0 + i / 4] = Elem<DT>::mfma32(cur[i], pf[i % 4], o[d0 + i / 4]);
        }
    }
    if (!active) return;
    if (__builtin_expect((odd_values[0] | odd_values[1] | odd_values[2] | odd_values[3]) != 0, 0))      // all written ahead of the last tile's barrier
#pragma unroll 1
        for (int j = max(TILE_KEYS * ks.begin, first_hidden & ~15); j < min(TILE_KEYS * ks.end, tl.key_end); ++j) {
            const uint16_t* row = odd_value_row<DT, D>(a, q, h, j);
            if (!row) continue;
#pragma unroll
            for (int d = 0; d < DTL; ++d)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const u32x2 x = *reinterpret_cast<const u32x2*>(row + 32 * d + 2 * i + 4 * half);
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[d][i + e] += odd_element<DT>(x[e / 2], e % 2, j <= p);
                }
        }
    const f2 l2 = both_halves(l);
    store_rows<DT, D>(a, tl, h, ks, tile_part<D>(a, ks, h, v, split), o, m, l2[0] + l2[1], wr0, tok, head);
}

template <int DT, int D, bool ALIBI, bool PAGED>
__global__ __launch_bounds__(256, 2) void tile_attention_kernel(AttnArgs a) { tile_block<DT, D, ALIBI, PAGED>(a, (int)blockIdx.x); }

// Both for a batch that may have sequences of either kind: the streaming kernel's workgroups, then the tile kernel's, which multiply while the others read.
// A launch of each / this one, us: two chunks of 512 beside 9 sequences that decode, 56 heads (8 K/V heads), biases, 74 / 67 with contexts of 100 to 6000, 125 / 117 with 900 to
// 6000; 250 with up to 2000 and one chunk, 64 heads (8), 150 / 143; 60 with up to 1000 and one chunk, 40 heads (40), 113 / 100; 4 with up to 800 and a chunk of 200, 32 heads
// (8), 23 / 16.  The tile kernel's workgroups first: 62 (contexts from 100), 210, 144, 15; by turns: 69, 193, 134, 15: streams that begin late end last.  With two column tiles the streaming kernel has more registers than two workgroups a compute unit leave: a launch of each.
template <int DT, int D, bool ALIBI>
__global__ __launch_bounds__(256, 2) void mixed_attention_kernel(AttnArgs stream, AttnArgs tile)
{
    const int streams = stream.workers / 4;
    if ((int)blockIdx.x < streams) stream_block<DT, D, 1, ALIBI>(stream, (int)blockIdx.x, *reinterpret_cast<ShareSmem*>(smem_raw));
    else tile_block<DT, D, ALIBI, true>(tile, (int)blockIdx.x - streams);
}

// Adds up the splits of a row tile and head (blockIdx.x), in order: a thread has four features of a row, a workgroup 1024 / D rows (blockIdx.y).  The loads of four
// splits are under way together.
template <int DT, int D>
__global__ __launch_bounds__(256) void tile_combine_kernel(AttnArgs a)
{
    constexpr int AHEAD = 4;
    const int h = (int)blockIdx.x / a.tiles, v = (int)blockIdx.x % a.tiles;
    Tile tl;
    if (!tile_of(a, v, &tl)) return;
    const KeySplit ks = key_split(tl.key_tiles, a.splits, a.least, 0);
    const int rr = (1024 / D) * (int)blockIdx.y + (int)threadIdx.x / (D / 4), f = 4 * ((int)threadIdx.x % (D / 4));
    if (ks.used == 1 || rr >= tl.n_rows) return;
    constexpr size_t SIZE = (size_t)TILE_ROWS_Q * (D + 2), ML = (size_t)TILE_ROWS_Q * D;
    const float* base = a.part + ((size_t)h * a.tiles + v) * a.splits * SIZE;
    float m = -INFINITY, l = 0.0f;
    f4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int k0 = 0; k0 < ks.used; k0 += AHEAD) {
        f2 ml[AHEAD];
        f4 o[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const float* ps = base + min(k0 + k, ks.used - 1) * SIZE;
            ml[k] = *reinterpret_cast<const f2*>(ps + ML + 2 * rr);
            o[k] = *reinterpret_cast<const f4*>(ps + (size_t)rr * D + f);
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            if (k0 + k >= ks.used) break;
            const float mn = fmaxf(m, ml[k][0]), ms = mn == -INFINITY ? 0.0f : mn, x = __builtin_amdgcn_exp2f(m - ms), y = __builtin_amdgcn_exp2f(ml[k][0] - ms);
            m = mn;
            l = l * x + ml[k][1] * y;
            sum = sum * x + o[k] * y;
        }
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    const int r = tl.row0 + rr, tok = r / a.group, head = h * a.group + r % a.group;
    const u32x2 x = {Elem<DT>::pack(sum[0] * inv, sum[1] * inv), Elem<DT>::pack(sum[2] * inv, sum[3] * inv)};
    *reinterpret_cast<u32x2*>(a.out + (size_t)(tl.q.first + tok) * a.heads * D + head * D + f) = x;
}

}  // namespace

// ---- host ------------------------------------------------------------------------------------------

// Room that the tile kernel's parts may take: its list has a place for each sequence, also for those that the streaming kernel does.
constexpr size_t MAX_PART_BYTES = (size_t)256 << 20;

// What a call launches: the streaming kernel, the tile kernel or, where a batch may have sequences of both kinds, both, in one launch if column tiles are single.
AttentionPlan attention_plan(const lpq_attn_cfg& c, bool paged, int n_seqs, int M, int max_q, int max_kv, int cus)
{
    AttentionPlan p{};
    const int group = c.n_heads / c.n_kv_heads;
    const int64_t most = (int64_t)std::min(max_q, M) * group;
    p.stream_tiles = 0;
    if (paged && most <= 2 * STREAM_ROWS) p.stream_tiles = most <= STREAM_ROWS ? 1 : 2;
    else if (paged && n_seqs > 1 && group <= 2 * STREAM_ROWS) p.stream_tiles = group <= STREAM_ROWS ? 1 : 2;
    p.tile = !(paged && most <= 2 * STREAM_ROWS);
    p.workers = 4 * STREAM_WAVES * cus;
    p.tiles = (int)tile_bound(M, group, n_seqs, TILE_ROWS_Q);
    p.splits = 1;
    if (p.tile) {
        // Workgroups that have rows, two to a compute unit: splits make one round of them, or two where the walks are long.  One round / two, us with the
        // combining kernel: 512 tokens of 32 heads (8 K/V heads) behind 8000 positions 80 / 83, behind 30000 240 / 223; of 40 heads (40) behind 4000 52 / 62; two
        // chunks of 512 beside 9 sequences that decode, 56 heads (8), up to 6000 positions 122 / 114.
        const int64_t wgs = std::max<int64_t>(1, ((int64_t)M * group + TILE_ROWS_Q - 1) / TILE_ROWS_Q) * c.n_kv_heads, slots = 2 * (int64_t)cus;
        const int64_t key_tiles = ((int64_t)max_kv + TILE_KEYS - 1) / TILE_KEYS;
        const int64_t fill = std::max<int64_t>(slots / wgs, std::min<int64_t>(2 * slots / wgs, key_tiles / LONG_KEY_TILES));
        p.splits = (int)std::max<int64_t>(1, std::min<int64_t>({fill, 16, key_tiles / LEAST_KEY_TILES}));
        const size_t split_bytes = (size_t)p.tiles * c.n_kv_heads * TILE_ROWS_Q * (c.head_dim + 2) * sizeof(float);
        p.splits = (int)std::max<size_t>(1, std::min<size_t>(p.splits, MAX_PART_BYTES / split_bytes));
        p.key_tiles = (int)key_tiles;
    }
    const size_t d2 = (size_t)c.head_dim + 2;
    if (p.stream_tiles) p.stream_floats = (size_t)p.workers * (2 * STREAM_ROWS * p.stream_tiles * d2 + sizeof(Cut) / sizeof(float));
    // lists of 32 parts and more, where the walks are long enough to be cut that often (4 sequences of up to 800 positions: long lists' form 7.2 us, the other's 4.0)
    p.long_lists = (int64_t)n_seqs * c.n_kv_heads * 32 <= p.workers && max_kv >= 64 * STREAM_KEYS;
    p.stream_rows = (int)std::min<int64_t>(STREAM_ROWS * p.stream_tiles, p.tile ? 2 * STREAM_ROWS : most);
    p.split_floats = (size_t)p.tiles * c.n_kv_heads * TILE_ROWS_Q * d2;
    return attention_plan_within(p, SIZE_MAX);
}

// The plan with partial results of at most `floats`: the streaming kernel's, whose room does not depend on the batch, go first, as a long walk that is not cut takes a
// hundred times as long there; the tile kernel makes as many splits as the rest has room for.
AttentionPlan attention_plan_within(AttentionPlan p, size_t floats)
{
    if (p.stream_floats > floats) p.stream_floats = 0;
    floats -= p.stream_floats;
    if (p.tile) p.splits = (int)std::max<size_t>(1, std::min<size_t>(p.splits, floats / p.split_floats));
    p.tile_floats = p.splits > 1 ? p.split_floats * p.splits : 0;
    p.least = std::max<int>(LEAST_KEY_TILES, (p.key_tiles + p.splits - 1) / p.splits);
    return p;
}

// LDS of a workgroup of the tile kernel: its tiles and a word per wave.  Allowed once per kernel and device where it is more than 64 KB.
constexpr size_t tile_lds(int d) { return (size_t)4 * TILE_KEYS * d * 2 + 4 * sizeof(uint32_t); }
template <auto KERNEL>
static hipError_t allow_lds(size_t bytes)
{
    static std::once_flag flags[64];
    static hipError_t results[64];
    int dev = 0;
    if (bytes <= 65536) return hipSuccess;
    const hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev < 0 || dev >= 64) return hipErrorInvalidDevice;
    std::call_once(flags[dev], [&] { results[dev] = hipFuncSetAttribute(reinterpret_cast<const void*>(KERNEL), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes); });
    return results[dev];
}

template <int DT, int D>
static hipError_t launch_attention(const AttentionPlan& p, const AttnArgs& a, float* part, hipStream_t s)
{
    const bool alibi = a.slopes != nullptr, both = p.stream_tiles && p.tile, mixed = both && p.stream_tiles == 1;
    const unsigned streams = (unsigned)p.workers / 4;
    AttnArgs st = a, tl = a;
    st.rows_from = 1;
    st.rows_to = both ? 2 * STREAM_ROWS + 1 : INT32_MAX;
    st.workers = p.workers;
    st.part = p.stream_floats ? part : nullptr;
    tl.rows_from = both ? 2 * STREAM_ROWS + 1 : 1;
    tl.rows_to = INT32_MAX;
    tl.tiles = p.tiles;
    tl.splits = p.splits;
    tl.least = p.least;
    tl.part = part + p.stream_floats;
    const int classes = a.kv_heads % 8 == 0 ? 1 : a.kv_heads % 4 == 0 ? 2 : a.kv_heads % 2 == 0 ? 4 : 8;
    const unsigned grid = (unsigned)(a.kv_heads * classes) * (unsigned)((p.tiles + classes - 1) / classes) * (unsigned)p.splits;
    constexpr size_t smem = tile_lds(D);
#define LPQ_ALIBI(KERNEL, GRID, SMEM, ...)                                                                              \
    do {                                                                                                                \
        if (alibi) KERNEL(true)<<<GRID, 256, SMEM, s>>>(__VA_ARGS__);                                                   \
        else       KERNEL(false)<<<GRID, 256, SMEM, s>>>(__VA_ARGS__);                                                  \
    } while (0)
#define LPQ_MIXED(A) mixed_attention_kernel<DT, D, A>
#define LPQ_STREAM1(A) stream_attention_kernel<DT, D, 1, A>
#define LPQ_STREAM2(A) stream_attention_kernel<DT, D, 2, A>
#define LPQ_TILE_PAGED(A) tile_attention_kernel<DT, D, A, true>
#define LPQ_TILE_PACKED(A) tile_attention_kernel<DT, D, A, false>
#define LPQ_ALLOW(KERNEL) (alibi ? allow_lds<&KERNEL(true)>(smem) : allow_lds<&KERNEL(false)>(smem))
    const hipError_t allowed = !p.tile ? hipSuccess : mixed ? LPQ_ALLOW(LPQ_MIXED) : a.kp ? LPQ_ALLOW(LPQ_TILE_PAGED) : LPQ_ALLOW(LPQ_TILE_PACKED);
    if (allowed != hipSuccess) return allowed;
    if (mixed) LPQ_ALIBI(LPQ_MIXED, streams + grid, smem, st, tl);
    else {
        if (p.stream_tiles == 1) LPQ_ALIBI(LPQ_STREAM1, streams, 0, st);
        else if (p.stream_tiles == 2) LPQ_ALIBI(LPQ_STREAM2, streams, 0, st);
        if (p.tile && a.kp) LPQ_ALIBI(LPQ_TILE_PAGED, grid, smem, tl);
        else if (p.tile) LPQ_ALIBI(LPQ_TILE_PACKED, grid, smem, tl);
    }
    if (st.part && p.stream_tiles) {
        const unsigned cuts = (unsigned)((p.workers + CUTS_PER_WG - 1) / CUTS_PER_WG), rows = (unsigned)p.stream_rows;
        if (p.stream_tiles == 1 && p.long_lists) stream_combine_kernel<DT, D, 1, true><<<dim3(cuts, rows * (D / 32)), 256, 0, s>>>(st);
        else if (p.stream_tiles == 1) stream_combine_kernel<DT, D, 1, false><<<dim3(cuts, rows), 256, 0, s>>>(st);
        else if (p.long_lists) stream_combine_kernel<DT, D, 2, true><<<dim3(cuts, rows * (D / 32)), 256, 0, s>>>(st);
        else stream_combine_kernel<DT, D, 2, false><<<dim3(cuts, rows), 256, 0, s>>>(st);
    }
    if (p.tile && p.splits > 1) tile_combine_kernel<DT, D><<<dim3((unsigned)(p.tiles * a.kv_heads), TILE_ROWS_Q * D / 1024), 256, 0, s>>>(tl);
    return hipGetLastError();
}

hipError_t launch_batch_attention(const AttentionPlan& p, const lpq_attn_cfg& c, const void* qkv, const void* kp, const void* vp, const int32_t* table,
                                  int shift, int n_pages, int max_pages, const int32_t* cu_q, const int32_t* kv_lens, const float* slopes, int n_seqs, int M,
                                  void* out, float* part, hipStream_t s)
{
    AttnArgs a{};
    a.qkv = static_cast<const uint16_t*>(qkv);
    a.kp = static_cast<const uint16_t*>(kp);
    a.vp = static_cast<const uint16_t*>(vp);
    a.table = table;
    a.cu_q = cu_q;
    a.kv_lens = kv_lens;
    a.slopes = slopes;
    a.out = static_cast<uint16_t*>(out);
    a.n_seqs = n_seqs;
    a.M = M;
    a.heads = c.n_heads;
    a.kv_heads = c.n_kv_heads;
    a.group = c.n_heads / c.n_kv_heads;
    a.shift = shift;
    a.n_pages = n_pages;
    a.max_pages = max_pages;
    if (c.dtype == LPQ_DT_FP16) return c.head_dim == 128 ? launch_attention<LPQ_DT_FP16, 128>(p, a, part, s) : launch_attention<LPQ_DT_FP16, 64>(p, a, part, s);
    return c.head_dim == 128 ? launch_attention<LPQ_DT_BF16, 128>(p, a, part, s) : launch_attention<LPQ_DT_BF16, 64>(p, a, part, s);
}

}  // namespace lpq

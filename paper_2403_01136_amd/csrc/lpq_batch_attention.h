// What the attention operators for batches of sequences of different lengths share: rows, pages and work of a sequence, the list of the streaming kernels' units
// and the kernel that adds up their parts, and the tile kernel with its combining kernel.
#pragma once
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
    const uint16_t *kp, *vp;             // pages (of either kind); null: keys are the rows themselves
    const int32_t *table, *cu_q, *kv_lens;
    const float* slopes;
    uint16_t* out;                       // [M][heads * D]
    float* part;                         // partial results, or null: nothing is split
    uint32_t group_reciprocal;           // 2^32 / group, at most 2^32 - 1
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

// ---- cells of 4 bits ------------------------------------------------------------------------------
// 16 positions of a head lie together: their codes, D / 2 bytes each, eight features to a word (code e at bit 4 (e / 2) + 16 (e % 2)), then a word of parameters
// for each: scale, zero.
template <int DT> __device__ __forceinline__ float param_scale(uint32_t p) { return (float)__builtin_bit_cast(typename Elem<DT>::t, (uint16_t)p); }
template <int DT> __device__ __forceinline__ float param_zero(uint32_t p) { return (float)__builtin_bit_cast(typename Elem<DT>::t, (uint16_t)(p >> 16)); }
__device__ __forceinline__ uint32_t and_or(uint32_t v, uint32_t mask, uint32_t bits)      // v & mask | bits, which the compiler makes two of
{
    uint32_t r;
    asm("v_and_or_b32 %0, %1, %2, %3" : "=v"(r) : "v"(v), "s"(mask), "v"(bits));
    return r;
}
// What a word of codes stands for, rounded once to the type; in bf16, which has no such instruction, to fp32 first.
template <int DT> __device__ __forceinline__ u32x4 cell_values(uint32_t w, uint32_t param)
{
    u32x4 x;
    if constexpr (DT == LPQ_DT_FP16) {                 // 1024 + code is an fp16 number with the code in its last bits
        const h2 p = as_h2(param), s = splat(p[0]), z = splat(p[1]), base = splat((_Float16)-1024.0f);
        uint32_t bias = 0x64006400u;
        asm("" : "+v"(bias));                          // in a register: of an instruction's operands one may be scalar
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = as_u32(pk_fma(as_h2(and_or(w >> (4 * e), 0x000f000fu, bias)) + base, s, z));
    } else {
        const float s = param_scale<DT>(param), z = param_zero<DT>(param);
        const uint32_t lo = w & 0x0f0f0f0fu, hi = w >> 4 & 0x0f0f0f0fu;          // bytes: features 0, 4, 1, 5 and 2, 6, 3, 7
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t b = e & 1 ? hi : lo;
            const int at = 8 * (e / 2);
            x[e] = Elem<DT>::pack(__builtin_fmaf((float)(b >> at & 255u), s, z), __builtin_fmaf((float)(b >> (at + 16) & 255u), s, z));
        }
    }
    return x;
}
// The four pairs of a word's codes as fp16 numbers without exponent, code * 2^-20.
__device__ __forceinline__ u32x4 code_pairs(uint32_t w)
{
    constexpr uint32_t M = 0x00f000f0u;
    return u32x4{w << 4 & M, w & M, w >> 4 & M, w >> 8 & M};
}
// Numbers of either type as fp16 ones that powers of two are taken out of.
__device__ __forceinline__ int exponent_of(float v)
{
    const int bits = (int)(__builtin_bit_cast(uint32_t, v) >> 23);
    return bits == 255 ? 0 : max(bits - 127, -100);
}
template <int DT> __device__ __forceinline__ float largest_of_pair(uint32_t pair, float top)
{
    return fmaxf(top, fmaxf(__builtin_fabsf(param_scale<DT>(pair)), __builtin_fabsf(param_zero<DT>(pair))));
}
template <int DT> __device__ __forceinline__ uint32_t scaled_pair(uint32_t pair, int ex0, int ex1)
{
    return Elem<LPQ_DT_FP16>::pack(__builtin_ldexpf(param_scale<DT>(pair), ex0), __builtin_ldexpf(param_zero<DT>(pair), ex1));
}
// A tile's values v are kept as v 2^-e in fp16, made from codes without exponent by scale * 2^(20 - e): e is the exponent of the largest of these numbers over its keys, which
// leaves the scales below 2^16 and the zeros below 2^15.  As bits of a number >= 0; what is not finite does not count.
template <int DT> __device__ __forceinline__ int cell_size(uint32_t param)
{
    const int bits = __builtin_bit_cast(int, fmaxf(__builtin_fabsf(param_scale<DT>(param)) * 32.0f, __builtin_fabsf(param_zero<DT>(param)) * 0x1p-14f));
    return not_finite<DT>(param) ? 0 : bits;
}
template <bool SCALED> __device__ __forceinline__ u32x4 tile_values(uint32_t w, uint32_t param)
{
    if constexpr (!SCALED) return cell_values<LPQ_DT_FP16>(w, param);
    const h2 p = as_h2(param), s = splat(p[0]), z = splat(p[1]);
    u32x4 x = code_pairs(w);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = as_u32(pk_fma(as_h2(x[e]), s, z));
    return x;
}
// Whether the values of key j of a sequence and K/V head are infinite or NaN (the same for the whole wave).
template <int DT, int D>
__device__ __forceinline__ bool odd_cell(const AttnArgs& a, const Seq& q, int h, int j)
{
    const int page = page_of_group(a, q.s, j >> 4);
    if (page < 0) return false;
    const uint8_t* b = reinterpret_cast<const uint8_t*>(a.vp) + cell_group(page, h, a.kv_heads, a.shift, (j >> 4) & ((1 << (a.shift - 4)) - 1), D);
    return not_finite<DT>(*reinterpret_cast<const uint32_t*>(b + 8 * D + 4 * (j & 15))) != 0;
}

// ---- the streaming kernels' work ----------------------------------------------------------------
constexpr int STREAM_WAVES = 1, CELL_WAVES = 2;          // waves a SIMD, of pages and of cells
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

// Adds up the parts of the row tiles that the entries of `cuts` name, 16 entries a workgroup; blockIdx.y: rows and, if LONG, slices of 32 features.  Many
// short lists of parts: a wave takes a row of a cut, D / 4 lanes of four features each for every (256 / D)-th part.  LONG, for few lists of hundreds of parts:
// the workgroup takes a slice, 8 lanes for every 32nd part, the sums added through LDS.  Either is right for any list.
template <int DT, int D, int TILE_ROWS, bool LONG>
__global__ __launch_bounds__(256) void stream_combine_kernel(AttnArgs a)
{
    constexpr int SLOT = TILE_ROWS * (D + 2), SLICES = LONG ? D / 32 : 1, LANES = D / SLICES / 4, WAYS = (LONG ? 256 : 64) / LANES;
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
template <int D> __device__ __forceinline__ int v_swizzle(int row) { return 4 * (D == 128 ? row & 3 : (row >> 1) & 1); }
// Values of cells are stored by 16 lanes of 16 rows and the same chunk: V's swizzle goes by the other bits of the row too, K's as it does.
template <int D> __device__ __forceinline__ int v_swizzle_cells(int row) { return v_swizzle<D>(row) + ((row >> 2) & 3); }

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

template <int DT, int D, bool ALIBI, int SRC>
__device__ __forceinline__ void tile_block(const AttnArgs& a, int block)
{
    // Products are of the rows' type; of cells in fp16 for either type, with tiles and queries of bf16 taken by powers of two.
    constexpr bool SCALED = SRC == SRC_CELLS && DT == LPQ_DT_BF16;
    // K of fp16 cells stays codes, whose products with a row get scale and zero behind them, as in the streaming kernel: rounded K puts 2.5e-4 of a result of ordinary scores into it,
    // V 2.0e-4, beside an output's rounding of 2.1e-4 (fp16) and 1.6e-3 (bf16).  It takes 6 % (two chunks of up to 512 tokens beside 9 sequences that decode, 56 heads over 8, biases:
    // 128.3 us; K rounded 120.8; parameters in LDS as fp32 products with c, twice the reads, 132.6).  V's values and the weights are rounded: 1.3 to 1.63 times an output's rounding over 60 batches.  V as codes
    // too, with weights times scales and what rounding takes from them as two operands, leaves the output's rounding alone, but takes 179 us there, and 738 for 523 of a chunk behind 6000 positions.
    constexpr bool K_CODES = SRC == SRC_CELLS && DT == LPQ_DT_FP16;
    constexpr int PT = SRC == SRC_CELLS ? (int)LPQ_DT_FP16 : DT;
    typedef typename Elem<PT>::v8 V8;
    constexpr int CH = D / 8, KS = D / 16, DTL = D / 32, ROWS = 512 / D, FILLS = 16 / ROWS;       // chunks of a row; feature steps; feature tiles; keys per load; loads of a wave's 16 keys
    constexpr int TILE_BYTES = TILE_KEYS * D * 2;
    constexpr bool PAGED = SRC != SRC_ROWS, CELLS = SRC == SRC_CELLS;
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
    float c = LOG2E / sqrtf((float)D);
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
    // cells: this wave's 16 keys of a tile as they lie, lane l has codes D / 4 (l / 16) .. of key l % 16, until place() puts their values in LDS
    typedef uint32_t codes_t __attribute__((ext_vector_type(D / 32)));
    codes_t kcodes = {}, vcodes = {};
    uint32_t kparam = 0, vparam = 0;
    // asks for tile j; which of its 16-key groups have no page
    auto fetch = [&](int j) -> uint32_t {
        if ((uint32_t)(j - ids_from) >= 16u) load_ids(j);
        const int id = max(__builtin_amdgcn_readlane(ids, 4 * (j - ids_from) + wave), 0);
        const size_t at = (size_t)cell_group(id, h, a.kv_heads, a.shift, (4 * j + wave) & ((1 << (a.shift - 4)) - 1), D);
        const uint8_t *kb = reinterpret_cast<const uint8_t*>(a.kp) + at, *vb = reinterpret_cast<const uint8_t*>(a.vp) + at;
        kcodes = *reinterpret_cast<const codes_t*>(kb + (lane & 15) * (D / 2) + (lane >> 4) * (D / 8));
        kparam = *reinterpret_cast<const uint32_t*>(kb + 8 * D + 4 * (lane & 15));
        vcodes = *reinterpret_cast<const codes_t*>(vb + (lane & 15) * (D / 2) + (lane >> 4) * (D / 8));
        vparam = *reinterpret_cast<const uint32_t*>(vb + 8 * D + 4 * (lane & 15));
        return (uint32_t)(bad_ids >> (4 * (j - ids_from))) & 15u;
    };
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
    float qsum = 0.0f;                                 // K_CODES: the sum of the row, in steps of the codes
    {
        const uint16_t* qp = a.qkv + (size_t)(q.first + tok) * cols + head * D + 8 * half;
#pragma unroll
        for (int k = 0; k < KS; ++k) qf[k] = *reinterpret_cast<const V8*>(qp + 16 * k);
        if constexpr (SCALED) {
            uint32_t pairs[4 * KS];
#pragma unroll
            for (int k = 0; k < 4 * KS; ++k) pairs[k] = __builtin_bit_cast(u32x4, qf[k / 4])[k % 4];
            float top = 0.0f;
#pragma unroll
            for (int k = 0; k < 4 * KS; ++k) top = largest_of_pair<DT>(pairs[k], top);
            const f2 z = both_halves(top);
            const int ex = exponent_of(fmaxf(z[0], z[1])) - 14;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                u32x4 x;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = scaled_pair<DT>(pairs[4 * k + e], -ex, -ex);
                qf[k] = __builtin_bit_cast(V8, x);
            }
            c = __builtin_ldexpf(c, ex);
        }
        if constexpr (K_CODES) {
#pragma unroll
            for (int k = 0; k < 4 * KS; ++k) qsum = Elem<PT>::add_pair(__builtin_bit_cast(u32x4, qf[k / 4])[k % 4], qsum);
            const f2 z = both_halves(qsum);
            qsum = (z[0] + z[1]) * 0x1p-20f;
            c *= 0x1p20f;
        }
    }
    f16x o[DTL];
#pragma unroll
    for (int d = 0; d < DTL; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
    float m = -INFINITY, l = 0.0f;                     // the maximum in use of the lane's row; this lane's part of its sum
    constexpr int TOP = Elem<PT>::TOP ? Elem<PT>::TOP - LAZY : 0;
    bool large = false;                                // the maximum of some row of the wave is
    // operand reads, bytes within a buffer
    uint32_t ka[KS], va[DTL];
#pragma unroll
    for (int k = 0; k < KS; ++k) ka[k] = (uint32_t)(col * D * 2 + 16 * ((2 * k + half) ^ k_swizzle<D>(col)));
#pragma unroll
    for (int d = 0; d < DTL; ++d) {
        const int row = 4 * half + (lane & 15) / 4, chunk = 4 * d + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
        va[d] = (uint32_t)(2 * TILE_BYTES + row * D * 2 + 16 * (chunk ^ (CELLS ? v_swizzle_cells<D>(row) : v_swizzle<D>(row))) + 8 * (lane & 1));
    }

    // keys from here on are not seen by every row of the tile; and whether a wave has set values of theirs to zero, in LDS behind the tiles
    const int first_hidden = min(tl.key_end, q.pos0 + tl.row0 / a.group + 1);
    uint32_t* const odd_values = reinterpret_cast<uint32_t*>(smem_raw + 4 * TILE_BYTES);
    if (lane == 0) odd_values[wave] = 0;

    float near[ALIBI ? 16 : 1];                        // bias of a register's key within its 32; K_CODES: over c
    if constexpr (ALIBI) {
        const float per_key = K_CODES ? slope / c : slope;
#pragma unroll
        for (int i = 0; i < 16; ++i) near[i] = per_key * (float)(8 * (i / 4) + i % 4);
    }

    // Cells: tile j's parameters have landed.  Keys that no row sees get none (values of zero, like their weights; K's scores are replaced); and, in
    // bf16, the largest of K's and of V's among the wave's keys for all waves.
    int* const tops = reinterpret_cast<int*>(smem_raw + 4 * TILE_BYTES + 16);    // [n % 2][K, V][wave]
    auto look = [&](int j, int buf, uint32_t no_page) {
        if ((no_page >> wave & 1) || TILE_KEYS * j + 16 * wave + (lane & 15) >= tl.key_end) kparam = vparam = 0;
        if constexpr (!SCALED) return;
        int kt = cell_size<DT>(kparam), vt = cell_size<DT>(vparam);
        auto step = [&](auto ctrl) {
            kt = max(kt, __builtin_amdgcn_update_dpp(0, kt, decltype(ctrl)::value, 0xf, 0xf, true));
            vt = max(vt, __builtin_amdgcn_update_dpp(0, vt, decltype(ctrl)::value, 0xf, 0xf, true));
        };
        step(std::integral_constant<int, 0xB1>());
        step(std::integral_constant<int, 0x4E>());
        step(std::integral_constant<int, 0x141>());
        step(std::integral_constant<int, 0x140>());
        if (lane == 0) {
            tops[8 * buf + wave] = kt;
            tops[8 * buf + 4 + wave] = vt;
        }
    };
    uint32_t* const kparams = reinterpret_cast<uint32_t*>(smem_raw + 4 * TILE_BYTES + 80);       // K_CODES: [n % 2][key]
    int k_ex = 0, v_ex = -200, k_ex_next = 0, v_ex_next = -200;                 // the tile's K is taken by 2^-k_ex, its V and the sums by 2^-v_ex
    // the values of the cells into LDS
    auto place = [&](int j, int buf) {
        const int row = 16 * wave + (lane & 15), key = TILE_KEYS * j + row;
        if (key >= first_hidden && __any(not_finite<DT>(vparam) != 0)) {         // not every row sees it: its values may not be infinite or NaN
            if (not_finite<DT>(vparam) != 0) vparam = 0;
            odd_values[wave] = 1;
        }
        uint32_t kp = kparam, vp = vparam;
        if constexpr (SCALED) {
            typedef int i32x4 __attribute__((ext_vector_type(4)));
            const i32x4 kt = *reinterpret_cast<const i32x4*>(tops + 8 * buf), vt = *reinterpret_cast<const i32x4*>(tops + 8 * buf + 4);
            k_ex_next = exponent_of(__builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(max(max(kt[0], kt[1]), max(kt[2], kt[3])))));
            v_ex_next = max(v_ex_next, exponent_of(__builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(max(max(vt[0], vt[1]), max(vt[2], vt[3]))))));
            kp = scaled_pair<DT>(kparam, 20 - k_ex_next, -k_ex_next);
            vp = scaled_pair<DT>(vparam, 20 - v_ex_next, -v_ex_next);
        }
        if (K_CODES && lane < 16) kparams[TILE_KEYS * buf + row] = kp;
        uint8_t *kr = smem_raw + buf * TILE_BYTES + row * D * 2, *vr = kr + 2 * TILE_BYTES;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
            const int chunk = (D / 32) * (lane >> 4) + i;
            *reinterpret_cast<u32x4*>(kr + 16 * (chunk ^ k_swizzle<D>(row))) = K_CODES ? code_pairs(kcodes[i]) : tile_values<SCALED>(kcodes[i], kp);
            *reinterpret_cast<u32x4*>(vr + 16 * (chunk ^ v_swizzle_cells<D>(row))) = tile_values<SCALED>(vcodes[i], vp);
        }
    };

    const int tiles = ks.end - ks.begin, j_first = BACKWARD ? ks.end - 1 : ks.begin;
    constexpr int STEP = BACKWARD ? -1 : 1;
    if constexpr (PAGED) load_ids(j_first);
    uint32_t bad = 0, bad_next = 0, bad_asked = 0;
    if constexpr (CELLS) {
        bad_next = fetch(j_first);
        look(j_first, 0, bad_next);
        if constexpr (SCALED) __syncthreads();
        place(j_first, 0);
        if (tiles > 1) bad_asked = fetch(j_first + STEP);
    } else bad_next = fill(j_first, 0);
    for (int n = 0; n < tiles; ++n) {
        const int j = j_first + STEP * n, buf = n & 1, j0 = TILE_KEYS * j;
        bad = bad_next;
        if constexpr (CELLS) {
            k_ex = k_ex_next;
            if (SCALED && v_ex_next > v_ex) {
                const float by = __builtin_ldexpf(1.0f, v_ex - v_ex_next);
#pragma unroll
                for (int d = 0; d < DTL; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[d][i] *= by;
                v_ex = v_ex_next;
            }
            if (n + 1 < tiles) look(j + STEP, buf ^ 1, bad_asked);
        } else __builtin_amdgcn_s_waitcnt(0x0F70);     // vmcnt(0): this wave's part of tile j has landed
        if (!CELLS && (bad != 0 || j0 + TILE_KEYS > tl.key_end)) {               // values of keys that no row sees: zero, like their weights
#pragma unroll
            for (int i = 0; i < FILLS; ++i) {
                const int row = 16 * wave + ROWS * i + lane / CH;
                if ((bad >> wave & 1) || j0 + row >= tl.key_end) *reinterpret_cast<u32x4*>(smem_raw + 2 * TILE_BYTES + buf * TILE_BYTES + (16 * wave + ROWS * i) * D * 2 + 16 * lane) = u32x4{};
            }
        }
        if (!CELLS && j0 + 16 * wave + 16 > first_hidden && first_hidden < tl.key_end) {      // the wave's keys are not seen by every row: none of their values may be infinite or NaN
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
        if constexpr (CELLS) {
            if (n + 1 < tiles) {
                bad_next = bad_asked;
                place(j + STEP, buf ^ 1);
                if (n + 2 < tiles) bad_asked = fetch(j + 2 * STEP);
            }
        } else if (n + 1 < tiles) bad_next = fill(j + STEP, buf ^ 1);
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
                const uint8_t* at8 = CELLS ? tile + (va[d0 + i / 4] ^ 32u) + 16 * (i % 4) * D * 2 : at;          // eight rows on: another swizzle
                const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_t)at), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_t)(at8 + 8 * D * 2));
                x[i] = __builtin_bit_cast(V8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
            }
        };
        f16x s[2];
        constexpr f16x zero = {};
        read_k(ra, 0);
        wait_reads();
        read_k(rb, 1);
#pragma unroll
        for (int k = 0; k < KS; ++k) s[0] = Elem<PT>::mfma32(ra[k], qf[k], k == 0 ? zero : s[0]);
        wait_reads();
        read_v(ra, 0);
#pragma unroll
        for (int k = 0; k < KS; ++k) s[1] = Elem<PT>::mfma32(rb[k], qf[k], k == 0 ? zero : s[1]);
        __builtin_amdgcn_sched_barrier(0);
        // Finite and not zero, whatever the powers of two (a row of zeros over keys of zeros): scores that are masked are -inf times it.  Sums of products are below 2^38.
        const float ct = SCALED ? __builtin_amdgcn_fmed3f(__builtin_ldexpf(c, k_ex), 0x1p-126f, 0x1.fffffep127f) : c;
        if constexpr (K_CODES)                         // by instructions that take the parameters as they are
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const u32x4 par = *reinterpret_cast<const u32x4*>(kparams + TILE_KEYS * buf + 32 * kt + 2 * i + 4 * half);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        s[kt][i + e] = __builtin_fmaf(param_scale<DT>(par[e]), s[kt][i + e], __builtin_fmaf(param_zero<DT>(par[e]), qsum, ALIBI ? near[ALIBI ? i + e : 0] : 0.0f));
                }
        float base[2] = {0.0f, 0.0f};                  // bias of a 32-key tile's first key; the others' are in near[]
        if constexpr (ALIBI)                           // to base 2, with the bias within the 32 keys
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                base[kt] = slope * (float)(j0 + 32 * kt + 4 * half - p);
#pragma unroll
                for (int i = 0; i < 16 && !K_CODES; ++i) s[kt][i] = __builtin_fmaf(s[kt][i], ct, near[i]);
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
        constexpr bool BASE_2 = ALIBI && !K_CODES;     // s is, with the bias
        float mx = BASE_2 ? fmaxf(mk[0] + base[0], mk[1] + base[1]) : ALIBI ? fmaxf(__builtin_fmaf(mk[0], ct, base[0]), __builtin_fmaf(mk[1], ct, base[1])) : fmaxf(mk[0], mk[1]) * ct;
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
                    for (int i = 0; i < 16; ++i) s[kt][i] = ((BASE_2 ? s[kt][i] : s[kt][i] * ct) + base[kt]) - (m == -INFINITY ? 0.0f : m);
        }
        const float ms = m == -INFINITY ? 0.0f : m, by = large ? 1.0f : ct;
        const float from[2] = {large ? 0.0f : ms - base[0], large ? 0.0f : ms - base[1]};
        V8 pf[4];                                      // P^T operands of the four 16-key steps
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int i = 0; i < 16; i += 8) {
                u32x4 x;
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const float e0 = __builtin_amdgcn_exp2f(BASE_2 ? s[kt][i + e] - from[kt] : __builtin_fmaf(s[kt][i + e], by, -from[kt]));
                    const float e1 = __builtin_amdgcn_exp2f(BASE_2 ? s[kt][i + e + 1] - from[kt] : __builtin_fmaf(s[kt][i + e + 1], by, -from[kt]));
                    x[e / 2] = Elem<PT>::pack(e0, e1);
                    l = Elem<PT>::add_pair(x[e / 2], l);
                }
                pf[2 * kt + i / 8] = __builtin_bit_cast(V8, x);
            }
#pragma unroll
        for (int d0 = 0; d0 < DTL; d0 += 2) {
            V8 (&cur)[8] = (d0 & 2) ? rb : ra;
            wait_reads();
            if (d0 + 2 < DTL) read_v((d0 & 2) ? ra : rb, d0 + 2);
#pragma unroll
            for (int i = 0; i < 8; ++i) o[d0 + i / 4] = Elem<PT>::mfma32(cur[i], pf[i % 4], o[d0 + i / 4]);
        }
    }
    if (!active) return;
    if constexpr (SCALED) {
        const float by = __builtin_ldexpf(1.0f, v_ex);
#pragma unroll
        for (int d = 0; d < DTL; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] *= by;
    }
    if (__builtin_expect((odd_values[0] | odd_values[1] | odd_values[2] | odd_values[3]) != 0, 0))      // all written ahead of the last tile's barrier
#pragma unroll 1
        for (int j = max(TILE_KEYS * ks.begin, first_hidden & ~15); j < min(TILE_KEYS * ks.end, tl.key_end); ++j) {
            if constexpr (CELLS) {                     // NaN all of it, as the append stores what is not finite
                if (odd_cell<DT, D>(a, q, h, j) && j <= p)
#pragma unroll
                    for (int d = 0; d < DTL; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[d][i] = __builtin_nanf("");
                continue;
            }
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

// LDS of a workgroup of the tile kernel: its tiles, a word per wave, and for cells the largest values and K's parameters of two tiles.  Allowed once per kernel and device where it is more than 64 KB.
constexpr size_t tile_lds(int d, bool cells) { return (size_t)4 * TILE_KEYS * d * 2 + (cells ? 20 + 2 * TILE_KEYS : 4) * sizeof(uint32_t); }
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

// Launches a plan with the kernels of Family: mixed, stream and tile, and tile_rows for packed rows.
template <typename Family, int DT, int D>
hipError_t launch_attention(const AttentionPlan& p, const AttnArgs& a, float* part, hipStream_t s)
{
    const bool alibi = a.slopes != nullptr, both = p.stream_tile && p.tile, mixed = both && p.stream_tile <= STREAM_ROWS;
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
    constexpr size_t smem = tile_lds(D, Family::CELLS);
    // with biases or without
    auto launch = [&](auto plain, auto biased, unsigned blocks, size_t lds, const auto&... args) {
        if (alibi) biased<<<blocks, 256, lds, s>>>(args...);
        else plain<<<blocks, 256, lds, s>>>(args...);
    };
    const hipError_t allowed = !p.tile ? hipSuccess : alibi ? Family::template allow<DT, D, true>(mixed, p.stream_tile, a.kp != nullptr, smem)
                                                            : Family::template allow<DT, D, false>(mixed, p.stream_tile, a.kp != nullptr, smem);
    if (allowed != hipSuccess) return allowed;
    auto streaming = [&](auto rows) {                  // what is launched with a streaming kernel whose tiles have this many rows
        constexpr int ROWS = decltype(rows)::value;
        if constexpr (Family::template has<ROWS>) {
            if constexpr (Family::template has_mixed<ROWS>)
                if (mixed) launch(Family::template mixed<DT, D, ROWS, false>, Family::template mixed<DT, D, ROWS, true>, streams + grid, smem, st, tl);
            if (!mixed) launch(Family::template stream<DT, D, ROWS, false>, Family::template stream<DT, D, ROWS, true>, streams, 0, st);
            if (!st.part) return;
            const unsigned per = Family::cuts_per_wg(p.long_lists), cuts = ((unsigned)p.workers + per - 1) / per, n = (unsigned)p.stream_rows;
            if (p.long_lists) Family::template combine<DT, D, ROWS, true><<<Family::CELLS ? dim3(n * (D / 32), cuts) : dim3(cuts, n * (D / 32)), 256, 0, s>>>(st);
            else Family::template combine<DT, D, ROWS, false><<<dim3(cuts, n), 256, 0, s>>>(st);
        }
    };
    if (p.tile && !mixed && a.kp) launch(Family::template tile<DT, D, false>, Family::template tile<DT, D, true>, grid, smem, tl);
    if constexpr (Family::ROWS)
        if (p.tile && !a.kp) launch(Family::template tile_rows<DT, D, false>, Family::template tile_rows<DT, D, true>, grid, smem, tl);
    switch (p.stream_tile) {
    case 4: streaming(std::integral_constant<int, 4>()); break;
    case 8: streaming(std::integral_constant<int, 8>()); break;
    case 16: streaming(std::integral_constant<int, 16>()); break;
    case 32: streaming(std::integral_constant<int, 32>()); break;
    }
    if (p.tile && p.splits > 1) tile_combine_kernel<DT, D><<<dim3((unsigned)(p.tiles * a.kv_heads), TILE_ROWS_Q * D / 1024), 256, 0, s>>>(tl);
    return hipGetLastError();
}

template <typename Family>
hipError_t launch_attention_of(const AttentionPlan& p, const lpq_attn_cfg& c, const AttentionBatch& b, float* part, hipStream_t s)
{
    AttnArgs a{};
    a.qkv = static_cast<const uint16_t*>(b.qkv);
    a.kp = static_cast<const uint16_t*>(b.kp);
    a.vp = static_cast<const uint16_t*>(b.vp);
    a.table = b.table;
    a.cu_q = b.cu_q;
    a.kv_lens = b.kv_lens;
    a.slopes = b.slopes;
    a.out = static_cast<uint16_t*>(b.out);
    a.n_seqs = b.n_seqs;
    a.M = b.M;
    a.heads = c.n_heads;
    a.kv_heads = c.n_kv_heads;
    a.group = c.n_heads / c.n_kv_heads;
    a.group_reciprocal = (uint32_t)std::min<uint64_t>(UINT32_MAX, ((uint64_t)1 << 32) / (uint32_t)a.group);
    a.shift = b.shift;
    a.n_pages = b.n_pages;
    a.max_pages = b.max_pages;
    if (c.dtype == LPQ_DT_FP16) return c.head_dim == 128 ? launch_attention<Family, LPQ_DT_FP16, 128>(p, a, part, s) : launch_attention<Family, LPQ_DT_FP16, 64>(p, a, part, s);
    return c.head_dim == 128 ? launch_attention<Family, LPQ_DT_BF16, 128>(p, a, part, s) : launch_attention<Family, LPQ_DT_BF16, 64>(p, a, part, s);
}

}  // namespace

}  // namespace lpq

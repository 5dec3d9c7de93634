// Causal attention of new tokens over pages of 4-bit cells:
//     out[row] = sum_j w_j v_j / sum_j w_j,   w_j = exp(q . k_j / sqrt(D) + slope (j - p)),   j <= p,   k_j = s_j c_j + z_j, v_j = s'_j c'_j + z'_j
// with codes c of 0 to 15 for each feature and a scale and a zero for each key and head.  Rows, work lists, splits and the joining of parts are those of the
// 16-bit caches' kernels.  The tile kernel (prompts and chunks) is theirs too, with codes or values made from the cells on their way into LDS.
//
// The streaming kernel multiplies the codes themselves: scale and zero are one number each for a key, so
//     q . k_j        = s_j (q . c_j) + z_j sum(q)
//     sum_j w_j v_jf = sum_j (w_j s'_j) c'_jf + sum_j w_j z'_j
// where the first sum of each is the matrix units' and the others cost two operations a score.  A code in bits 4 to 7 of an fp16 number without exponent is that number,
// code * 2^-20: unpacking a word of eight takes three shifts and four ANDs, for queries of either type: those in bf16 are taken by a power of two for each row, which changes
// none of their eight bits that count.  Codes are exact; what is rounded are the weights w s', to fp16 beside a largest of 2^12 or more.  What that takes from them is multiplied as well, in columns
// that tiles of up to 8 rows leave idle (16 sequences of 40 heads 18.6 us for 18.4 without, 61 of 64 heads over 8 35.8 for 35.4), in fp16 also by second products of larger tiles (24 drafts 31.6 us for
// 29.7): an error of 2.1e-4 of a result in fp16, all of it the output's rounding, for 2.7e-4 to 3.2e-4 without.  Larger tiles in bf16, whose outputs are rounded at 1.66e-3, would take as much for 1.67e-3:
// there it is added up in 32 bits and counts as for a code of 8, so that only the codes' distance from it sees the rounding.
#include <algorithm>

#include "lpq_batch_attention.h"

namespace lpq {

namespace {

// ---- streaming kernel -----------------------------------------------------------------------------
// Bound by the memory while it streams, D + 8 bytes per key and K/V head; by starts and ends of walks where they are short.  Workers are single waves, two a SIMD (the 32-row tile, with
// its registers, one), with equal shares of the list of 32-key steps; the loads of one step are under way while the step before is computed.  61 sequences of 100 to 7000 positions, 64 heads (8 K/V heads),
// bf16, 30.0 us and 4.7 for the parts (112 MB; 3.7 TB/s, with some 8 us of start and end in it); one of 90001, 56 heads (8), fp16 25.7 and 4.8; 16 of 400 to 700, 40 heads 14.8 and 3.9; one wave
// a SIMD 62 for the first, three 41.
// Products on 16x16x32, columns = rows of the problem:
//   S^T = C_k . Q^T  lane (i = lane % 16, q = lane / 16) holds codes D / 4 q .. of key i as they lie; a word makes an operand of four pairs, of neighbours, as the query's row has them.
//                    Register r of the result: key 4 q + r, column i.
//   O^T = C_v^T . P^T over 32 keys: quarter q contracts over its own keys {4 q + 0..3, 16 + 4 q + 0..3}.  A lane has a word (D = 128; half a word, D = 64) of each of the
//                    eight; halves of two keys' words are put side by side, and what makes pairs of a word's neighbours makes a pair of keys of one feature.
// A tile of 4 or 8 rows has its columns four times or twice: each copy scores all keys and does the softmax of its part of them (16 columns doing all of it: 50.9 us for the first case where this
// took 47.1, both before other steps).
// Weights: P = exp2(score - m), its sum and its sum with the zeros in fp32; t = P s' is taken by a power of two G for each column so that the largest so far is below 2^15.
// G is renewed where t G passes 2^15, to a largest of 2^12 to 2^13 (2^8, 2^10, 2^14: 24 drafts 29.7, 29.6, 31.2 us for 30.4).  m is renewed where t passes 2^60, or the sum of a lane's P of a step
// 2^40: t alone says nothing of P where s' is zero (a flat head) or tiny.  That sum is made for l anyway.  Sums of P and of P z' are then in range for z' up to 2^64 and 2^23 keys.
// (2^24, 2^40, 2^60 and nothing asked: 24 drafts with biases 34.4, 33.8, 33.5, 33.3 us; without biases 30.3 to 30.5, 30.1.)
constexpr float LARGEST_T = 0x1p15f, NEW_T = 0x1p12f, RENEW_T = 0x1p60f, RENEW_P = 0x1p40f;

// v <- op(v, v of the lanes that have the same row): the four quarters, and where a tile has 8 or 4 rows the columns that are 8 or 4 apart.
template <int ROWS, typename Op>
__device__ __forceinline__ float over_row(float v, Op op)
{
    if constexpr (ROWS <= 4) v = op(v, dpp_move<0x124>(v));                      // row_ror
    if constexpr (ROWS <= 8) v = op(v, dpp_move<0x128>(v));
    f2 z = both_rows(v);
    z = both_halves(op(z[0], z[1]));
    return op(z[0], z[1]);
}

// ---- the list: walks (sequence, K/V head, row tile) of 32-key steps, with WALK_COST units ahead of each for what its start and end take; a share's worker needs no
// other wave to find it (0, 3, 6 units: 61 sequences 42.8, 36.8, 37.1 us, 24 drafts 35.2, 30.7, 29.8).  Lanes have 64 sequences side by side.
constexpr int WALK_COST = 3;
__device__ __forceinline__ int64_t read_lane64(int64_t v, int lane)
{
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, lane));
}
__device__ __forceinline__ int64_t last_lane64(int64_t v) { return read_lane64(v, 63); }
template <int CTRL, int ROW_MASK> __device__ __forceinline__ int64_t add_from(int64_t v)      // v + another lane's, or + 0 where there is none
{
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROW_MASK, 0xf, false), hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(v >> 32), CTRL, ROW_MASK, 0xf, false);
    return v + (int64_t)((uint64_t)hi << 32 | lo);
}
struct SeqLanes { int base, first, len, pos0, ctx; int64_t units, upto; };       // sequences base + lane; units, and those up to and with this lane's
template <int ROWS> __device__ __forceinline__ SeqLanes seq_lanes(const AttnArgs& a, int base)
{
    const int s = base + (int)(threadIdx.x & 63);
    SeqLanes r{base, 0, 0, 0, 0, 0, 0};
    if (s < a.n_seqs) {
        const Seq q = load_seq(a, s);
        r.first = q.first;
        r.len = q.len;
        r.pos0 = q.pos0;
        r.ctx = q.ctx;
        if (takes(a, q.rows)) r.units = (int64_t)a.kv_heads * stream_row_tiles(q.rows, ROWS) * (stream_key_steps(q.ctx) + WALK_COST);
    }
    int64_t v = r.units;
    v = add_from<0x111, 0xf>(v);                       // row_shr by 1, 2, 4, 8; row_bcast 15, 31
    v = add_from<0x112, 0xf>(v);
    v = add_from<0x114, 0xf>(v);
    v = add_from<0x118, 0xf>(v);
    v = add_from<0x142, 0xa>(v);
    r.upto = add_from<0x143, 0xc>(v);
    return r;
}
// r / group: the product with the reciprocal's 32 bits is at most one below.
__device__ __forceinline__ int over_group(const AttnArgs& a, int r)
{
    const uint32_t n = (uint32_t)r, q = __umulhi(n, a.group_reciprocal);
    return (int)(n - q * (uint32_t)a.group >= (uint32_t)a.group ? q + 1 : q);
}

template <int DT, int D, int ROWS, bool ALIBI>
__device__ __forceinline__ void stream4_block(const AttnArgs& a, int block)
{
    constexpr int W = D / 32, F = D / 16;                                        // words of a lane's codes of a key; its features of V
    constexpr int NT = ROWS == 32 ? 2 : 1, PARTS = ROWS < 16 ? 16 / ROWS : 1, N = 8 / PARTS;     // column tiles; parts of the keys; a lane's keys of a step
    constexpr int SLOT = ROWS * (D + 2);
    constexpr bool FINE = DT == LPQ_DT_FP16 || PARTS > 1, SECOND = FINE && PARTS == 1;           // what rounding takes from weights is multiplied: in idle columns, or by products of its own
    typedef uint32_t kcodes_t __attribute__((ext_vector_type(W)));
    typedef uint32_t params_t __attribute__((ext_vector_type(N < 4 ? N : 4)));
    typedef std::conditional_t<D == 128, uint32_t, uint16_t> vcodes_t;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, quarter = lane >> 4, part = PARTS > 1 ? col / ROWS : 0;
    const int cols = (a.heads + 2 * a.kv_heads) * D, group_mask = (1 << (a.shift - 4)) - 1;

    // this wave's share of the list
    SeqLanes seqs;
    const int w = __builtin_amdgcn_readfirstlane(4 * block + wave);
    int64_t total = 0;
    for (int base = 0; base < a.n_seqs; base += 64) {
        seqs = seq_lanes<ROWS>(a, base);
        total += last_lane64(seqs.upto);
    }
    const int workers = (int)min<int64_t>(a.workers, total);
    const int64_t share_u = w < workers ? uniform64(stream_begin(total, w, workers)) : 0, share_end = w < workers ? uniform64(stream_begin(total, w + 1, workers)) : 0;
    int64_t u = share_u, s_begin = 0, s_units = 0;     // where the share goes on; of the sequence at hand: its first unit, its units
    int at_lane = -1;
    Cut cut{0, 0, 0, 0};
    if (u < share_end) {                               // the sequence that has unit u
        int64_t carry = 0;
        for (int base = 0; base < a.n_seqs; base += 64) {
            if (a.n_seqs > 64) seqs = seq_lanes<ROWS>(a, base);
            const int64_t before = carry + seqs.upto - seqs.units;
            const uint64_t found = __ballot(u >= before && u < before + seqs.units);
            if (found) {
                at_lane = __builtin_ctzll(found);
                s_begin = read_lane64(before, at_lane);
                s_units = read_lane64(seqs.units, at_lane);
                break;
            }
            carry += last_lane64(seqs.upto);
        }
        if (at_lane < 0) u = share_end;                // lengths that change under the kernel
    }

    while (u < share_end) {
        if (u >= s_begin + s_units) {                  // the next sequence with units: there is one, u is below the total
            s_begin += s_units;
            uint64_t left = __ballot(seqs.units > 0) & (at_lane == 63 ? 0 : ~0ull << (at_lane + 1));
            while (!left && seqs.base + 64 < a.n_seqs) {
                seqs = seq_lanes<ROWS>(a, seqs.base + 64);
                left = __ballot(seqs.units > 0);
            }
            if (!left) break;                          // lengths that change under the kernel
            at_lane = __builtin_ctzll(left);
            s_units = read_lane64(seqs.units, at_lane);
        }
        const int s = seqs.base + at_lane;
        Seq q;
        q.s = s;
        q.first = __builtin_amdgcn_readlane(seqs.first, at_lane);
        q.len = __builtin_amdgcn_readlane(seqs.len, at_lane);
        q.pos0 = __builtin_amdgcn_readlane(seqs.pos0, at_lane);
        q.ctx = __builtin_amdgcn_readlane(seqs.ctx, at_lane);
        q.rows = q.len * a.group;
        const int steps = stream_key_steps(q.ctx), tiles = stream_row_tiles(q.rows, ROWS);
        const int64_t at = u - s_begin, tile = at >> 31 ? at / (steps + WALK_COST) : (int64_t)__builtin_amdgcn_readfirstlane((uint32_t)at / (uint32_t)(steps + WALK_COST));
        const int64_t first = s_begin + tile * (steps + WALK_COST) + WALK_COST;  // the walk's first step that is one
        const int h = tiles == 1 ? (int)tile : (int)((uint32_t)tile / (uint32_t)tiles), rt = tiles == 1 ? 0 : (int)((uint32_t)tile % (uint32_t)tiles);
        if (share_end <= first || (!a.part && first < share_u)) {      // the share ends ahead of it; nowhere to leave parts: a worker takes the row tiles that begin in its share, whole
            u = share_end <= first ? share_end : first + steps;
            continue;
        }
        const int n0 = (int)max<int64_t>(0, u - first), n1 = a.part ? (int)min<int64_t>(steps, share_end - first) : steps;
        const int row0 = rt * ROWS, n_rows = min(ROWS, q.rows - row0);
        const int t_first = over_group(a, row0), t_last = over_group(a, row0 + n_rows - 1);
        const int key_end = min(q.ctx, q.pos0 + t_last + 1);                     // no row sees a key from here on (may be below 1)
        const int all_see = min(key_end, q.pos0 + t_first + 1);                 // every row sees the keys below
        const int n_last = max(n0, min(n1, (key_end + STREAM_KEYS - 1) / STREAM_KEYS));

        // pages: lane 2 n + i holds the page of 16-key group i of step k + n, 32 steps at a time.  No load stands under a condition: the compiler would wait for all of
        // them where the ways meet; what is not there is read from elsewhere (the row's last entry, page 0) and masked.
        int ids = 0;
        auto load_ids = [&](int k) {
            const int e = (2 * k + lane) >> (a.shift - 4);
            int id = a.table[(size_t)s * a.max_pages + min(e, a.max_pages - 1)];
            asm volatile("" : "+v"(id));
            ids = k + lane / 2 < n_last && e < a.max_pages ? page_checked(id, a.n_pages) : -1;
        };
        load_ids(n0);
        // the lane's column(s): query row, as fp16 pairs later
        u32x4 qw[NT][W];
        int p[NT], heads[NT];
        float slope[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int r = row0 + min(STREAM_ROWS * t + (PARTS > 1 ? col % ROWS : col), n_rows - 1), tok = over_group(a, r);
            heads[t] = h * a.group + r - tok * a.group;
            p[t] = q.pos0 + tok;
            slope[t] = ALIBI ? a.slopes[heads[t]] * LOG2E : 0.0f;
            const uint16_t* qp = a.qkv + (size_t)(q.first + tok) * cols + heads[t] * D + (D / 4) * quarter;
#pragma unroll
            for (int j = 0; j < W; ++j) qw[t][j] = *reinterpret_cast<const u32x4*>(qp + 8 * j);
        }
        __builtin_amdgcn_sched_barrier(0);
        float m[NT], l[NT], zs[NT], ws[NT], G[NT];     // reference; sums of P, of P z' and, over 8, of t G less its rounding; the power of two
        f4 o[NT][F];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            m[t] = -INFINITY;
            l[t] = zs[t] = ws[t] = 0.0f;
            G[t] = 0x1p100f;
#pragma unroll
            for (int e = 0; e < F; ++e) o[t][e] = f4{0.0f, 0.0f, 0.0f, 0.0f};
        }

        const int rest_of = PARTS > 1 ? __builtin_amdgcn_update_dpp(0, part, 0x120 + ROWS, 0xf, 0xf, false) : 0;
        // the lane's keys of a step, in order of the quarters' eight {4 quarter + 0..3, 16 + 4 quarter + 0..3}: N from the part's N-th on
        const int my_group = N < 8 ? part * N / 4 : 0, my_key = 16 * my_group + 4 * quarter + part * N % 4;
        const uint32_t koff = (uint32_t)(col * (D / 2) + quarter * (D / 8)), voff = (uint32_t)(4 * quarter * (D / 2) + col * (D / 32)), poff = (uint32_t)(8 * D + 4 * (my_key % 16));
        kcodes_t kc[2];
        vcodes_t vc[2][4];
        params_t kp[N / 4 + !(N / 4)], vp[N / 4 + !(N / 4)];
        uint32_t bad_next = 0;                         // of the step that is asked for: bit i: 16-key group i has no page
        int64_t at_of[2];                              // and where the groups are
        uint64_t bad_ids = 0;                          // bit l: lane l's group has none
        int ids_from = n0;
        auto load_params = [&](const uint8_t* b0, const uint8_t* b1, params_t* p) {
            if constexpr (N == 8) {
                p[0] = __builtin_nontemporal_load(reinterpret_cast<const params_t*>(b0 + poff));
                p[1] = __builtin_nontemporal_load(reinterpret_cast<const params_t*>(b1 + poff));
            } else p[0] = __builtin_nontemporal_load(reinterpret_cast<const params_t*>((my_group ? b1 : b0) + poff));
        };
        auto load_k = [&](int n) {
            if (n - ids_from >= 32) {
                ids_from = n;
                load_ids(n);
                bad_ids = __ballot(ids < 0);
            }
            bad_next = (uint32_t)(bad_ids >> (2 * (n - ids_from))) & 3u;
            const uint8_t* b[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int id = max(__builtin_amdgcn_readlane(ids, 2 * (n - ids_from) + i), 0);
                at_of[i] = cell_group(id, h, a.kv_heads, a.shift, (2 * n + i) & group_mask, D);
                b[i] = reinterpret_cast<const uint8_t*>(a.kp) + at_of[i];
                kc[i] = __builtin_nontemporal_load(reinterpret_cast<const kcodes_t*>(b[i] + koff));
            }
            load_params(b[0], b[1], kp);
        };
        auto load_v = [&] {
            const uint8_t* b[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                b[i] = reinterpret_cast<const uint8_t*>(a.vp) + at_of[i];
#pragma unroll
                for (int r = 0; r < 4; ++r) vc[i][r] = __builtin_nontemporal_load(reinterpret_cast<const vcodes_t*>(b[i] + voff + (D / 2) * r));
            }
            load_params(b[0], b[1], vp);
        };
        bad_ids = __ballot(ids < 0);
        load_k(n0);
        load_v();
        __builtin_amdgcn_sched_barrier(0);
        // what the scores are multiplied by, and the sum of the row
        float c[NT], qsum[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            int ex = 0;                                // the row is taken by 2^-ex: its largest is 2^14 or more
            if constexpr (DT == LPQ_DT_BF16) {
                float top = 0.0f;
#pragma unroll
                for (int j = 0; j < W; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) top = largest_of_pair<DT>(qw[t][j][e], top);
                f2 z = both_rows(top);
                z = both_halves(fmaxf(z[0], z[1]));
                ex = exponent_of(fmaxf(z[0], z[1])) - 14;
            }
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < W; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (DT == LPQ_DT_BF16) qw[t][j][e] = scaled_pair<DT>(qw[t][j][e], -ex, -ex);
                    sum = Elem<LPQ_DT_FP16>::add_pair(qw[t][j][e], sum);
                }
            f2 z = both_rows(sum);
            z = both_halves(z[0] + z[1]);
            qsum[t] = (z[0] + z[1]) * 0x1p-20f;
            c[t] = __builtin_ldexpf(LOG2E / sqrtf((float)D), 20 + ex);
        }
        auto step = [&](int n) {
#pragma clang fp contract(off)                         // scores are rounded before the reference is taken from them, whatever their size
            const int key0 = STREAM_KEYS * n;
            const uint32_t bad = bad_next;
            const bool plain = bad == 0 && key0 + STREAM_KEYS <= all_see;
            float sc[NT][N];                           // of the lane's keys
            {
                f4 acc[NT][2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    u32x4 kw[W];
#pragma unroll
                    for (int j = 0; j < W; ++j) kw[j] = code_pairs(kc[i][j]);
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        acc[t][i] = f4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                        for (int j = 0; j < W; ++j)
                            acc[t][i] = Elem<LPQ_DT_FP16>::mfma16(__builtin_bit_cast(h8, kw[j]), __builtin_bit_cast(h8, qw[t][j]), acc[t][i]);
                    }
                }
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int k = 0; k < N; ++k) {
                        const uint32_t par = kp[k / 4][k % 4];
                        float v;
                        if constexpr (PARTS == 1) v = acc[t][k / 4][k % 4];
                        else if constexpr (PARTS == 2) v = part ? acc[t][1][k] : acc[t][0][k];
                        else v = part & 2 ? (part & 1 ? acc[t][1][2 + k] : acc[t][1][k]) : part & 1 ? acc[t][0][2 + k] : acc[t][0][k];
                        v = __builtin_fmaf(param_zero<DT>(par), qsum[t], param_scale<DT>(par) * v) * c[t];
                        if constexpr (ALIBI) v = __builtin_fmaf(slope[t], (float)(key0 + my_key + 16 * (k / 4) + k % 4 - p[t]), v);
                        sc[t][k] = v;
                    }
            }
            __builtin_amdgcn_sched_barrier(0);
            load_k(min(n + 1, n_last - 1));
            __builtin_amdgcn_sched_barrier(0);
            h8 pf[NT], rf[SECOND ? NT : 1];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                uint32_t par[N];
#pragma unroll
                for (int k = 0; k < N; ++k) par[k] = vp[k / 4][k % 4];
                if (!plain)                            // what the row does not see: no weight, and no scale or zero that could be infinite or NaN
#pragma unroll
                    for (int k = 0; k < N; ++k) {
                        const int key = key0 + my_key + 16 * (k / 4) + k % 4;
                        const bool hidden = (bad >> (my_group + k / 4) & 1) || key > p[t] || key >= key_end;
                        sc[t][k] = hidden ? -INFINITY : sc[t][k];
                        par[k] = hidden ? 0u : par[k];
                    }
                float pw[N], ts[N], tm = 0.0f, sum = 0.0f;
                auto weights = [&] {
                    const float ms = m[t] == -INFINITY ? 0.0f : m[t];
                    tm = sum = 0.0f;
#pragma unroll
                    for (int k = 0; k < N; ++k) {
                        pw[k] = __builtin_amdgcn_exp2f(sc[t][k] - ms);
                        ts[k] = pw[k] * param_scale<DT>(par[k]);
                        tm = fmaxf(tm, __builtin_fabsf(ts[k]));
                    }
#pragma unroll
                    for (int k = 0; k < N; k += 2) sum += pw[k] + pw[k + 1];
                };
                weights();
                if (__any(m[t] == -INFINITY || !(tm * G[t] < LARGEST_T) || !(sum < RENEW_P))) {
                    float alpha = 1.0f;
                    if (__any(m[t] == -INFINITY || !(tm < RENEW_T) || !(sum < RENEW_P))) {
                        float mx = -INFINITY;
#pragma unroll
                        for (int k = 0; k < N; ++k) mx = fmaxf(mx, sc[t][k]);
                        const float mn = fmaxf(m[t], over_row<ROWS>(mx, OpMax()));
                        alpha = __builtin_amdgcn_exp2f(m[t] - (mn == -INFINITY ? 0.0f : mn));
                        l[t] *= alpha;
                        zs[t] *= alpha;
                        m[t] = mn;
                        weights();
                    }
                    // NEW_T over the power of two in the largest t, none above 2^100; the sums in o and ws are of t G
                    const int e = max((int)(__builtin_bit_cast(uint32_t, over_row<ROWS>(tm, OpMax())) >> 23) - 127, -86);
                    const float g = fminf(fminf(G[t] / alpha, 0x1p100f), __builtin_ldexpf(NEW_T, -e)), by = alpha * g / G[t];
                    ws[t] *= by;
#pragma unroll
                    for (int f = 0; f < F; ++f) o[t][f] *= by;
                    G[t] = g;
                }
                l[t] += sum;
                uint32_t pk[N / 2], rk[N / 2];
#pragma unroll
                for (int k = 0; k < N; k += 2) {
                    const float t0 = ts[k] * G[t], t1 = ts[k + 1] * G[t];
                    zs[t] = __builtin_fmaf(pw[k], param_zero<DT>(par[k]), zs[t]);
                    zs[t] = __builtin_fmaf(pw[k + 1], param_zero<DT>(par[k + 1]), zs[t]);
                    pk[k / 2] = Elem<LPQ_DT_FP16>::pack(t0, t1);
                    if constexpr (FINE) {
                        const h2 p16 = as_h2(pk[k / 2]);
                        rk[k / 2] = Elem<LPQ_DT_FP16>::pack(t0 - (float)p16[0], t1 - (float)p16[1]);
                        if constexpr (!SECOND) rk[k / 2] = __builtin_amdgcn_update_dpp(0, rk[k / 2], 0x120 + ROWS, 0xf, 0xf, false);      // row_ror
                    } else ws[t] = __builtin_amdgcn_fdot2(as_h2(pk[k / 2]), h2{-1, -1}, ws[t] + (t0 + t1), false);
                }
                u32x4 operand;                         // this part's keys; what the next part's lost; zero for the others
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    operand[k] = PARTS == 1 || part == k / (N / 2) ? pk[k % (N / 2)] : PARTS == 2 || rest_of == k / (N / 2) ? rk[k % (N / 2)] : 0u;
                pf[t] = __builtin_bit_cast(h8, operand);
                if constexpr (SECOND) rf[t] = __builtin_bit_cast(h8, u32x4{rk[0], rk[1], rk[2], rk[3]});
            }
            // V^T operands: halves of two keys' words side by side, then pairs
#pragma unroll
            for (int half = 0; half < W / 2; ++half) { // D = 128: even, odd features; D = 64: the lane has a half of a word only
                u32x4 pair[4];                         // [keys][e]: feature 2 e + half of the word
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    pair[k] = code_pairs(__builtin_amdgcn_perm(vc[k / 2][2 * (k % 2) + 1], vc[k / 2][2 * (k % 2)], half ? 0x07060302u : 0x05040100u));
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const u32x4 vt = {pair[0][e], pair[1][e], pair[2][e], pair[3][e]};
                    const int f = D == 128 ? 2 * e + half : e;
#pragma unroll
                    for (int t = 0; t < NT; ++t) o[t][f] = Elem<LPQ_DT_FP16>::mfma16(__builtin_bit_cast(h8, vt), pf[t], o[t][f]);
                    if constexpr (SECOND)
#pragma unroll
                        for (int t = 0; t < NT; ++t) o[t][f] = Elem<LPQ_DT_FP16>::mfma16(__builtin_bit_cast(h8, vt), rf[t], o[t][f]);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            load_v();
            __builtin_amdgcn_sched_barrier(0);
        };
        for (int n = n0; n < n_last; ++n) step(n);

        // a whole row tile's results, or a part's sums
        const bool whole = n0 == 0 && n1 == steps;
        float* const slot = a.part + (size_t)(2 * w + (first < share_u ? 0 : 1)) * SLOT;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int ri = STREAM_ROWS * t + col;
            const float L = over_row<ROWS>(l[t], OpAdd()), inv_g = 1.0f / G[t], rest = 8.0f * over_row<ROWS>(ws[t], OpAdd()), zero = over_row<ROWS>(zs[t], OpAdd());
            if constexpr (PARTS > 1)                   // columns of the same row
#pragma unroll
                for (int f = 0; f < F; ++f)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        if constexpr (ROWS <= 4) o[t][f][g] += dpp_move<0x124>(o[t][f][g]);
                        o[t][f][g] += dpp_move<0x128>(o[t][f][g]);
                    }
            // feature k of the lane's word g: words 4 quarter + g (D = 128), 2 quarter + g (D = 64, even features from one row, odd ones from the next)
            auto value = [&](int g, int k) {
                const float v = D == 128 ? o[t][k][g] : o[t][k / 2][2 * g + k % 2];
                return __builtin_fmaf(__builtin_fmaf(v, 0x1p20f, rest), inv_g, zero);
            };
            if (ri < n_rows) {
                if (whole) {
                    const float inv = L == 0.0f ? 0.0f : 1.0f / L;
                    uint16_t* op = a.out + (size_t)(q.first + p[t] - q.pos0) * a.heads * D + heads[t] * D;
#pragma unroll
                    for (int g = 0; g < W; ++g) {
                        u32x4 y;
#pragma unroll
                        for (int k = 0; k < 8; k += 2) y[k / 2] = Elem<DT>::pack(value(g, k) * inv, value(g, k + 1) * inv);
                        *reinterpret_cast<u32x4*>(op + 8 * (W * quarter + g)) = y;
                    }
                } else {
#pragma unroll
                    for (int g = 0; g < W; ++g)
#pragma unroll
                        for (int k = 0; k < 8; k += 4)
                            *reinterpret_cast<f4*>(slot + ri * D + 8 * (W * quarter + g) + k) = f4{value(g, k), value(g, k + 1), value(g, k + 2), value(g, k + 3)};
                    if (quarter == 0) *reinterpret_cast<f2*>(slot + ROWS * D + 2 * ri) = f2{m[t], L};
                }
            }
        }
        if (!whole && first >= share_u)                // it begins here and ends in another worker's share
            cut = Cut{stream_worker(total, first + steps - 1, workers) - w + 1, q.first, row0, 64 * h + n_rows};
        u = first + n1;
    }
    if (a.part && lane == 0) reinterpret_cast<Cut*>(a.part + (size_t)2 * a.workers * SLOT)[w] = cut;
}

template <int DT, int D, int ROWS, bool ALIBI>
__global__ __launch_bounds__(256, ROWS <= 16 ? CELL_WAVES : STREAM_WAVES) void stream4_attention_kernel(AttnArgs a)
{
    stream4_block<DT, D, ROWS, ALIBI>(a, (int)blockIdx.x);
}

// Adds up the parts of the row tiles that the entries of `cuts` name, a row at a time: all maxima and sums first, a part to a lane, then the parts' features,
// whose loads do not wait for the former.  A wave takes an entry, four to a workgroup; LONG, for few lists of hundreds of parts: a workgroup takes 16 entries, of
// which it finds one at most as a rule, and a slice of 32 features; ids count rows and slices first, so that a list's workgroups are on all XCDs.  Either is right for any list.
// (Parts one after the other, the maximum carried along, 16 entries to a workgroup in both forms: 3.9, 5.5, 12.6 us for 16 sequences of 40 heads, 61 of 8 K/V heads, one of 90001 positions; so 2.8, 4.7, 5.1, with the last list's workgroups on one XCD 12.4.)
template <int DT, int D, int ROWS, bool LONG>
__global__ __launch_bounds__(256) void combine4_kernel(AttnArgs a)
{
    constexpr int SLOT = ROWS * (D + 2), TEAM = LONG ? 256 : 64, SLICES = LONG ? D / 32 : 1, LANES = D / SLICES / 4, WAYS = TEAM / LANES, ENTRIES = LONG ? 16 : 1;
    __shared__ __attribute__((aligned(16))) float weights[LONG ? 256 : 1], sums[LONG ? 4 : 1][40];
    const Cut* cuts = reinterpret_cast<const Cut*>(a.part + (size_t)2 * a.workers * SLOT);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), me = LONG ? (int)threadIdx.x : lane;
    const int y = LONG ? blockIdx.x : blockIdx.y, block = LONG ? blockIdx.y : blockIdx.x, rows_apart = (int)(LONG ? gridDim.x : gridDim.y) / SLICES;
    const int f = 32 * (y % SLICES) + 4 * (me % LANES), way = me / LANES, ri = y / SLICES;
    const int w0 = LONG ? 16 * block : 4 * block + wave;
    Cut mine{0, 0, 0, 0};
    if (lane < ENTRIES && w0 + lane < a.workers) mine = cuts[w0 + lane];
    for (uint64_t todo = __ballot(mine.parts != 0); todo; todo &= todo - 1) {
        const int k0 = __builtin_ctzll(todo), w = w0 + k0;
        const int parts = __builtin_amdgcn_readlane(mine.parts, k0), first = __builtin_amdgcn_readlane(mine.first, k0);
        const int row0 = __builtin_amdgcn_readlane(mine.row0, k0), hr = __builtin_amdgcn_readlane(mine.head_rows, k0), h = hr >> 6, n_rows = hr & 63;
        for (int row = ri; row < n_rows; row += rows_apart) {
            // part k: worker w + k; the first is in its slot 1, the others, which begin inside the row tile, in their slot 0
            auto part = [&](int k) { return a.part + (size_t)(2 * (w + k) + (k == 0 ? 1 : 0)) * SLOT; };
            float m = -INFINITY, l = 0.0f;
            f4 v = {0.0f, 0.0f, 0.0f, 0.0f};
            for (int c0 = 0; c0 < parts; c0 += TEAM) {                           // one turn but for the longest lists
                const f2 ml = c0 + me < parts ? *reinterpret_cast<const f2*>(part(c0 + me) + ROWS * D + 2 * row) : f2{-INFINITY, 0.0f};
                constexpr int AHEAD = 8;
                f4 o[AHEAD];
                const int end = min(parts - c0, TEAM);
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) o[i] = *reinterpret_cast<const f4*>(part(c0 + min(way + WAYS * i, end - 1)) + row * D + f);
                float top = group_reduce<64>(ml[0], OpMax());
                if constexpr (LONG) {
                    __syncthreads();                   // the last turn's are read
                    if (lane == 0) sums[wave][0] = top;
                    __syncthreads();
                    top = fmaxf(fmaxf(sums[0][0], sums[1][0]), fmaxf(sums[2][0], sums[3][0]));
                }
                const float mn = fmaxf(m, top), ms = mn == -INFINITY ? 0.0f : mn, alpha = __builtin_amdgcn_exp2f(m - ms), x = __builtin_amdgcn_exp2f(ml[0] - ms);
                m = mn;
                l = l * alpha + x * ml[1];             // this lane's parts' sum
                v *= alpha;
                if constexpr (LONG) {
                    weights[me] = x;
                    __syncthreads();
                }
                auto weight = [&](int k) { return LONG ? weights[k] : __shfl(x, k); };
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) {
                    const int k = way + WAYS * i;
                    const float y = weight(min(k, TEAM - 1));
                    if (k < end) v += y * o[i];
                }
                for (int k = way + WAYS * AHEAD; k - way < end; k += WAYS) {     // every lane as often
                    const float y = weight(min(k, TEAM - 1));
                    if (k < end) v += y * *reinterpret_cast<const f4*>(part(c0 + k) + row * D + f);
                }
            }
            l = group_reduce<64>(l, OpAdd());
#pragma unroll
            for (int d = LANES; d < 64; d *= 2) v += f4{__shfl_xor(v[0], d), __shfl_xor(v[1], d), __shfl_xor(v[2], d), __shfl_xor(v[3], d)};
            if constexpr (LONG) {
                __syncthreads();
                if (lane < LANES) *reinterpret_cast<f4*>(&sums[wave][4 * lane]) = v;
                if (lane == 0) sums[wave][32] = l;
                __syncthreads();
                v = f4{0.0f, 0.0f, 0.0f, 0.0f};
                l = 0.0f;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    v += *reinterpret_cast<const f4*>(&sums[k][4 * (lane % LANES)]);
                    l += sums[k][32];
                }
            }
            if (way != 0) continue;
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;
            const int r = row0 + row, tok = over_group(a, r), head = h * a.group + r - tok * a.group;
            *reinterpret_cast<u32x2*>(a.out + (size_t)(first + tok) * a.heads * D + head * D + f) =
                u32x2{Elem<DT>::pack(v[0] * inv, v[1] * inv), Elem<DT>::pack(v[2] * inv, v[3] * inv)};
        }
    }
}

template <int DT, int D, bool ALIBI>
__global__ __launch_bounds__(256, 2) void tile4_attention_kernel(AttnArgs a) { tile_block<DT, D, ALIBI, SRC_CELLS>(a, (int)blockIdx.x); }

// Both for a batch that may have sequences of either kind, as for 16-bit caches.
template <int DT, int D, int ROWS, bool ALIBI>
__global__ __launch_bounds__(256, 2) void mixed4_attention_kernel(AttnArgs stream, AttnArgs tile)
{
    const int streams = stream.workers / 4;
    if ((int)blockIdx.x < streams) stream4_block<DT, D, ROWS, ALIBI>(stream, (int)blockIdx.x);
    else tile_block<DT, D, ALIBI, SRC_CELLS>(tile, (int)blockIdx.x - streams);
}

}  // namespace

struct CellKernels {
    static constexpr bool CELLS = true, ROWS = false;
    template <int TILE> static constexpr bool has = true;
    template <int TILE> static constexpr bool has_mixed = TILE == 8 || TILE == STREAM_ROWS;
    template <int DT, int D, int TILE, bool ALIBI> static constexpr auto mixed = &mixed4_attention_kernel<DT, D, TILE, ALIBI>;
    template <int DT, int D, int TILE, bool ALIBI> static constexpr auto stream = &stream4_attention_kernel<DT, D, TILE, ALIBI>;
    template <int DT, int D, int TILE, bool LONG> static constexpr auto combine = &combine4_kernel<DT, D, TILE, LONG>;
    static constexpr unsigned cuts_per_wg(bool long_lists) { return long_lists ? 16 : 4; }
    template <int DT, int D, bool ALIBI> static constexpr auto tile = &tile4_attention_kernel<DT, D, ALIBI>;
    template <int DT, int D, bool ALIBI>
    static hipError_t allow(bool mixed_launch, int rows, bool, size_t lds)
    {
        return !mixed_launch ? allow_lds<tile<DT, D, ALIBI>>(lds) : rows == 8 ? allow_lds<mixed<DT, D, 8, ALIBI>>(lds) : allow_lds<mixed<DT, D, STREAM_ROWS, ALIBI>>(lds);
    }
};

hipError_t launch_cell_attention(const AttentionPlan& p, const lpq_attn_cfg& c, const AttentionBatch& b, float* part, hipStream_t s)
{
    return launch_attention_of<CellKernels>(p, c, b, part, s);
}

}  // namespace lpq

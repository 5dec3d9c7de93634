// Causal attention of new tokens over pages of 4-bit cells:
//     out[row] = sum_j w_j v_j / sum_j w_j,   w_j = exp(q . k_j / sqrt(D) + slope (j - p)),   j <= p,   k_j = s_j c_j + z_j, v_j = s'_j c'_j + z'_j
// with codes c of 0 to 15 for each feature and a scale and a zero for each key and head.  Rows, work lists, splits and the joining of parts are those of the
// 16-bit caches' kernels.  The tile kernel (prompts and chunks) is theirs too, with values made from the cells on their way into LDS, rounded to the type.
//
// The streaming kernel multiplies the codes themselves: scale and zero are one number each for a key, so
//     q . k_j        = s_j (q . c_j) + z_j sum(q)
//     sum_j w_j v_jf = sum_j (w_j s'_j) (c'_jf - 8) + sum_j w_j (z'_j + 8 s'_j)
// where the first sum of each is the matrix units' and the others cost two operations a score.  A code in the last bits of an fp16 number with no exponent is
// that number, code * 2^-24 (or 2^-20 four bits higher): unpacking is one AND per pair and half a shift, for queries of either type: those in bf16 are taken by a power of two
// for each row, which changes none of their eight bits that count.  Codes are exact; what is rounded are the weights w s', to fp16 beside a
// largest of 2^15, and only the codes' distance from 8 sees it.
#include <algorithm>

#include "lpq_batch_attention.h"

namespace lpq {

namespace {

// ---- streaming kernel -----------------------------------------------------------------------------
// Bound by the memory: D + 8 bytes per key and K/V head.  Workers are single waves with equal shares of the list of 32-key units.
// Products on 16x16x32, columns = rows of the problem:
//   S^T = C_k . Q^T  lane (i = lane % 16, q = lane / 16) holds codes D / 4 q .. of key i as they lie; a word has pairs 0 and 2 at 2^-24, 1 and 3 at 2^-20, which go to a
//                    product each, with the query's pairs in that order.  Register r of the result: key 4 q + r, column i.
//   O^T = C_v^T . P^T over 32 keys: quarter q contracts over its own keys {4 q + 0..3, 16 + 4 q + 0..3}.  A lane has a word (D = 128; half a word, D = 64) of each of the
//                    eight; halves of two keys' words are put side by side, and an AND gives a pair of keys of one feature.
// Weights: P = exp2(score - m), its sum and its sum with the zeros in fp32; t = P s' is taken by a power of two G for each column so that the largest so far is below 2^15.
// Both m and G are renewed only where t G passes 2^15: one maximum a step decides (P may be up to 2^60).
constexpr int CELL_DEPTH = 2;                          // units under way
constexpr float LARGEST_T = 0x1p15f, RENEW_T = 0x1p60f;

// The four pairs of a word's codes as fp16 numbers, code * 2^-20.
__device__ __forceinline__ u32x4 code_pairs(uint32_t w)
{
    constexpr uint32_t M = 0x00f000f0u;
    return u32x4{w << 4 & M, w & M, w >> 4 & M, w >> 8 & M};
}

template <int DT, int D, int NT, bool ALIBI>
__device__ __forceinline__ void stream4_block(const AttnArgs& a, int block, ShareSmem& sm)
{
    constexpr int W = D / 32, F = D / 16, TILE_ROWS = STREAM_ROWS * NT;          // words of a lane's codes of a key; its features of V
    constexpr int SLOT = TILE_ROWS * (D + 2);
    typedef uint32_t kcodes_t __attribute__((ext_vector_type(W)));
    typedef std::conditional_t<D == 128, uint32_t, uint16_t> vcodes_t;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, quarter = lane >> 4;
    const int cols = (a.heads + 2 * a.kv_heads) * D, group_mask = (1 << (a.shift - 4)) - 1;

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

        // the lane's column(s): query row as fp16 pairs, what its scores are multiplied by, sum of the row, position, slope
        u32x4 qw[NT][W];
        float c[NT], qsum[NT], slope[NT];
        int p[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int r = row0 + min(STREAM_ROWS * t + col, n_rows - 1), tok = r / a.group, head = h * a.group + r % a.group;
            const uint16_t* qp = a.qkv + (size_t)(q.first + tok) * cols + head * D + (D / 4) * quarter;
#pragma unroll
            for (int j = 0; j < W; ++j) qw[t][j] = *reinterpret_cast<const u32x4*>(qp + 8 * j);
            int ex = 0;                                // the row is taken by 2^-ex: its largest is 2^14 or more
            if constexpr (DT == LPQ_DT_BF16) {
                float top = 0.0f;
#pragma unroll
                for (int j = 0; j < W; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) top = largest_of_pair<DT>(qw[t][j][e], top);
                f2 z = both_rows(top);
                z = both_halves(fmaxf(z[0], z[1]));
                ex = exponent_to_14(fmaxf(z[0], z[1]));
            }
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < W; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (DT == LPQ_DT_BF16) qw[t][j][e] = scaled_pair<DT>(qw[t][j][e], -ex);
                    sum = Elem<LPQ_DT_FP16>::add_pair(qw[t][j][e], sum);
                }
            f2 z = both_rows(sum);
            z = both_halves(z[0] + z[1]);
            qsum[t] = (z[0] + z[1]) * 0x1p-20f;
            c[t] = __builtin_ldexpf(LOG2E / sqrtf((float)D), 20 + ex);
            p[t] = q.pos0 + tok;
            slope[t] = ALIBI ? a.slopes[head] * LOG2E : 0.0f;
        }
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

        const uint32_t koff = (uint32_t)(col * (D / 2) + quarter * (D / 8)), voff = (uint32_t)(4 * quarter * (D / 2) + col * (D / 32)), poff = (uint32_t)(8 * D + 16 * quarter);
        kcodes_t kc[CELL_DEPTH][2];
        vcodes_t vc[CELL_DEPTH][2][4];
        u32x4 kp[CELL_DEPTH][2], vp[CELL_DEPTH][2];    // parameters of keys 4 quarter ..
        uint32_t bad_of[CELL_DEPTH];                   // of the buffers' steps: bit i: 16-key group i has no page
        uint64_t bad_ids = 0;                          // bit l: lane l's group has none
        int ids_from = n0;
        auto group_bytes = [&](const uint16_t* pages, int n, int i) {
            const int id = max(__builtin_amdgcn_readlane(ids, 2 * (n - ids_from) + i), 0);
            return reinterpret_cast<const uint8_t*>(pages) + (size_t)cell_group(id, h, a.kv_heads, a.shift, (2 * n + i) & group_mask, D);
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
                const uint8_t* b = group_bytes(a.kp, n, i);
                kc[x][i] = __builtin_nontemporal_load(reinterpret_cast<const kcodes_t*>(b + koff));
                kp[x][i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(b + poff));
            }
        };
        auto load_v = [&](int n, int x) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint8_t* b = group_bytes(a.vp, n, i);
#pragma unroll
                for (int r = 0; r < 4; ++r) vc[x][i][r] = __builtin_nontemporal_load(reinterpret_cast<const vcodes_t*>(b + voff + (D / 2) * r));
                vp[x][i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(b + poff));
            }
        };
        if (n0 < n_last) bad_ids = __ballot(ids < 0);
#pragma unroll
        for (int x = 0; x < CELL_DEPTH; ++x)
            if (n0 + x < n_last) {
                load_k(n0 + x, x);
                load_v(n0 + x, x);
            }
        auto step = [&](int n, int x) {
#pragma clang fp contract(off)                         // scores are rounded before the reference is taken from them, whatever their size
            const int key0 = STREAM_KEYS * n;
            const uint32_t bad = bad_of[x];
            const bool plain = bad == 0 && key0 + STREAM_KEYS <= all_see, more = n + CELL_DEPTH < n_last;
            float sc[NT][8];                           // [4 i + r]: key 16 i + 4 quarter + r
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                u32x4 kw[W];
#pragma unroll
                for (int j = 0; j < W; ++j) kw[j] = code_pairs(kc[x][i][j]);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    f4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int j = 0; j < W; ++j) acc = Elem<LPQ_DT_FP16>::mfma16(__builtin_bit_cast(h8, kw[j]), __builtin_bit_cast(h8, qw[t][j]), acc);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        float v = __builtin_fmaf(param_zero<DT>(kp[x][i][r]), qsum[t], param_scale<DT>(kp[x][i][r]) * acc[r]) * c[t];
                        if constexpr (ALIBI) v = __builtin_fmaf(slope[t], (float)(key0 + 16 * i + 4 * quarter + r - p[t]), v);
                        sc[t][4 * i + r] = v;
                    }
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            if (more) load_k(n + CELL_DEPTH, x);
            __builtin_amdgcn_sched_barrier(0);
            h8 pf[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                u32x4 par[2] = {vp[x][0], vp[x][1]};
                if (!plain)                            // what the column does not see: no weight, and no scale or zero that could be infinite or NaN
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const int key = key0 + 16 * i + 4 * quarter + r;
                            const bool hidden = (bad >> i & 1) || key > p[t] || key >= key_end;
                            sc[t][4 * i + r] = hidden ? -INFINITY : sc[t][4 * i + r];
                            par[i][r] = hidden ? 0u : par[i][r];
                        }
                float pw[8], ts[8], tm = 0.0f;
                auto weights = [&] {
                    const float ms = m[t] == -INFINITY ? 0.0f : m[t];
                    tm = 0.0f;
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        pw[k] = __builtin_amdgcn_exp2f(sc[t][k] - ms);
                        ts[k] = pw[k] * param_scale<DT>(par[k / 4][k % 4]);
                        tm = fmaxf(tm, ts[k]);
                    }
                    f2 z = both_rows(tm);
                    z = both_halves(fmaxf(z[0], z[1]));
                    tm = fmaxf(z[0], z[1]);
                };
                weights();
                if (__any(m[t] == -INFINITY || !(tm * G[t] < LARGEST_T))) {
                    float alpha = 1.0f;
                    if (__any(m[t] == -INFINITY || !(tm < RENEW_T))) {
                        float mx = -INFINITY;
#pragma unroll
                        for (int k = 0; k < 8; ++k) mx = fmaxf(mx, sc[t][k]);
                        f2 z = both_rows(mx);
                        z = both_halves(fmaxf(z[0], z[1]));
                        const float mn = fmaxf(m[t], fmaxf(z[0], z[1]));
                        alpha = __builtin_amdgcn_exp2f(m[t] - (mn == -INFINITY ? 0.0f : mn));
                        l[t] *= alpha;
                        zs[t] *= alpha;
                        m[t] = mn;
                        weights();
                    }
                    // 2^14 over the power of two in the largest t, none above 2^100; the sums in o and ws are of t G
                    const int e = max((int)(__builtin_bit_cast(uint32_t, tm) >> 23) - 127, -86);
                    const float g = fminf(fminf(G[t] / alpha, 0x1p100f), __builtin_ldexpf(1.0f, 14 - e)), by = alpha * g / G[t];
                    ws[t] *= by;
#pragma unroll
                    for (int f = 0; f < F; ++f) o[t][f] *= by;
                    G[t] = g;
                }
                u32x4 pk;
#pragma unroll
                for (int k = 0; k < 8; k += 2) {
                    const float t0 = ts[k] * G[t], t1 = ts[k + 1] * G[t];
                    l[t] += pw[k] + pw[k + 1];
                    zs[t] = __builtin_fmaf(pw[k], param_zero<DT>(par[k / 4][k % 4]), zs[t]);
                    zs[t] = __builtin_fmaf(pw[k + 1], param_zero<DT>(par[k / 4][k % 4 + 1]), zs[t]);
                    pk[k / 2] = Elem<LPQ_DT_FP16>::pack(t0, t1);
                    const h2 rounded = as_h2(pk[k / 2]);
                    ws[t] += (t0 - (float)rounded[0]) + (t1 - (float)rounded[1]);
                }
                pf[t] = __builtin_bit_cast(h8, pk);
            }
            // V^T operands: halves of two keys' words side by side, then pairs by AND
#pragma unroll
            for (int half = 0; half < W / 2; ++half) { // D = 128: even, odd features; D = 64: the lane has a half of a word only
                u32x4 pair[4];                         // [keys][e]: feature 2 e + half of the word
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    pair[k] = code_pairs(__builtin_amdgcn_perm(vc[x][k / 2][2 * (k % 2) + 1], vc[x][k / 2][2 * (k % 2)], half ? 0x07060302u : 0x05040100u));
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const u32x4 vt = {pair[0][e], pair[1][e], pair[2][e], pair[3][e]};
                    const int f = D == 128 ? 2 * e + half : e;
#pragma unroll
                    for (int t = 0; t < NT; ++t) o[t][f] = Elem<LPQ_DT_FP16>::mfma16(__builtin_bit_cast(h8, vt), pf[t], o[t][f]);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            if (more) load_v(n + CELL_DEPTH, x);
            __builtin_amdgcn_sched_barrier(0);
        };
        for (int n = n0; n < n_last; n += CELL_DEPTH)
#pragma unroll
            for (int x = 0; x < CELL_DEPTH; ++x)       // buffers by name
                if (n + x < n_last) step(n + x, x);

        // a whole row tile's results, or a part's sums
        const bool whole = n0 == 0 && n1 == steps;
        float* const slot = a.part + (size_t)(2 * w + (first < share.u ? 0 : 1)) * SLOT;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int ri = STREAM_ROWS * t + col, r = row0 + min(ri, n_rows - 1), tok = r / a.group, head = h * a.group + r % a.group;
            auto over_quarters = [](float v) {
                f2 z = both_rows(v);
                z = both_halves(z[0] + z[1]);
                return z[0] + z[1];
            };
            const float L = over_quarters(l[t]), inv_g = 1.0f / G[t], rest = 8.0f * over_quarters(ws[t]), zero = over_quarters(zs[t]);
            // feature k of the lane's word g: words 4 quarter + g (D = 128), 2 quarter + g (D = 64, even features from one row, odd ones from the next)
            auto value = [&](int g, int k) {
                const float v = D == 128 ? o[t][k][g] : o[t][k / 2][2 * g + k % 2];
                return __builtin_fmaf(__builtin_fmaf(v, 0x1p20f, rest), inv_g, zero);
            };
            if (ri < n_rows) {
                if (whole) {
                    const float inv = L == 0.0f ? 0.0f : 1.0f / L;
                    uint16_t* op = a.out + (size_t)(q.first + tok) * a.heads * D + head * D;
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
__global__ __launch_bounds__(256, NT == 1 ? CELL_WAVES : STREAM_WAVES) void stream4_attention_kernel(AttnArgs a)
{
    __shared__ ShareSmem sm;
    stream4_block<DT, D, NT, ALIBI>(a, (int)blockIdx.x, sm);
}

template <int DT, int D, bool ALIBI>
__global__ __launch_bounds__(256, 2) void tile4_attention_kernel(AttnArgs a) { tile_block<DT, D, ALIBI, SRC_CELLS>(a, (int)blockIdx.x); }

// Both for a batch that may have sequences of either kind, as for 16-bit caches.
template <int DT, int D, bool ALIBI>
__global__ __launch_bounds__(256, 2) void mixed4_attention_kernel(AttnArgs stream, AttnArgs tile)
{
    const int streams = stream.workers / 4;
    if ((int)blockIdx.x < streams) stream4_block<DT, D, 1, ALIBI>(stream, (int)blockIdx.x, *reinterpret_cast<ShareSmem*>(smem_raw));
    else tile_block<DT, D, ALIBI, SRC_CELLS>(tile, (int)blockIdx.x - streams);
}

}  // namespace

struct CellKernels {
    static constexpr bool CELLS = true;
    template <int DT, int D, bool ALIBI> static constexpr auto mixed = &mixed4_attention_kernel<DT, D, ALIBI>;
    template <int DT, int D, int NT, bool ALIBI> static constexpr auto stream = &stream4_attention_kernel<DT, D, NT, ALIBI>;
    template <int DT, int D, bool ALIBI> static constexpr auto tile = &tile4_attention_kernel<DT, D, ALIBI>;
    template <int DT, int D, bool ALIBI> static constexpr auto tile_rows = tile<DT, D, ALIBI>;     // there are no packed rows of cells: not reached
};

hipError_t launch_cell_attention(const AttentionPlan& p, const lpq_attn_cfg& c, const AttentionBatch& b, float* part, hipStream_t s)
{
    return launch_attention_of<CellKernels>(p, c, b, part, s);
}

}  // namespace lpq

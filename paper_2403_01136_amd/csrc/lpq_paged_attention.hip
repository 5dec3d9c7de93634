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

#include "lpq_batch_attention.h"

namespace lpq {

namespace {

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

// One wave per SIMD, two units under way: few, long, contiguous streams suit the memory.  Waves per SIMD / units, us, 61 sequences of 8 K/V heads and one of 90001
// positions: 1 / 1 77.8, 66.0; 1 / 2 76.9, 63.2; 1 / 3 77.6, 62.7; 2 / 1 80.4, 66.4; 2 / 2 81.6, 66.5; 3 / 1 85.0, 72.4.
constexpr int DEPTH = 2;

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
        const int h = tiles == 1 ? (int)tile : (int)((uint32_t)tile / (uint32_t)tiles), rt = tiles == 1 ? 0 : (int)((uint32_t)tile % (uint32_t)tiles);
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

template <int DT, int D, bool ALIBI, int SRC>
__global__ __launch_bounds__(256, 2) void tile_attention_kernel(AttnArgs a) { tile_block<DT, D, ALIBI, SRC>(a, (int)blockIdx.x); }

// Both for a batch that may have sequences of either kind: the streaming kernel's workgroups, then the tile kernel's, which multiply while the others read.
// A launch of each / this one, us: two chunks of 512 beside 9 sequences that decode, 56 heads (8 K/V heads), biases, 74 / 67 with contexts of 100 to 6000, 125 / 117 with 900 to
// 6000; 250 with up to 2000 and one chunk, 64 heads (8), 150 / 143; 60 with up to 1000 and one chunk, 40 heads (40), 113 / 100; 4 with up to 800 and a chunk of 200, 32 heads
// (8), 23 / 16.  The tile kernel's workgroups first: 62 (contexts from 100), 210, 144, 15; by turns: 69, 193, 134, 15: streams that begin late end last.  With two column tiles the streaming kernel has more registers than two workgroups a compute unit leave: a launch of each.
template <int DT, int D, bool ALIBI>
__global__ __launch_bounds__(256, 2) void mixed_attention_kernel(AttnArgs stream, AttnArgs tile)
{
    const int streams = stream.workers / 4;
    if ((int)blockIdx.x < streams) stream_block<DT, D, 1, ALIBI>(stream, (int)blockIdx.x, *reinterpret_cast<ShareSmem*>(smem_raw));
    else tile_block<DT, D, ALIBI, SRC_PAGES>(tile, (int)blockIdx.x - streams);
}

}  // namespace

// ---- host ------------------------------------------------------------------------------------------

// Room that the tile kernel's parts may take: its list has a place for each sequence, also for those that the streaming kernel does.
constexpr size_t MAX_PART_BYTES = (size_t)256 << 20;
constexpr int FEW_STEPS = 8, SHORT_WALK = 2048, WHOLE_WALK = 192;        // steps of a worker, positions: see below

// What a call launches: the streaming kernel, the tile kernel or, where a batch may have sequences of both kinds, both, in one launch if column tiles are single.
AttentionPlan attention_plan(const lpq_attn_cfg& c, AttentionSource source, int n_seqs, int M, int max_q, int max_kv, int cus)
{
    AttentionPlan p{};
    const bool paged = source != SRC_ROWS;
    const int group = c.n_heads / c.n_kv_heads;
    const int64_t most = (int64_t)std::min(max_q, M) * group;
    // Rows of the streaming kernel's tiles: those to expect where it is alone, else those of a decoding sequence; from 4 on for cells.  Two tiles of 8 rows for 9 to 16 where walks are
    // short and a worker has few steps of them: cells read twice cost less there than a softmax that idle columns share saves.  One tile of 16 / two of 8, us: 16 sequences of 400 to 700
    // positions, 80 heads (5 K/V heads) 20.2 / 16.6; 24, 64 (8), two tokens, up to 700 20.5 / 18.4; 24, 40 (8), three tokens, up to 2600 26.4 / 24.3, up to 4000 28.5 / 29.0, up to 9000 36.7 / 39.6; 8 such up to 4000 26.8 / 27.7, up
    // to 8000 31.2 / 34.7; one of 90001, 112 (8) 37.8 / 43.9.
    auto tile_of_rows = [&](int64_t rows, int smallest) { return rows <= 4 && smallest <= 4 ? 4 : rows <= 8 && smallest <= 8 ? 8 : rows <= STREAM_ROWS ? STREAM_ROWS : 2 * STREAM_ROWS; };
    const int smallest = source == SRC_CELLS ? 4 : STREAM_ROWS;
    p.stream_tile = 0;
    if (paged && most <= 2 * STREAM_ROWS) p.stream_tile = tile_of_rows(most, smallest);
    else if (paged && n_seqs > 1 && group <= 2 * STREAM_ROWS) p.stream_tile = tile_of_rows(group, std::max(smallest, 8));
    p.tile = !(paged && most <= 2 * STREAM_ROWS);
    const int64_t steps = (int64_t)n_seqs * c.n_kv_heads * (((int64_t)max_kv + STREAM_KEYS - 1) / STREAM_KEYS);
    if (source == SRC_CELLS && !p.tile && p.stream_tile == STREAM_ROWS && max_kv <= SHORT_WALK && steps < (int64_t)FEW_STEPS * 4 * cus * CELL_WAVES) p.stream_tile = 8;
    p.workers = 4 * cus * (source == SRC_CELLS && p.stream_tile <= STREAM_ROWS && !p.tile ? CELL_WAVES : STREAM_WAVES);
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
    // Cells of short walks are left whole, without a second launch.  Split / whole, us on the device, for 3 sequences of 64-wide heads, 16 of 40 heads, 61 of 64 (8 K/V heads), 24 drafts: up to
    // 128 positions 8.4 / 6.5, 11.9 / 9.9, 14.7 / 10.8, 15.5 / 13.8, 160 to 190 8.6 / 8.2, 13.6 / 12.9, 16.7 / 11.3, 17.9 / 15.6, up to 256 8.7 / 9.3, 13.3 / 13.7, 17.0 / 14.8, 17.9 / 19.1.
    const bool whole = source == SRC_CELLS && !p.tile && max_kv <= WHOLE_WALK;
    if (p.stream_tile && !whole) p.stream_floats = (size_t)p.workers * (2 * p.stream_tile * d2 + sizeof(Cut) / sizeof(float));
    // lists of 32 parts and more, where the walks are long enough to be cut that often (4 sequences of up to 800 positions: long lists' form 7.2 us, the other's 4.0)
    p.long_lists = (int64_t)n_seqs * c.n_kv_heads * 32 <= p.workers && max_kv >= 64 * STREAM_KEYS;
    p.stream_rows = (int)std::min<int64_t>(p.stream_tile, p.tile ? 2 * STREAM_ROWS : most);
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

struct PageKernels {
    static constexpr bool CELLS = false, ROWS = true;
    template <int TILE> static constexpr bool has = TILE == STREAM_ROWS || TILE == 2 * STREAM_ROWS;
    template <int TILE> static constexpr bool has_mixed = TILE == STREAM_ROWS;
    template <int DT, int D, int TILE, bool ALIBI> static constexpr auto mixed = &mixed_attention_kernel<DT, D, ALIBI>;
    template <int DT, int D, int TILE, bool ALIBI> static constexpr auto stream = &stream_attention_kernel<DT, D, TILE / STREAM_ROWS, ALIBI>;
    template <int DT, int D, int TILE, bool LONG> static constexpr auto combine = &stream_combine_kernel<DT, D, TILE, LONG>;
    static constexpr unsigned cuts_per_wg(bool) { return CUTS_PER_WG; }
    template <int DT, int D, bool ALIBI> static constexpr auto tile = &tile_attention_kernel<DT, D, ALIBI, SRC_PAGES>;
    template <int DT, int D, bool ALIBI> static constexpr auto tile_rows = &tile_attention_kernel<DT, D, ALIBI, SRC_ROWS>;
    template <int DT, int D, bool ALIBI>
    static hipError_t allow(bool mixed_launch, int, bool pages, size_t lds)
    {
        return mixed_launch ? allow_lds<mixed<DT, D, STREAM_ROWS, ALIBI>>(lds) : pages ? allow_lds<tile<DT, D, ALIBI>>(lds) : allow_lds<tile_rows<DT, D, ALIBI>>(lds);
    }
};

hipError_t launch_batch_attention(const AttentionPlan& p, const lpq_attn_cfg& c, const AttentionBatch& b, float* part, hipStream_t s)
{
    return launch_attention_of<PageKernels>(p, c, b, part, s);
}

}  // namespace lpq

// Paged caches: the plan of a step (block tables, slots and positions from the requests' lengths) and the append of its K and V to the
// pages.  Both are bound by latency in a decode step; the append of long prompts is a copy at the memory's rate.
#include <algorithm>

#include "lpq_common.h"
#include "lpq_device.h"
#include "lpq_paged_index.h"

namespace lpq {

namespace {

// ---- the plan ---------------------------------------------------------------------------------
// With q = max(q_lens, 0), n = past + q, page size P and a table of W entries per sequence:
//   offsets    cu[s] = sum of q before s, at most M
//   owned      min(ceil(past / P), W);  need = ceil(n / P) - owned if q > 0
//   starved    rows end behind M, n > W P, or need > 0 and the sum of the needs up to s exceeds the free pages
// 2.9 us for one sequence, 4.3 for 64 that decode, 8.1 for 1000: kernel start and end and a chain of loads (lengths, scan, table, store).
// One workgroup: all of it hangs on three prefix sums over the sequences, which are a handful of numbers per thread; what is left is
// a search (in LDS) per new page, returned page and row.  The lengths and the pool's counters may be updated in place: every thread has read what
// it needs of them ahead of the first barrier.
constexpr int PLAN_THREADS = 1024;
constexpr int ROWS_AHEAD = 4;                         // of a thread
constexpr uint32_t SUM_CAP = 1u << 30;                 // sums stop here: above any number of rows or pages that can be served

__device__ __forceinline__ uint32_t capped_add(uint32_t a, uint32_t b) { return min(a + b, SUM_CAP); }

// Exclusive prefix sums of v0 (sequence 2 t) and v1 (2 t + 1) over the workgroup, and the total.  part: a word per wave.
struct Scan { uint32_t before, total; };
__device__ __forceinline__ Scan block_scan(uint32_t v, uint32_t* part)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = (blockDim.x + 63) >> 6;
    uint32_t sum = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t o = (uint32_t)__shfl_up((int)sum, d);
        if (lane >= d) sum = capped_add(sum, o);
    }
    const uint32_t prev = (uint32_t)__shfl_up((int)sum, 1);
    Scan r{lane ? prev : 0u, 0u};
    if (waves == 1) {
        r.total = (uint32_t)__shfl((int)sum, 63);
        return r;
    }
    if (lane == 63) part[wave] = sum;
    __syncthreads();
    uint32_t base = 0;
    for (int w = 0; w < waves; ++w) {
        const uint32_t p = part[w];
        if (w < wave) base = capped_add(base, p);
        r.total = capped_add(r.total, p);
    }
    r.before = capped_add(base, r.before);
    return r;
}

// The last sequence whose prefix sum is at most i[k] (prefix[0] is 0): of several with the same sum, the one that has elements.  N searches side by side,
// each a chain of LDS reads; top: the largest power of two below n, or 0.
template <int N>
__device__ __forceinline__ void last_at_most(const uint32_t* prefix, int n, int top, const uint32_t (&i)[N], int (&s)[N])
{
#pragma unroll
    for (int k = 0; k < N; ++k) s[k] = 0;
    for (int d = top; d; d >>= 1)
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int at = s[k] + d;
            if (prefix[min(at, n - 1)] <= i[k] && at < n) s[k] = at;
        }
}

__device__ __forceinline__ int ring_at(uint32_t at, int n_pages) { return at >= (uint32_t)n_pages ? (int)(at - n_pages) : (int)at; }

struct PlanArgs {
    const int32_t *past, *q_lens, *counters;
    int32_t *table, *ring, *counters_out, *cu_q, *kv_lens, *slots, *positions, *info;
    int32_t n, M, shift, n_pages, width;
};

__device__ __forceinline__ void write_row(const PlanArgs& a, int r, int page, int pos)
{
    const int id = page_checked(page, a.n_pages);
    a.slots[r] = id < 0 ? -1 : (id << a.shift) + (pos & ((1 << a.shift) - 1));
    a.positions[r] = pos;
}

// The rows of a long batch have a launch of their own behind the rest, whose workgroups need to know which sequences are starved and the others' cached
// positions, and the lengths may have been updated in place.  Each finds that (-1: starved) in its own rows' slots: in the first row that a sequence has of
// them.  Nothing is kept outside of the caller's buffers, so plans may overlap any call that leaves those alone.
constexpr int PLAN_ROWS_PER_WG = 256 * ROWS_AHEAD;

template <bool ROWS_APART>
__global__ __launch_bounds__(PLAN_THREADS) void paged_plan_kernel(PlanArgs a)
{
    __shared__ uint32_t cu[PAGED_MAX_SEQS], need_before[PAGED_MAX_SEQS], back_before[PAGED_MAX_SEQS];
    __shared__ int32_t base[PAGED_MAX_SEQS];
    __shared__ uint32_t part[3][PLAN_THREADS / 64];
    __shared__ uint32_t taken_s, starved_s;
    const int tid = threadIdx.x, n = a.n, P = 1 << a.shift;
    const int64_t room = (int64_t)a.width << a.shift;
    if (tid == 0) taken_s = 0, starved_s = 0;
    int head = a.counters[0], free_pages = a.counters[1];
    free_pages = clamp_int(free_pages, 0, a.n_pages);
    head = head < 0 ? 0 : head % a.n_pages;
    int past[2], q[2], owned[2];
    bool done[2];
    uint32_t rows[2], back[2], need[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int s = 2 * tid + i;
        past[i] = s < n ? max(a.past[s], 0) : 0;
        const int ql = s < n ? a.q_lens[s] : 0;
        done[i] = ql < 0;
        q[i] = max(ql, 0);
        owned[i] = (int)min<int64_t>(((int64_t)past[i] + P - 1) >> a.shift, a.width);
        rows[i] = min((uint32_t)q[i], SUM_CAP);
        back[i] = done[i] ? (uint32_t)owned[i] : 0u;
    }
    const Scan sr = block_scan(capped_add(rows[0], rows[1]), part[0]), sb = block_scan(capped_add(back[0], back[1]), part[1]);
    bool late[2];
    uint32_t before = sr.before;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int s = 2 * tid + i;
        if (s < n) {
            cu[s] = before;
            back_before[s] = i ? capped_add(sb.before, back[0]) : sb.before;
            a.cu_q[s] = (int)min(before, (uint32_t)a.M);
        }
        before = capped_add(before, rows[i]);
        const int64_t total = (int64_t)past[i] + q[i];
        late[i] = q[i] > 0 && (before > (uint32_t)a.M || total > room);
        need[i] = q[i] > 0 && !late[i] ? (uint32_t)(((total + P - 1) >> a.shift) - owned[i]) : 0u;
    }
    const Scan sn = block_scan(capped_add(need[0], need[1]), part[2]);      // a barrier, if there is more than a wave: taken_s is zero
    uint32_t sum = sn.before;
    uint32_t n_starved = 0, most = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int s = 2 * tid + i;
        if (s >= n) break;
        need_before[s] = sum;
        sum = capped_add(sum, need[i]);
        const bool starved = late[i] || (need[i] > 0 && sum > (uint32_t)free_pages);
        if (need[i] > 0 && !starved) most = sum;
        n_starved += starved;
        base[s] = starved ? -1 : past[i];
        if (ROWS_APART && q[i] > 0 && cu[s] < (uint32_t)a.M) a.slots[cu[s]] = base[s];
        a.kv_lens[s] = done[i] ? 0 : starved ? past[i] : past[i] + q[i];
    }
    if (most) atomicMax(&taken_s, most);
    if (n_starved) atomicAdd(&starved_s, n_starved);
    __syncthreads();
    const int taken = (int)taken_s, returned = (int)min(sb.total, (uint32_t)(a.n_pages - free_pages)), total_rows = (int)min(sr.total, (uint32_t)a.M);
    if (tid == 0) {
        a.cu_q[n] = total_rows;
        a.counters_out[0] = ring_at((uint32_t)head + (uint32_t)taken, a.n_pages);
        a.counters_out[1] = free_pages - taken + returned;
        a.info[0] = total_rows;
        a.info[1] = taken;
        a.info[2] = returned;
        a.info[3] = (int)starved_s;
    }
    const int top = n > 1 ? 1 << (31 - __builtin_clz(n - 1)) : 0, threads = (int)blockDim.x - (ROWS_APART ? 64 : 0);
    if (ROWS_APART && tid >= threads) {                // the last wave, beside the others
        for (int r = (tid - threads) * PLAN_ROWS_PER_WG; r < total_rows; r += 64 * PLAN_ROWS_PER_WG) {
            int s[1];
            last_at_most<1>(cu, n, top, {(uint32_t)r}, s);
            a.slots[r] = base[s[0]];
        }
        return;
    }
    for (int i = tid; i < taken; i += threads) {
        int s[1];
        last_at_most<1>(need_before, n, top, {(uint32_t)i}, s);
        const int e = ((base[s[0]] + P - 1) >> a.shift) + (i - (int)need_before[s[0]]);
        a.table[(size_t)s[0] * a.width + e] = a.ring[ring_at((uint32_t)head + (uint32_t)i, a.n_pages)];
    }
    // behind the free pages: no entry that is read here, as no more are returned than the ring has room for
    for (int i = tid; i < returned; i += threads) {
        int s[1];
        last_at_most<1>(back_before, n, top, {(uint32_t)i}, s);
        const uint32_t at = (uint32_t)head + (uint32_t)free_pages;
        a.ring[ring_at((uint32_t)ring_at(at, a.n_pages) + (uint32_t)i, a.n_pages)] = a.table[(size_t)s[0] * a.width + (i - (int)back_before[s[0]])];
    }
    if constexpr (ROWS_APART) return;
    for (int r0 = tid; r0 < a.M; r0 += ROWS_AHEAD * threads) {
        uint32_t r[ROWS_AHEAD];
        int s[ROWS_AHEAD], pos[ROWS_AHEAD], page[ROWS_AHEAD];
#pragma unroll
        for (int k = 0; k < ROWS_AHEAD; ++k) r[k] = (uint32_t)(r0 + k * threads);
        last_at_most<ROWS_AHEAD>(cu, n, top, r, s);
#pragma unroll
        for (int k = 0; k < ROWS_AHEAD; ++k) {
            page[k] = -1;
            pos[k] = 0;
            if (r[k] >= (uint32_t)total_rows || base[s[k]] < 0) continue;
            pos[k] = base[s[k]] + (int)(r[k] - cu[s[k]]);
            const int e = pos[k] >> a.shift, held = (base[s[k]] + P - 1) >> a.shift;
            // a new page's entry may not be in the table yet: from the ring
            page[k] = e < held ? a.table[(size_t)s[k] * a.width + e] : a.ring[ring_at((uint32_t)head + need_before[s[k]] + (uint32_t)(e - held), a.n_pages)];
        }
#pragma unroll
        for (int k = 0; k < ROWS_AHEAD; ++k)
            if (r[k] < (uint32_t)a.M) write_row(a, (int)r[k], page[k], pos[k]);
    }
}

// The rows of a long batch, behind the kernel above: the table is complete.
__global__ __launch_bounds__(256) void paged_plan_rows_kernel(PlanArgs a)
{
    __shared__ uint32_t cu[PAGED_MAX_SEQS];
    for (int s = threadIdx.x; s < a.n; s += 256) cu[s] = (uint32_t)a.cu_q[s];
    const uint32_t total = (uint32_t)a.cu_q[a.n], from = blockIdx.x * (uint32_t)PLAN_ROWS_PER_WG;
    __syncthreads();
    const int top = a.n > 1 ? 1 << (31 - __builtin_clz(a.n - 1)) : 0;
    uint32_t r[ROWS_AHEAD];
    int s[ROWS_AHEAD], base[ROWS_AHEAD], pos[ROWS_AHEAD], page[ROWS_AHEAD];
#pragma unroll
    for (int k = 0; k < ROWS_AHEAD; ++k) r[k] = from + 256u * k + threadIdx.x;
    last_at_most<ROWS_AHEAD>(cu, a.n, top, r, s);
#pragma unroll
    for (int k = 0; k < ROWS_AHEAD; ++k) base[k] = r[k] < total ? a.slots[max(cu[s[k]], from)] : -1;
    __syncthreads();                                   // they have been read: the slots can be written
#pragma unroll
    for (int k = 0; k < ROWS_AHEAD; ++k) {
        page[k] = -1;
        pos[k] = 0;
        if (base[k] < 0) continue;
        pos[k] = base[k] + (int)(r[k] - cu[s[k]]);
        page[k] = a.table[(size_t)s[k] * a.width + min(pos[k] >> a.shift, a.width - 1)];
    }
#pragma unroll
    for (int k = 0; k < ROWS_AHEAD; ++k)
        if (r[k] < (uint32_t)a.M) write_row(a, (int)r[k], page[k], pos[k]);
}

// ---- the append: each row's K and V parts to its slot, 16 bytes a thread at a time ----------------
// Rows without a slot are skipped.
template <int D>
__global__ __launch_bounds__(256) void paged_append_kernel(const uint16_t* __restrict__ qkv, uint16_t* __restrict__ kp, uint16_t* __restrict__ vp,
                                                           const int32_t* __restrict__ slots, int M, int H, int KV, int shift, int n_pages)
{
    constexpr int CH = D / 8;                          // 16-byte chunks of a head
    const int per_row = KV * CH, cols = (H + 2 * KV) * D;
    const uint32_t i = blockIdx.x * 256u + threadIdx.x, row = i / (uint32_t)per_row;      // below 2^31: the host's bound on M
    if (row >= (uint32_t)M) return;
    const int c = (int)(i - row * (uint32_t)per_row), h = c / CH;
    const uint16_t* src = qkv + (size_t)row * cols + H * D + 8 * c;
    const u32x4 k = *reinterpret_cast<const u32x4*>(src), v = *reinterpret_cast<const u32x4*>(src + KV * D);
    const int slot = slot_checked(slots[row], n_pages, shift);
    if (slot < 0) return;
    const size_t at = (size_t)page_element(slot >> shift, h, KV, shift, D) + (size_t)(slot & ((1 << shift) - 1)) * D + 8 * (c % CH);
    *reinterpret_cast<u32x4*>(kp + at) = k;
    *reinterpret_cast<u32x4*>(vp + at) = v;
}

}  // namespace

// One launch / the rows in one of their own, us: 16 sequences, 4096 rows 8.1 / 8.7, 6144 rows 9.6 / 8.8; one sequence, 4096 rows 7.0 / 7.2, 8000 8.5 / 7.4; 300, 3900
// rows 10.2 / 10.8, 6000 13.1 / 11.4; 2000, 6000 rows 13.6 / 14.3, 12000 18.5 / 14.9.
constexpr int PLAN_ONE_LAUNCH_ROWS = 6144;

hipError_t launch_paged_plan(const lpq_page_pool& pool, int shift, const int32_t* past, const int32_t* q_lens, int n_seqs, int M, const lpq_page_plan& out,
                             hipStream_t s)
{
    const PlanArgs a{past, q_lens, pool.counters, pool.table, pool.ring, out.counters, out.cu_q, out.kv_lens, out.slots, out.positions, out.info,
                     n_seqs, M, shift, pool.n_pages, pool.max_pages};
    // threads for the sequences (two each) and, up to sixteen waves, for the rows (with a launch of their own: for the new pages)
    const bool apart = M > PLAN_ONE_LAUNCH_ROWS;
    const int want = std::max((n_seqs + 1) / 2, apart ? 512 + 64 : M), threads = std::min(PLAN_THREADS, (want + 63) / 64 * 64);
    if (apart) {
        paged_plan_kernel<true><<<1, threads, 0, s>>>(a);
        paged_plan_rows_kernel<<<(unsigned)((M + PLAN_ROWS_PER_WG - 1) / PLAN_ROWS_PER_WG), 256, 0, s>>>(a);
    } else paged_plan_kernel<false><<<1, threads, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_paged_append(const void* qkv, const lpq_attn_cfg& c, int shift, int n_pages, void* k_pages, void* v_pages, const int32_t* slots, int M,
                               hipStream_t s)
{
    const uint16_t* q = static_cast<const uint16_t*>(qkv);
    uint16_t *k = static_cast<uint16_t*>(k_pages), *v = static_cast<uint16_t*>(v_pages);
    const int64_t chunks = (int64_t)M * c.n_kv_heads * (c.head_dim / 8);
    const unsigned grid = (unsigned)((chunks + 255) / 256);
    if (c.head_dim == 128) paged_append_kernel<128><<<grid, 256, 0, s>>>(q, k, v, slots, M, c.n_heads, c.n_kv_heads, shift, n_pages);
    else                   paged_append_kernel<64><<<grid, 256, 0, s>>>(q, k, v, slots, M, c.n_heads, c.n_kv_heads, shift, n_pages);
    return hipGetLastError();
}

}  // namespace lpq

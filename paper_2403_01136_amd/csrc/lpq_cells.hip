// What a layer does with its rows around a 4-bit paged cache: norms of q and k for each head with the rotation of their positions, the append that quantises K and V
// into cells, and its inverse.  All three move bytes: a thread has 16 or 32 bytes of a head, a head's lanes are neighbours and share sums and
// extremes by lane exchanges, nothing goes through LDS.
#include "lpq_batch_attention.h"

namespace lpq {

namespace {

// ---- norms and rotation ---------------------------------------------------------------------------
// y = x / sqrt(mean(x^2) + eps) * gamma for q and k of each head, then for the head's first rotary_dim features, a pair (a, b) at angle i:
//     (a cos - b sin, b cos + a sin)
// all of it in fp32, rounded once.  A thread has two chunks of eight features: of paired halves one of either, so that both of a pair are its own.
struct RotaryArgs {
    const uint16_t* in;
    uint16_t* out;
    const int32_t *positions, *slots;
    const float* table;
    const uint16_t *q_gamma, *k_gamma;
    float eps;
    int M, H, KV, heads;                 // heads that are written: with V's where out is not in
    int turned, max_pos, groups;         // rotary_dim; groups of heads, a wave each
};

template <int DT> __device__ __forceinline__ void to_floats(const u32x4& x, float* v)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[2 * e] = param_scale<DT>(x[e]);
        v[2 * e + 1] = param_zero<DT>(x[e]);
    }
}
template <int DT> __device__ __forceinline__ u32x4 from_floats(const float* v)
{
    u32x4 x;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = Elem<DT>::pack(v[2 * e], v[2 * e + 1]);
    return x;
}

// Bound by the memory: rows in and out, 16 bytes a load.  A wave has 8 heads (D = 128) of a row once: 4168 rows of 120 heads, every byte of them, 47.4 us (5.4 TB/s), with two
// such turns a wave, sharing the angles, 51.9, with four 50.0; 43 rows of 72 heads 3.3, 3.8, 4.9.
template <int DT, int D, bool ADJACENT>
__global__ __launch_bounds__(256) void qk_norm_rotary_kernel(RotaryArgs a)
{
    constexpr int LANES = D / 16, SLOTS = 64 / LANES;  // lanes of a head; heads of a wave
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)((blockIdx.y * gridDim.x + blockIdx.x) * 4 + threadIdx.x / 64));
    const int row = wave / a.groups, h = wave % a.groups * SLOTS + lane / LANES;
    if (row >= a.M || (a.slots && a.slots[row] < 0)) return;
    const int p = a.turned ? a.positions[row] : 0;
    if (a.turned && (uint32_t)p >= (uint32_t)a.max_pos) return;
    if (h >= a.heads) return;                          // all lanes of a head
    const int li = lane % LANES, half = a.turned / 16;                           // chunks of half a turned part
    const bool turn = li < half && h < a.H + a.KV;
    const int c0 = ADJACENT ? 2 * li : li < half ? li : 2 * half + 2 * (li - half), c1 = ADJACENT || li >= half ? c0 + 1 : li + half;
    const size_t at = ((size_t)row * (a.H + 2 * a.KV) + h) * D;
    u32x4 x0 = *reinterpret_cast<const u32x4*>(a.in + at + 8 * c0), x1 = *reinterpret_cast<const u32x4*>(a.in + at + 8 * c1);
    if (h < a.H + a.KV) {
        float v[16];
        to_floats<DT>(x0, v);
        to_floats<DT>(x1, v + 8);
        const uint16_t* gamma = h < a.H ? a.q_gamma : a.k_gamma;
        if (gamma) {
            float ss = 0.0f, g[16];
            to_floats<DT>(*reinterpret_cast<const u32x4*>(gamma + 8 * c0), g);
            to_floats<DT>(*reinterpret_cast<const u32x4*>(gamma + 8 * c1), g + 8);
#pragma unroll
            for (int e = 0; e < 16; ++e) ss = __builtin_fmaf(v[e], v[e], ss);
            ss = group_reduce<LANES>(ss, OpAdd());
            const float r = 1.0f / sqrtf(ss * (1.0f / D) + a.eps);
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] = v[e] * r * g[e];
        }
        if (turn) {
            const f4 *t = reinterpret_cast<const f4*>(a.table + (size_t)p * a.turned + 8 * li), *u = reinterpret_cast<const f4*>(a.table + (size_t)p * a.turned + a.turned / 2 + 8 * li);
            const f4 cs[2] = {t[0], t[1]}, sn[2] = {u[0], u[1]};                 // angles 8 li .. 8 li + 7
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float c = cs[i / 4][i % 4], s = sn[i / 4][i % 4];
                float &va = v[ADJACENT ? 2 * i : i], &vb = v[ADJACENT ? 2 * i + 1 : 8 + i];
                const float ra = va * c - vb * s, rb = vb * c + va * s;
                va = ra;
                vb = rb;
            }
        }
        x0 = from_floats<DT>(v);
        x1 = from_floats<DT>(v + 8);
    }
    *reinterpret_cast<u32x4*>(a.out + at + 8 * c0) = x0;
    *reinterpret_cast<u32x4*>(a.out + at + 8 * c1) = x1;
}

// ---- cells ------------------------------------------------------------------------------------------
// A thread has eight features of a row's K head and of the V head (the append: 16), neighbours the whole heads.
struct CellArgs {
    uint16_t* qkv;
    uint8_t *kp, *vp;
    const int32_t* slots;
    int M, H, KV, shift, n_pages;
};
struct Cell { uint16_t* row; int head, chunk, slot; };                           // K's features in the row, null behind the last one; slot as the caller gave it
// TOGETHER rows of one head are neighbours, then come the other heads, then the next rows.
template <int D, int FEATURES, int TOGETHER> __device__ __forceinline__ Cell cell_of(const CellArgs& a)
{
    constexpr int LANES = D / FEATURES;
    const uint32_t i = (blockIdx.x * 256u + threadIdx.x) / LANES, rows = i / ((uint32_t)a.KV * TOGETHER) * TOGETHER, n = i - rows * (uint32_t)a.KV;      // below 2^31: the host's bound on M
    const uint32_t h = n / TOGETHER, row = rows + n % TOGETHER, chunk = threadIdx.x % LANES;
    if (row >= (uint32_t)a.M) return Cell{};
    return Cell{a.qkv + (size_t)row * ((a.H + 2 * a.KV) * D) + (a.H + h) * D + FEATURES * chunk, (int)h, (int)chunk, a.slots[row]};
}
// Where the cell's group of 16 positions begins; its slot is one.
template <int D> __device__ __forceinline__ size_t group_of(const CellArgs& a, const Cell& c)
{
    return (size_t)cell_group(c.slot >> a.shift, c.head, a.KV, a.shift, (c.slot & ((1 << a.shift) - 1)) >> 4, D);
}

// Codes and parameters of a head of which this lane has 16 features:
//     scale = type((max - min) / 15), a last place less if 15 scales above zero would round to infinity;  zero = min;
//     code = clamp(rint((x - zero) / scale), 0, 15), 0 where scale is
// with quotients rounded to fp32, made without a division: of q = a / s, q0 = a rcp(s) is off by 1.5 2^-23 of it at most, the remainder a - q0 s is exact in one FMA (s has eleven bits),
// and q0 + remainder * rcp(s) before its rounding by 2^-45 of q.  That rounds as the quotient does: where a rounds differently above than below, a / s is half way between two fp32
// numbers, a number m of 25 bits; a - m s, of numbers of 24 and 36 bits, is zero or 2^-37 of a at least, and zero it is not, as m s has more than 24 bits.  Scales below 2^-100, where
// the remainder may be too small for an exponent, divide.
// A head with an infinity or a NaN in it, or (in bf16) a range beyond fp32, is NaN throughout.
template <int DT, int LANES>
__device__ __forceinline__ u32x2 quantise_head(const u32x4 (&x)[2], uint32_t* param)
{
    typedef typename Elem<DT>::t T;
    constexpr int N = 16;
    float v[N], lo, hi, probe = 0.0f;
    to_floats<DT>(x[0], v);
    to_floats<DT>(x[1], v + 8);
    lo = hi = v[0];
#pragma unroll
    for (int e = 1; e < N; ++e) {
        lo = fminf(lo, v[e]);
        hi = fmaxf(hi, v[e]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) probe = Elem<DT>::probe_pair(x[e / 4][e % 4], probe);
    struct OpMin { __device__ __forceinline__ float operator()(float a, float b) const { return fminf(a, b); } };
    lo = group_reduce<LANES>(lo, OpMin());
    hi = group_reduce<LANES>(hi, OpMax());
    const T scale = (T)__fdiv_rn(__fsub_rn(hi, lo), 15.0f), zero = (T)__fadd_rn(lo, 0.0f);      // lo is a number of the type; -0 becomes 0
    uint16_t sb = __builtin_bit_cast(uint16_t, scale);
    const uint16_t zb = __builtin_bit_cast(uint16_t, zero);
    const float z = (float)zero;
    const uint64_t bad_lanes = __ballot(probe != probe);
    const bool odd = (bad_lanes >> (threadIdx.x & 63 & -LANES) & ((1ull << LANES) - 1)) != 0 || !__builtin_isfinite((float)scale);
    if (!odd && __builtin_isinf((float)(T)__builtin_fmaf(15.0f, (float)scale, z))) --sb;
    const float s = (float)__builtin_bit_cast(T, sb);
    const float rcp = __builtin_amdgcn_rcpf(s);
    float r[N];
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const float a = __fsub_rn(v[e], z), q0 = __fmul_rn(a, rcp);
        r[e] = __builtin_fmaf(__builtin_fmaf(-q0, s, a), rcp, q0);
    }
    if constexpr (DT == LPQ_DT_BF16)                   // fp16 has no such scales
        if (__any(s > 0.0f && s < 0x1p-100f))
#pragma unroll
            for (int e = 0; e < N; ++e) r[e] = __fdiv_rn(__fsub_rn(v[e], z), s);
#pragma unroll
    for (int e = 0; e < N; ++e) r[e] = __builtin_rintf(__builtin_amdgcn_fmed3f(r[e], 0.0f, 15.0f));
    // code e at bit 4 (e / 2) of its half: sums below 2^16, exact
    auto half = [&](int e) { return (uint32_t)__builtin_fmaf(r[e + 6], 4096.0f, __builtin_fmaf(r[e + 4], 256.0f, __builtin_fmaf(r[e + 2], 16.0f, r[e]))); };
    constexpr uint32_t NOT_A_NUMBER = DT == LPQ_DT_FP16 ? 0x7e007e00u : 0x7fc07fc0u;
    *param = odd ? NOT_A_NUMBER : (uint32_t)sb | (uint32_t)zb << 16;
    return odd || sb == 0 ? u32x2{0, 0} : u32x2{half(0) | half(1) << 16, half(8) | half(9) << 16};
}

// Bound by the memory, of which its reads are most (256 bytes of a row and head at D = 128); what it writes lies in the order of positions, so 16 rows of a head are neighbours here:
// a group's codes and parameters are whole lines of one XCD's L2.  7246 rows of 8 heads: row by row, eight features a thread and IEEE divisions near halves, 14.4 us; 16 features, no divisions 12.8; so 12.6; quotients by a remainder instead of
// whole numbers and a test of doubt 10.6 (3.5 TB/s read and written).
constexpr int APPEND_TOGETHER = 16;
template <int DT, int D>
__global__ __launch_bounds__(256) void paged_append4_kernel(CellArgs a)
{
    const Cell c = cell_of<D, 16, APPEND_TOGETHER>(a);
    if (!c.row) return;                                // all lanes of a head or none, here as below
    const u32x4 *kr = reinterpret_cast<const u32x4*>(c.row), *vr = reinterpret_cast<const u32x4*>(c.row + a.KV * D);
    const u32x4 k[2] = {kr[0], kr[1]}, v[2] = {vr[0], vr[1]};
    if (slot_checked(c.slot, a.n_pages, a.shift) < 0) return;
    uint32_t kparam, vparam;
    const u32x2 kw = quantise_head<DT, D / 16>(k, &kparam), vw = quantise_head<DT, D / 16>(v, &vparam);
    const size_t group = group_of<D>(a, c);
    uint8_t *kg = a.kp + group, *vg = a.vp + group;
    const int at = c.slot & 15;
    *reinterpret_cast<u32x2*>(kg + at * (D / 2) + 8 * c.chunk) = kw;
    *reinterpret_cast<u32x2*>(vg + at * (D / 2) + 8 * c.chunk) = vw;
    if (c.chunk == 0) {
        *reinterpret_cast<uint32_t*>(kg + 8 * D + 4 * at) = kparam;
        *reinterpret_cast<uint32_t*>(vg + 8 * D + 4 * at) = vparam;
    }
}

template <int DT, int D>
__global__ __launch_bounds__(256) void paged_load4_kernel(CellArgs a)
{
    const Cell c = cell_of<D, 8, 1>(a);
    if (!c.row || slot_checked(c.slot, a.n_pages, a.shift) < 0) return;
    const size_t group = group_of<D>(a, c);
    const uint8_t *kg = a.kp + group, *vg = a.vp + group;
    const int at = c.slot & 15;
    const uint32_t kw = *reinterpret_cast<const uint32_t*>(kg + at * (D / 2) + 4 * c.chunk), vw = *reinterpret_cast<const uint32_t*>(vg + at * (D / 2) + 4 * c.chunk);
    const uint32_t kparam = *reinterpret_cast<const uint32_t*>(kg + 8 * D + 4 * at), vparam = *reinterpret_cast<const uint32_t*>(vg + 8 * D + 4 * at);
    *reinterpret_cast<u32x4*>(c.row) = cell_values<DT>(kw, kparam);
    *reinterpret_cast<u32x4*>(c.row + a.KV * D) = cell_values<DT>(vw, vparam);
}

template <int DT, int D>
hipError_t launch_rotary(RotaryArgs a, bool adjacent, hipStream_t s)
{
    constexpr int SLOTS = 64 / (D / 16);
    a.groups = (a.heads + SLOTS - 1) / SLOTS;
    // M heads are at most 2^27, so waves fit 32 bits; threads need not
    const unsigned blocks = (unsigned)(((int64_t)a.M * a.groups + 3) / 4), across = std::min(blocks, 1u << 23);
    const dim3 grid(across, (blocks + across - 1) / across);
    if (adjacent) qk_norm_rotary_kernel<DT, D, true><<<grid, 256, 0, s>>>(a);
    else          qk_norm_rotary_kernel<DT, D, false><<<grid, 256, 0, s>>>(a);
    return hipGetLastError();
}

template <bool APPEND, int DT, int D>
hipError_t launch_cells_of(const CellArgs& a, hipStream_t s)
{
    const int64_t rows = APPEND ? ((int64_t)a.M + APPEND_TOGETHER - 1) / APPEND_TOGETHER * APPEND_TOGETHER : a.M;
    const unsigned grid = (unsigned)((rows * a.KV * (D / (APPEND ? 16 : 8)) + 255) / 256);
    if constexpr (APPEND) paged_append4_kernel<DT, D><<<grid, 256, 0, s>>>(a);
    else                  paged_load4_kernel<DT, D><<<grid, 256, 0, s>>>(a);
    return hipGetLastError();
}
template <bool APPEND>
hipError_t launch_cells(const lpq_attn_cfg& c, const CellArgs& a, hipStream_t s)
{
    if (c.dtype == LPQ_DT_FP16) return c.head_dim == 128 ? launch_cells_of<APPEND, LPQ_DT_FP16, 128>(a, s) : launch_cells_of<APPEND, LPQ_DT_FP16, 64>(a, s);
    return c.head_dim == 128 ? launch_cells_of<APPEND, LPQ_DT_BF16, 128>(a, s) : launch_cells_of<APPEND, LPQ_DT_BF16, 64>(a, s);
}

}  // namespace

hipError_t launch_qk_norm_rotary(const void* qkv, const lpq_attn_cfg& c, const lpq_rotary& r, const int32_t* positions, const int32_t* slots, int M, void* out,
                                 hipStream_t s)
{
    if (qkv == out && r.rotary_dim == 0 && !r.q_gamma && !r.k_gamma) return hipSuccess;
    RotaryArgs a{};
    a.in = static_cast<const uint16_t*>(qkv);
    a.out = static_cast<uint16_t*>(out);
    a.positions = positions;
    a.slots = slots;
    a.table = r.cos_sin;
    a.q_gamma = static_cast<const uint16_t*>(r.q_gamma);
    a.k_gamma = static_cast<const uint16_t*>(r.k_gamma);
    a.eps = r.eps;
    a.M = M;
    a.H = c.n_heads;
    a.KV = c.n_kv_heads;
    a.heads = c.n_heads + (qkv == out ? 1 : 2) * c.n_kv_heads;
    a.turned = r.rotary_dim;
    a.max_pos = r.max_pos;
    const bool adjacent = r.pairs == LPQ_PAIRS_ADJACENT;
    if (c.dtype == LPQ_DT_FP16) return c.head_dim == 128 ? launch_rotary<LPQ_DT_FP16, 128>(a, adjacent, s) : launch_rotary<LPQ_DT_FP16, 64>(a, adjacent, s);
    return c.head_dim == 128 ? launch_rotary<LPQ_DT_BF16, 128>(a, adjacent, s) : launch_rotary<LPQ_DT_BF16, 64>(a, adjacent, s);
}

hipError_t launch_paged_append4(const void* qkv, const lpq_attn_cfg& c, int shift, int n_pages, void* k_pages, void* v_pages, const int32_t* slots, int M,
                                hipStream_t s)
{
    return launch_cells<true>(c, CellArgs{static_cast<uint16_t*>(const_cast<void*>(qkv)), static_cast<uint8_t*>(k_pages), static_cast<uint8_t*>(v_pages), slots, M,
                                          c.n_heads, c.n_kv_heads, shift, n_pages}, s);
}

hipError_t launch_paged_load4(const void* k_pages, const void* v_pages, const lpq_attn_cfg& c, int shift, int n_pages, const int32_t* slots, int M, void* qkv,
                              hipStream_t s)
{
    return launch_cells<false>(c, CellArgs{static_cast<uint16_t*>(qkv), static_cast<uint8_t*>(const_cast<void*>(k_pages)), static_cast<uint8_t*>(const_cast<void*>(v_pages)),
                                           slots, M, c.n_heads, c.n_kv_heads, shift, n_pages}, s);
}

}  // namespace lpq

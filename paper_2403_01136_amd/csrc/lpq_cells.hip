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

template <int DT, int D, bool ADJACENT, int HEADS>
__global__ __launch_bounds__(256) void qk_norm_rotary_kernel(RotaryArgs a)
{
    constexpr int LANES = D / 16, SLOTS = 64 / LANES;  // lanes of a head; heads of a wave at a time, HEADS times
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + threadIdx.x / 64));
    const int row = wave / a.groups, group = wave % a.groups;
    if (row >= a.M || (a.slots && a.slots[row] < 0)) return;
    const int p = a.turned ? a.positions[row] : 0;
    if (a.turned && (uint32_t)p >= (uint32_t)a.max_pos) return;
    const int li = lane % LANES, half = a.turned / 16;                           // chunks of half a turned part
    const bool turn = li < half;
    const int c0 = ADJACENT ? 2 * li : turn ? li : 2 * half + 2 * (li - half), c1 = ADJACENT || !turn ? c0 + 1 : li + half;
    f4 cs[2], sn[2];                                                             // angles 8 li .. 8 li + 7
    if (turn) {
        const f4* t = reinterpret_cast<const f4*>(a.table + (size_t)p * a.turned + 8 * li);
        cs[0] = t[0], cs[1] = t[1];
        t = reinterpret_cast<const f4*>(a.table + (size_t)p * a.turned + a.turned / 2 + 8 * li);
        sn[0] = t[0], sn[1] = t[1];
    }
    const size_t base = (size_t)row * ((a.H + 2 * a.KV) * D);
    u32x4 x[HEADS][2];
#pragma unroll
    for (int n = 0; n < HEADS; ++n) {
        const int h = (group * HEADS + n) * SLOTS + lane / LANES;
        if (h >= a.heads) continue;
        x[n][0] = *reinterpret_cast<const u32x4*>(a.in + base + h * D + 8 * c0);
        x[n][1] = *reinterpret_cast<const u32x4*>(a.in + base + h * D + 8 * c1);
    }
#pragma unroll
    for (int n = 0; n < HEADS; ++n) {
        const int h = (group * HEADS + n) * SLOTS + lane / LANES;
        const uint16_t* gamma = h < a.H ? a.q_gamma : h < a.H + a.KV ? a.k_gamma : nullptr;
        if (h < a.H + a.KV) {
            float v[16];
            to_floats<DT>(x[n][0], v);
            to_floats<DT>(x[n][1], v + 8);
            if (gamma) {
                float ss = 0.0f;
#pragma unroll
                for (int e = 0; e < 16; ++e) ss = __builtin_fmaf(v[e], v[e], ss);
                ss = group_reduce<LANES>(ss, OpAdd());
                const float r = 1.0f / sqrtf(ss * (1.0f / D) + a.eps);
                float g[16];
                to_floats<DT>(*reinterpret_cast<const u32x4*>(gamma + 8 * c0), g);
                to_floats<DT>(*reinterpret_cast<const u32x4*>(gamma + 8 * c1), g + 8);
#pragma unroll
                for (int e = 0; e < 16; ++e) v[e] = v[e] * r * g[e];
            }
            if (turn)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float c = cs[i / 4][i % 4], s = sn[i / 4][i % 4];
                    float &va = v[ADJACENT ? 2 * i : i], &vb = v[ADJACENT ? 2 * i + 1 : 8 + i];
                    const float ra = va * c - vb * s, rb = vb * c + va * s;
                    va = ra;
                    vb = rb;
                }
            x[n][0] = from_floats<DT>(v);
            x[n][1] = from_floats<DT>(v + 8);
        }
        if (h >= a.heads) continue;
        *reinterpret_cast<u32x4*>(a.out + base + h * D + 8 * c0) = x[n][0];
        *reinterpret_cast<u32x4*>(a.out + base + h * D + 8 * c1) = x[n][1];
    }
}

// ---- cells ------------------------------------------------------------------------------------------
// A thread has eight features of a row's K head and of the V head, LANES neighbours the whole heads.
struct CellArgs {
    uint16_t* qkv;
    uint8_t *kp, *vp;
    const int32_t* slots;
    int M, H, KV, shift, n_pages;
};
struct Cell { bool any; uint16_t* row; size_t group; int at, chunk; };           // K's eight features in the row; the 16-position group and the place in it
template <int D> __device__ __forceinline__ Cell cell_of(const CellArgs& a)
{
    constexpr int LANES = D / 8;
    const int per_row = a.KV * LANES;
    const uint32_t i = blockIdx.x * 256u + threadIdx.x, row = i / (uint32_t)per_row;      // below 2^31: the host's bound on M
    Cell c{};
    if (row >= (uint32_t)a.M) return c;
    const int n = (int)(i - row * (uint32_t)per_row), h = n / LANES, slot = slot_checked(a.slots[row], a.n_pages, a.shift);
    if (slot < 0) return c;
    c.any = true;
    c.chunk = n % LANES;
    c.row = a.qkv + (size_t)row * ((a.H + 2 * a.KV) * D) + (a.H + h) * D + 8 * c.chunk;
    c.at = slot & 15;
    c.group = (size_t)cell_group(slot >> a.shift, h, a.KV, a.shift, (slot & ((1 << a.shift) - 1)) >> 4, D);
    return c;
}

// Codes and parameters of a head of which this lane has eight features:
//     scale = type((max - min) / 15), a last place less if 15 scales above zero would round to infinity;  zero = min;
//     code = clamp(rint((x - zero) / scale), 0, 15), 0 where scale is
// with quotients rounded to fp32.  The division is done where a product with the reciprocal (off by less than 2^-18 below 16) is within 2^-13 of a half.
// A head with an infinity or a NaN in it, or a range beyond the type's, is NaN throughout.
template <int DT, int LANES>
__device__ __forceinline__ uint32_t quantise_head(const u32x4& x, uint32_t* param)
{
    typedef typename Elem<DT>::t T;
    float v[8], lo, hi, probe = 0.0f;
    to_floats<DT>(x, v);
    lo = hi = v[0];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        lo = fminf(lo, v[e]);
        hi = fmaxf(hi, v[e]);
        probe = __builtin_fmaf(v[e], 0.0f, probe);
    }
    struct OpMin { __device__ __forceinline__ float operator()(float a, float b) const { return fminf(a, b); } };
    lo = group_reduce<LANES>(lo, OpMin());
    hi = group_reduce<LANES>(hi, OpMax());
    probe = group_reduce<LANES>(probe, OpAdd());
    const T scale = (T)__fdiv_rn(__fsub_rn(hi, lo), 15.0f), zero = (T)__fadd_rn(lo, 0.0f);      // lo is a number of the type; -0 becomes 0
    uint16_t sb = __builtin_bit_cast(uint16_t, scale);
    const uint16_t zb = __builtin_bit_cast(uint16_t, zero);
    const float z = (float)zero;
    const bool odd = probe != probe || !__builtin_isfinite((float)scale);
    if (!odd && __builtin_isinf((float)(T)__builtin_fmaf(15.0f, (float)scale, z))) --sb;
    const float s = (float)__builtin_bit_cast(T, sb);
    const bool fast = s >= 0x1p-100f && s <= 0x1p100f;
    float rcp = __builtin_amdgcn_rcpf(s);
    rcp = __builtin_fmaf(__builtin_fmaf(-s, rcp, 1.0f), rcp, rcp);
    uint32_t word = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float num = __fsub_rn(v[e], z);
        float t = __fmul_rn(num, rcp), r = __builtin_rintf(t);
        if (!fast || __builtin_fabsf(__builtin_fabsf(t - r) - 0.5f) < 0x1p-13f) r = __builtin_rintf(__fdiv_rn(num, s));
        word |= (uint32_t)fminf(fmaxf(r, 0.0f), 15.0f) << (4 * (e / 2) + 16 * (e % 2));
    }
    constexpr uint32_t NOT_A_NUMBER = DT == LPQ_DT_FP16 ? 0x7e007e00u : 0x7fc07fc0u;
    *param = odd ? NOT_A_NUMBER : (uint32_t)sb | (uint32_t)zb << 16;
    return odd || sb == 0 ? 0u : word;
}

template <int DT, int D>
__global__ __launch_bounds__(256) void paged_append4_kernel(CellArgs a)
{
    const Cell c = cell_of<D>(a);
    if (!c.any) return;                                // all lanes of a head or none
    const u32x4 k = *reinterpret_cast<const u32x4*>(c.row), v = *reinterpret_cast<const u32x4*>(c.row + a.KV * D);
    uint32_t kparam, vparam;
    const uint32_t kw = quantise_head<DT, D / 8>(k, &kparam), vw = quantise_head<DT, D / 8>(v, &vparam);
    uint8_t *kg = a.kp + c.group, *vg = a.vp + c.group;
    *reinterpret_cast<uint32_t*>(kg + c.at * (D / 2) + 4 * c.chunk) = kw;
    *reinterpret_cast<uint32_t*>(vg + c.at * (D / 2) + 4 * c.chunk) = vw;
    if (c.chunk == 0) {
        *reinterpret_cast<uint32_t*>(kg + 8 * D + 4 * c.at) = kparam;
        *reinterpret_cast<uint32_t*>(vg + 8 * D + 4 * c.at) = vparam;
    }
}

template <int DT, int D>
__global__ __launch_bounds__(256) void paged_load4_kernel(CellArgs a)
{
    const Cell c = cell_of<D>(a);
    if (!c.any) return;
    const uint8_t *kg = a.kp + c.group, *vg = a.vp + c.group;
    const uint32_t kw = *reinterpret_cast<const uint32_t*>(kg + c.at * (D / 2) + 4 * c.chunk), vw = *reinterpret_cast<const uint32_t*>(vg + c.at * (D / 2) + 4 * c.chunk);
    const uint32_t kparam = *reinterpret_cast<const uint32_t*>(kg + 8 * D + 4 * c.at), vparam = *reinterpret_cast<const uint32_t*>(vg + 8 * D + 4 * c.at);
    *reinterpret_cast<u32x4*>(c.row) = cell_values<DT>(kw, kparam);
    *reinterpret_cast<u32x4*>(c.row + a.KV * D) = cell_values<DT>(vw, vparam);
}

template <int DT, int D>
hipError_t launch_rotary(RotaryArgs a, bool adjacent, hipStream_t s)
{
    constexpr int SLOTS = 64 / (D / 16), HEADS = 2;
    a.groups = (a.heads + SLOTS * HEADS - 1) / (SLOTS * HEADS);
    const unsigned grid = (unsigned)(((int64_t)a.M * a.groups + 3) / 4);
    if (adjacent) qk_norm_rotary_kernel<DT, D, true, HEADS><<<grid, 256, 0, s>>>(a);
    else          qk_norm_rotary_kernel<DT, D, false, HEADS><<<grid, 256, 0, s>>>(a);
    return hipGetLastError();
}

template <bool APPEND, int DT, int D>
hipError_t launch_cells_of(const CellArgs& a, hipStream_t s)
{
    const unsigned grid = (unsigned)(((int64_t)a.M * a.KV * (D / 8) + 255) / 256);
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

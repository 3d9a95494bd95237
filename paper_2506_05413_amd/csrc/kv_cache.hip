// New keys and values into a paged cache, turned by their positions on the way, and rows of the cache back as fp16.
//
//   halves:  y_i = x_i cos_i - x_{i+D/2} sin_i,   y_{i+D/2} = x_{i+D/2} cos_i + x_i sin_i       (pairs: 2i and 2i + 1)
//   Hadamard: y <- y H_D / sqrt(D) inside the head, butterflies over strides 1, 2, 4, ..
//   4 bits, per token and head:  D = (hi - lo) * (1 / 15), z = -rint(lo / D), code = clamp(rint(v / D) + z, 0, 15)
//
// Every product, sum and quotient is rounded on its own (no fused multiply-add): keys are rounded to fp16 and values next to
// a rounding boundary take the code that the formula in fp32 gives, whoever evaluates it.
//
// Pure streaming.  Eight values (16 bytes) per lane, D / 8 lanes per row, a row being one head of one token, query, key or
// value; the head's other half, the butterflies and the range of a row are exchanged between those lanes with operand
// permutations, without LDS.
#include "sr_common.h"

namespace sr {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
union Eight { u32x4 v; uint32_t w[4]; __half h[8]; };

// lane ^ MASK inside a row of 16 lanes
template <int MASK, typename T> __device__ __forceinline__ T lane_xor(T v)
{
    if constexpr (MASK == 1) return lane_perm<0xB1>(v);
    else if constexpr (MASK == 2) return lane_perm<0x4E>(v);
    else if constexpr (MASK == 4) return lane_perm<0x1B>(lane_perm<0x141>(v));    // 7 - i, then 3 - i inside the quad
    else return lane_perm<0x128>(v);                                              // rotation by 8 of 16
}

template <int MASK> __device__ __forceinline__ void butterfly(float (&v)[8], int lane)
{
    const uint32_t flip = lane & MASK ? 0x80000000u : 0u;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float other = lane_xor<MASK>(v[e]);
        v[e] = other + __uint_as_float(__float_as_uint(v[e]) ^ flip);
    }
}

// v <- v H / sqrt(D) over the 8 values of each of the D / 8 lanes
template <int D> __device__ __forceinline__ void hadamard_row(float (&v)[8], int lane)
{
#pragma clang fp contract(off)
#pragma unroll
    for (int h = 1; h < 8; h *= 2)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (!(e & h)) {
                const float a = v[e], b = v[e + h];
                v[e] = a + b;
                v[e + h] = a - b;
            }
    butterfly<1>(v, lane);
    butterfly<2>(v, lane);
    butterfly<4>(v, lane);
    if constexpr (D == 128) butterfly<8>(v, lane);
    constexpr float norm = D == 128 ? 0.08838834764831845f : 0.125f;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = v[e] * norm;
}

template <int D, bool PAIRS> __device__ __forceinline__ void rotate_row(float (&v)[8], const Eight &x, const float *row, int lane)
{
#pragma clang fp contract(off)
    if constexpr (PAIRS) {
        const f32x4 c = *reinterpret_cast<const f32x4 *>(row + 4 * lane), s = *reinterpret_cast<const f32x4 *>(row + D / 2 + 4 * lane);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float a = v[2 * e], b = v[2 * e + 1];
            v[2 * e] = a * c[e] - b * s[e];
            v[2 * e + 1] = b * c[e] + a * s[e];
        }
    } else {
        const int first = 8 * (lane & (D / 16 - 1));
        Eight p;
#pragma unroll
        for (int i = 0; i < 4; ++i) p.w[i] = (uint32_t)lane_xor<D / 16>((int)x.w[i]);
        const uint32_t flip = lane < D / 16 ? 0x80000000u : 0u;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const f32x4 c = *reinterpret_cast<const f32x4 *>(row + first + 4 * q), s = *reinterpret_cast<const f32x4 *>(row + D / 2 + first + 4 * q);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float sine = __uint_as_float(__float_as_uint(s[e]) ^ flip);
                v[4 * q + e] = v[4 * q + e] * c[e] + __half2float(p.h[4 * q + e]) * sine;
            }
        }
    }
}

// four-bit codes of a row spread over D / 8 lanes; scale and zero are the same in all of them
template <int D> __device__ __forceinline__ uint32_t quantise_row(const Eight &x, float clip, float &scale, float &zero)
{
#pragma clang fp contract(off)
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __half2float(x.h[e]);
    float mx = fmaxf(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), fmaxf(fmaxf(v[4], v[5]), fmaxf(v[6], v[7])));
    float mn = fminf(fminf(fminf(v[0], v[1]), fminf(v[2], v[3])), fminf(fminf(v[4], v[5]), fminf(v[6], v[7])));
    mx = fmaxf(mx, lane_perm<0xB1>(mx)), mn = fminf(mn, lane_perm<0xB1>(mn));
    mx = fmaxf(mx, lane_perm<0x4E>(mx)), mn = fminf(mn, lane_perm<0x4E>(mn));
    mx = fmaxf(mx, lane_perm<0x141>(mx)), mn = fminf(mn, lane_perm<0x141>(mn));
    if constexpr (D == 128) mx = fmaxf(mx, lane_perm<0x140>(mx)), mn = fminf(mn, lane_perm<0x140>(mn));
    const float hi = clip * mx, lo = clip * mn;
    scale = hi == lo ? 1.f : (hi - lo) * (1.f / 15.f);
    zero = -rintf(lo / scale);
    uint32_t word = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float c = fminf(fmaxf(rintf(v[e] / scale) + zero, 0.f), 15.f);
        word |= (uint32_t)c << (4 * e);
    }
    return word;
}

struct Append {
    const __half *q, *k, *v;
    int64_t ldq, ldk, ldv;
    uint32_t rows;                       // tokens * (heads + 2 * kv)
    int heads, kv;
    const int32_t *positions;
    const int64_t *slots;
    const float *table;
    int max_pos;
    float clip;
    void *K, *V;
    float *Kp, *Vp;
    int64_t n_slots;
    int page_shift;
    __half *qo, *ko;
    int64_t ldqo, ldko;
};

template <int D, bool I4, bool PAIRS, bool HAD> __global__ __launch_bounds__(256) void rope_kv_append_kernel(Append a)
{
    constexpr int LPR = D / 8;
    const int lane = threadIdx.x & (LPR - 1);
    const uint32_t row = blockIdx.x * (256u / LPR) + threadIdx.x / LPR;
    if (row >= a.rows) return;
    const uint32_t per = a.heads + 2 * a.kv, token = row / per;
    const int head = (int)(row - token * per);
    const bool is_q = head < a.heads, is_v = head >= a.heads + a.kv;
    const int h = is_q ? head : is_v ? head - a.heads - a.kv : head - a.heads;
    const __half *src = is_q ? a.q + token * a.ldq : is_v ? a.v + token * a.ldv : a.k + token * a.ldk;
    Eight x;
    x.v = *reinterpret_cast<const u32x4 *>(src + (int64_t)h * D + 8 * lane);
    const int64_t slot = is_q ? 0 : a.slots[token];
    if (!is_v && (a.table || HAD)) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __half2float(x.h[e]);
        if (a.table) {
            const int pos = min(max(a.positions[token], 0), a.max_pos - 1);
            rotate_row<D, PAIRS>(v, x, a.table + (int64_t)pos * D, lane);
        }
        if constexpr (HAD) hadamard_row<D>(v, lane);
#pragma unroll
        for (int e = 0; e < 8; ++e) x.h[e] = __float2half_rn(v[e]);
    }
    if (is_q) {
        *reinterpret_cast<u32x4 *>(a.qo + token * a.ldqo + (int64_t)h * D + 8 * lane) = x.v;
        return;
    }
    if (!is_v && a.ko) *reinterpret_cast<u32x4 *>(a.ko + token * a.ldko + (int64_t)h * D + 8 * lane) = x.v;
    if (slot < 0 || slot >= a.n_slots) return;
    // page-major, then head, then token of the page
    const int64_t at = (((slot >> a.page_shift) * a.kv + h) << a.page_shift) + (slot & ((1 << a.page_shift) - 1));
    void *cache = is_v ? a.V : a.K;
    if constexpr (I4) {
        float scale, zero;
        const uint32_t word = quantise_row<D>(x, a.clip, scale, zero);
        static_cast<uint32_t *>(cache)[at * LPR + lane] = word;
        if (lane == 0) reinterpret_cast<float2 *>(is_v ? a.Vp : a.Kp)[at] = make_float2(scale, zero);
    } else {
        static_cast<u32x4 *>(cache)[at * LPR + lane] = x.v;
    }
}

struct Gather {
    const int64_t *slots;
    uint32_t rows;                       // tokens * 2 * kv
    int kv;
    const void *K, *V;
    const float *Kp, *Vp;
    int64_t n_slots;
    int page_shift;
    __half *ko, *vo;
    int64_t ldko, ldvo;
};

template <int D, bool I4> __global__ __launch_bounds__(256) void kv_gather_kernel(Gather a)
{
#pragma clang fp contract(off)
    constexpr int LPR = D / 8;
    const int lane = threadIdx.x & (LPR - 1);
    const uint32_t row = blockIdx.x * (256u / LPR) + threadIdx.x / LPR;
    if (row >= a.rows) return;
    const uint32_t token = row / (2 * a.kv);
    const int side = (int)(row - token * (2 * a.kv)), h = side % a.kv;
    const bool is_v = side >= a.kv;
    const int64_t slot = a.slots[token];
    Eight x;
    x.v = 0u;
    if (slot >= 0 && slot < a.n_slots) {
        const int64_t at = (((slot >> a.page_shift) * a.kv + h) << a.page_shift) + (slot & ((1 << a.page_shift) - 1));
        const void *cache = is_v ? a.V : a.K;
        if constexpr (I4) {
            const uint32_t word = static_cast<const uint32_t *>(cache)[at * LPR + lane];
            const float2 p = reinterpret_cast<const float2 *>(is_v ? a.Vp : a.Kp)[at];
#pragma unroll
            for (int e = 0; e < 8; ++e) x.h[e] = __float2half_rn(((float)((word >> (4 * e)) & 15u) - p.y) * p.x);
        } else {
            x.v = static_cast<const u32x4 *>(cache)[at * LPR + lane];
        }
    }
    __half *dst = is_v ? a.vo + token * a.ldvo : a.ko + token * a.ldko;
    *reinterpret_cast<u32x4 *>(dst + (int64_t)h * D + 8 * lane) = x.v;
}

inline int shift_of(int64_t page) { return __builtin_ctzll((unsigned long long)page); }

template <int D, bool I4> hipError_t append_dim(const Append &a, bool pairs, bool had, hipStream_t st)
{
    const dim3 grid((unsigned)(((uint64_t)a.rows * (D / 8) + 255) / 256)), block(256);
    if (pairs && had) hipLaunchKernelGGL((rope_kv_append_kernel<D, I4, true, true>), grid, block, 0, st, a);
    else if (pairs) hipLaunchKernelGGL((rope_kv_append_kernel<D, I4, true, false>), grid, block, 0, st, a);
    else if (had) hipLaunchKernelGGL((rope_kv_append_kernel<D, I4, false, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((rope_kv_append_kernel<D, I4, false, false>), grid, block, 0, st, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rope_kv_append(const void *Q, int64_t ldq, const void *K, int64_t ldk, const void *V, int64_t ldv, int64_t T,
                                 int64_t n_heads, const int32_t *positions, const int64_t *slots, const float *cos_sin,
                                 int64_t max_pos, bool pairs, bool had, float clip, const KvCache &c, void *Q_out, int64_t ldqo,
                                 void *K_out, int64_t ldko, hipStream_t st)
{
    Append a;
    a.q = static_cast<const __half *>(Q), a.k = static_cast<const __half *>(K), a.v = static_cast<const __half *>(V);
    a.ldq = ldq, a.ldk = ldk, a.ldv = ldv;
    a.rows = (uint32_t)(T * (n_heads + 2 * c.heads));
    a.heads = (int)n_heads, a.kv = (int)c.heads;
    a.positions = positions, a.slots = slots, a.table = cos_sin;
    a.max_pos = (int)max_pos, a.clip = clip;
    a.K = c.K, a.V = c.V, a.Kp = c.Kp, a.Vp = c.Vp;
    a.n_slots = c.pages * c.page_size, a.page_shift = shift_of(c.page_size);
    a.qo = static_cast<__half *>(Q_out), a.ko = static_cast<__half *>(K_out);
    a.ldqo = ldqo, a.ldko = ldko;
    if (c.dim == 128) return c.i4 ? append_dim<128, true>(a, pairs, had, st) : append_dim<128, false>(a, pairs, had, st);
    return c.i4 ? append_dim<64, true>(a, pairs, had, st) : append_dim<64, false>(a, pairs, had, st);
}

hipError_t launch_kv_gather(const int64_t *slots, int64_t T, const KvCache &c, void *K_out, int64_t ldko, void *V_out, int64_t ldvo,
                            hipStream_t st)
{
    Gather a;
    a.slots = slots, a.rows = (uint32_t)(T * 2 * c.heads), a.kv = (int)c.heads;
    a.K = c.K, a.V = c.V, a.Kp = c.Kp, a.Vp = c.Vp;
    a.n_slots = c.pages * c.page_size, a.page_shift = shift_of(c.page_size);
    a.ko = static_cast<__half *>(K_out), a.vo = static_cast<__half *>(V_out);
    a.ldko = ldko, a.ldvo = ldvo;
    const dim3 grid((unsigned)(((uint64_t)a.rows * (c.dim / 8) + 255) / 256)), block(256);
    if (c.dim == 128 && c.i4) hipLaunchKernelGGL((kv_gather_kernel<128, true>), grid, block, 0, st, a);
    else if (c.dim == 128) hipLaunchKernelGGL((kv_gather_kernel<128, false>), grid, block, 0, st, a);
    else if (c.i4) hipLaunchKernelGGL((kv_gather_kernel<64, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((kv_gather_kernel<64, false>), grid, block, 0, st, a);
    return hipGetLastError();
}

}  // namespace sr

// New keys and values into a paged cache, turned by their positions on the way, and rows of the cache back as fp16.
//
//   halves:  y_i = x_i cos_i - x_{i+D/2} sin_i,   y_{i+D/2} = x_{i+D/2} cos_i + x_i sin_i       (pairs: 2i and 2i + 1)
//   Hadamard: y <- y H_D / sqrt(D) inside the head, butterflies over strides 1, 2, 4, ..
//   4 bits, per token and head:  D = (hi - lo) * (1 / 15), z = -rint(lo / D), code = clamp(rint(v / D) + z, 0, 15)
//
// Every product, sum and quotient comes out as rounded on its own: keys are rounded to fp16 and values next to a rounding
// boundary take the code that the formula in fp32 gives, whoever evaluates it.
//
// Bound by its bytes where there are many tokens (16384 with 32 query heads and 8 key/value heads of 128, 4 bits: 363 MB in 80 us,
// 4.5 TB/s; 2047 with the transform 14 us, 3.3 TB/s), else by the launch (one token 2.5 us).  Eight values (16 bytes) per lane,
// D / 8 lanes per row, a row being one head of one token, query, key or value; the head's other half, the butterflies and the
// range of a row are exchanged between those lanes with operand permutations, without LDS.
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

// Lanes with bit MASK clear get own + other, the others own - other, the negative of what the transform says: one fused
// multiply-add of the partner's value by 1 or -1, which rounds like the sum.  Partners of later steps carry the same signs, so
// that all of them come to one sign per lane at the end.  (Spelled out: from the exchange and the multiply-add the compiler makes
// a move and an operation per value.  A lane exchange of a register needs two cycles after it was written.)
template <int MASK> __device__ __forceinline__ void butterfly(float (&v)[8], int lane)
{
    const float sign = lane & MASK ? -1.f : 1.f;
#define SR_STEP(CTRL)                                                                                                              \
    asm("s_nop 1\n\t"                                                                                                              \
        "v_fmac_f32_dpp %0, %0, %8 " CTRL " row_mask:0xf bank_mask:0xf\n\tv_fmac_f32_dpp %1, %1, %8 " CTRL " row_mask:0xf bank_mask:0xf\n\t" \
        "v_fmac_f32_dpp %2, %2, %8 " CTRL " row_mask:0xf bank_mask:0xf\n\tv_fmac_f32_dpp %3, %3, %8 " CTRL " row_mask:0xf bank_mask:0xf\n\t" \
        "v_fmac_f32_dpp %4, %4, %8 " CTRL " row_mask:0xf bank_mask:0xf\n\tv_fmac_f32_dpp %5, %5, %8 " CTRL " row_mask:0xf bank_mask:0xf\n\t" \
        "v_fmac_f32_dpp %6, %6, %8 " CTRL " row_mask:0xf bank_mask:0xf\n\tv_fmac_f32_dpp %7, %7, %8 " CTRL " row_mask:0xf bank_mask:0xf"     \
        : "+v"(v[0]), "+v"(v[1]), "+v"(v[2]), "+v"(v[3]), "+v"(v[4]), "+v"(v[5]), "+v"(v[6]), "+v"(v[7])                             \
        : "v"(sign))
    if constexpr (MASK == 1) SR_STEP("quad_perm:[1,0,3,2]");
    else if constexpr (MASK == 2) SR_STEP("quad_perm:[2,3,0,1]");
    else if constexpr (MASK == 8) SR_STEP("row_ror:8");
    else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = fmaf(lane_xor<4>(v[e]), sign, v[e]);
    }
#undef SR_STEP
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
    const float norm = (__popc(lane) & 1 ? -1.f : 1.f) * (D == 128 ? 0.08838834764831845f : 0.125f);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = v[e] * norm;
}

// a lane's share of a position's angles: those of its eight values (PAIRS: four pairs)
template <bool PAIRS> struct Angles {
    static constexpr int N = PAIRS ? 1 : 2;
    f32x4 c[N], s[N];
};
template <int D, bool PAIRS> __device__ __forceinline__ Angles<PAIRS> angles_at(const float *row, int lane)
{
    Angles<PAIRS> a;
    const int first = PAIRS ? 4 * lane : 8 * (lane & (D / 16 - 1));
#pragma unroll
    for (int i = 0; i < a.N; ++i) {
        a.c[i] = *reinterpret_cast<const f32x4 *>(row + first + 4 * i);
        a.s[i] = *reinterpret_cast<const f32x4 *>(row + D / 2 + first + 4 * i);
    }
    return a;
}
template <int D, bool PAIRS> __device__ __forceinline__ void rotate_row(float (&v)[8], const Eight &x, const Angles<PAIRS> &a, int lane)
{
#pragma clang fp contract(off)
    if constexpr (PAIRS) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float p = v[2 * e], q = v[2 * e + 1];
            v[2 * e] = p * a.c[0][e] - q * a.s[0][e];
            v[2 * e + 1] = q * a.c[0][e] + p * a.s[0][e];
        }
    } else {
        Eight p;
#pragma unroll
        for (int i = 0; i < 4; ++i) p.w[i] = (uint32_t)lane_xor<D / 16>((int)x.w[i]) ^ (lane < D / 16 ? 0x80008000u : 0u);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = v[e] * a.c[e / 4][e % 4] + __half2float(p.h[e]) * a.s[e / 4][e % 4];
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
    // Quotients from the correctly rounded reciprocal y: q = a y, and one step q + (a - q d) y with the exact remainder gives
    // the correctly rounded a / d (Markstein, 1990); a and d are far from the ends of fp32's range.
    const float y = 1.f / scale;
    auto over_scale = [&](float a) {
        const float q = a * y;
        return fmaf(fmaf(-q, scale, a), y, q);
    };
    zero = -rintf(over_scale(lo));
    // Adding 1.5 * 2^23 rounds a quotient (below 2^16 in size) to the nearest integer, ties to even, in the low bits.
    constexpr uint32_t kMagic = 0x4B400000u;
    const int shift = (int)zero - (int)kMagic;
    uint32_t word = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int c = (int)__float_as_uint(over_scale(v[e]) + __uint_as_float(kMagic)) + shift;
        word |= (uint32_t)min(max(c, 0), 15) << (4 * e);
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

// (One row per group of lanes: two or four, on their way together, were 2 - 8 % slower up to 4096 tokens and 4 % faster at 16384.)
template <int D, bool I4, bool PAIRS, bool HAD> __global__ __launch_bounds__(256) void rope_kv_append_kernel(Append a)
{
    constexpr int LPR = D / 8, GROUPS = 256 / LPR;
    const int lane = threadIdx.x & (LPR - 1);
    const uint32_t per = a.heads + 2 * a.kv, first = blockIdx.x * (uint32_t)GROUPS, row = first + threadIdx.x / LPR;
    if (row >= a.rows) return;
    const uint32_t token0 = first / per, rest = row - token0 * per;
    // (the quotient, 32 at most, is half a row away from the next whole number)
    const uint32_t on = (uint32_t)(((float)rest + 0.5f) * __builtin_amdgcn_rcpf((float)per)), token = token0 + on;
    const int head = (int)(rest - on * per);
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
            rotate_row<D, PAIRS>(v, x, angles_at<D, PAIRS>(a.table + (int64_t)pos * D, lane), lane);
        }
        if constexpr (HAD) hadamard_row<D>(v, lane);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            asm("" : "+v"(v[e]));                        // a number of fp32: the last product is not to be rounded to fp16 at once
            x.h[e] = __float2half_rn(v[e]);
        }
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

// N rows per group of lanes, a workgroup's apart: their slots, then their rows, then their values
template <int D, bool I4, int N> __global__ __launch_bounds__(256) void kv_gather_kernel(Gather a)
{
#pragma clang fp contract(off)
    constexpr int LPR = D / 8, GROUPS = 256 / LPR;
    const int lane = threadIdx.x & (LPR - 1);
    const uint32_t per = 2 * a.kv, first = blockIdx.x * (uint32_t)(GROUPS * N), token0 = first / per, rest0 = first - token0 * per;
    const float per_row = __builtin_amdgcn_rcpf((float)per);
    uint32_t token[N];
    int side[N];                                         // head, or kv + head; of rows behind the last: the last one's
    int64_t at[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const uint32_t rest = min(rest0 + GROUPS * k + threadIdx.x / LPR, a.rows - 1 - token0 * per);
        const uint32_t on = (uint32_t)(((float)rest + 0.5f) * per_row);      // 64 at most, half a row away from a whole number
        token[k] = token0 + on, side[k] = (int)(rest - on * per);
        const int64_t slot = a.slots[token[k]];
        const int h = side[k] < a.kv ? side[k] : side[k] - a.kv;
        at[k] = slot >= 0 && slot < a.n_slots ? (((slot >> a.page_shift) * a.kv + h) << a.page_shift) + (slot & ((1 << a.page_shift) - 1)) : -1;
    }
    uint32_t word[N];
    float2 params[N];
    Eight x[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        x[k].v = 0u, word[k] = 0, params[k] = make_float2(0.f, 0.f);
        if (at[k] < 0) continue;
        const void *cache = side[k] < a.kv ? a.K : a.V;
        if constexpr (I4) {
            word[k] = static_cast<const uint32_t *>(cache)[at[k] * LPR + lane];
            params[k] = reinterpret_cast<const float2 *>(side[k] < a.kv ? a.Kp : a.Vp)[at[k]];
        } else {
            x[k].v = static_cast<const u32x4 *>(cache)[at[k] * LPR + lane];
        }
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
        if constexpr (I4) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float v = ((float)((word[k] >> (4 * e)) & 15u) - params[k].y) * params[k].x;
                asm("" : "+v"(v));
                x[k].h[e] = __float2half_rn(v);
            }
        }
        __half *dst = side[k] < a.kv ? a.ko + token[k] * a.ldko + (int64_t)side[k] * D : a.vo + token[k] * a.ldvo + (int64_t)(side[k] - a.kv) * D;
        *reinterpret_cast<u32x4 *>(dst + 8 * lane) = x[k].v;
    }
}

// Two rows per group of lanes from eight workgroups on every compute unit on (16384 tokens of 8 heads of 128, 4 bits: 21.9 ->
// 19.8 us, 86 MB; four 19.3, but 4096 tokens 6.3 -> 6.7); nothing gained or lost below.
template <int D, bool I4> hipError_t gather_dim(const Gather &a, hipStream_t st)
{
    constexpr unsigned rows = 256 / (D / 8);
    if (a.rows >= 8 * rows * (unsigned)compute_units()) hipLaunchKernelGGL((kv_gather_kernel<D, I4, 2>), dim3((a.rows + 2 * rows - 1) / (2 * rows)), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((kv_gather_kernel<D, I4, 1>), dim3((a.rows + rows - 1) / rows), dim3(256), 0, st, a);
    return hipGetLastError();
}

inline int shift_of(int64_t page) { return __builtin_ctzll((unsigned long long)page); }

template <int D, bool I4> hipError_t append_dim(const Append &a, bool pairs, bool had, hipStream_t st)
{
    constexpr unsigned rows = 256 / (D / 8);
    const dim3 grid((a.rows + rows - 1) / rows), block(256);
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
    if (c.dim == 128) return c.i4 ? gather_dim<128, true>(a, st) : gather_dim<128, false>(a, st);
    return c.i4 ? gather_dim<64, true>(a, st) : gather_dim<64, false>(a, st);
}

}  // namespace sr

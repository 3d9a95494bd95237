// New keys and values into a paged cache, turned by their positions on the way, and rows of the cache back as fp16.
//
//   halves:  y_i = x_i cos_i - x_{i+D/2} sin_i,   y_{i+D/2} = x_{i+D/2} cos_i + x_i sin_i       (pairs: 2i and 2i + 1)
//   Hadamard: y <- y H_D / sqrt(D) inside the head, butterflies over strides 1, 2, 4, ..
//   4 bits, per token and head:  D = (hi - lo) * (1 / 15), z = -rint(lo / D), code = clamp(rint(v / D) + z, 0, 15)
//
// Every product, sum and quotient comes out as rounded on its own: keys are rounded to fp16 and values next to a rounding
// boundary take the code that the formula in fp32 gives, whoever evaluates it.
//
// Bound by its bytes where there are many tokens (16384 with 32 query heads and 8 key/value heads of 128, 4 bits: 387 MB in 76 us,
// 5.1 TB/s; 2047 with the transform 13.2 us, 3.7 TB/s), else by the launch (one token 2.7 us).  Eight values (16 bytes) per lane,
// D / 8 lanes per row, a row being one head of one token, query, key or value; the head's other half, the butterflies and the
// range of a row are exchanged between those lanes with operand permutations, without LDS.
#include "sr_common.h"

namespace sr {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
union Eight { u32x4 v; uint32_t w[4]; __half h[8]; f16x2 p[4]; };

// Lane l of a row holds the eight values number l ^ 3 if bit 2 of l is set, else l: number ^ 4 then is in lane l ^ 7, which is one
// exchange (l ^ 4 would be two).  Everything below goes by that number, called lane.
__device__ __forceinline__ int number_of(int l) { return l ^ (l & 4 ? 3 : 0); }
// number ^ MASK inside a row of 16 lanes, MASK half of a row of D / 8
template <int MASK> __device__ __forceinline__ int lane_xor(int v)
{
    static_assert(MASK == 4 || MASK == 8);
    return lane_perm<MASK == 4 ? 0x141 : 0x128>(v);                               // lane 7 - l of eight; rotation by 8 of 16
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
    else if constexpr (MASK == 4) SR_STEP("row_half_mirror");
    else SR_STEP("row_ror:8");
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

// NaN if one of eight numbers is infinite or none, else zero
__device__ __forceinline__ float not_finite(const Eight &x)
{
    const f16x2 none = {(_Float16)0.f, (_Float16)0.f};
    f16x2 t = x.p[0] * none;
#pragma unroll
    for (int i = 1; i < 4; ++i) t = __builtin_elementwise_fma(x.p[i], none, t);
    return (float)(t[0] + t[1]);
}

// Four-bit codes of a row spread over D / 8 lanes; scale and zero are the same in all of them.  A row with a value that is not finite
// (a key may become so by the transform) has no codes: it gets those of zeros, and NaN for its scale.
template <int D> __device__ __forceinline__ uint32_t quantise_row(Eight x, float clip, float &scale, float &zero)
{
#pragma clang fp contract(off)
    float bad = not_finite(x);
    if (__any(bad != bad)) {                                                     // (seldom: the maximum below takes no notice of NaN)
        bad += lane_perm<0xB1>(bad);
        bad += lane_perm<0x4E>(bad);
        bad += lane_perm<0x141>(bad);
        if constexpr (D == 128) bad += lane_perm<0x140>(bad);
        if (bad != bad) x.v = 0u;
    }
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
    // the correctly rounded a / d (Markstein, 1990); a and d are far from the ends of fp32's range (d is 2^-92 at least).
    const float y = 1.f / scale;
    auto over_scale = [&](float a) {
        const float q = a * y;
        return fmaf(fmaf(-q, scale, a), y, q);
    };
    zero = -rintf(over_scale(lo));
    // clamp(rint(q) + z, 0, 15) = rint(clamp(q, -z, 15 - z)) + z: |z| is below 2^16 whatever the clipping ratio (a row's range is at
    // least one fp16 spacing of its largest value), while q grows with the ratio's inverse.  Adding 1.5 * 2^23 rounds the clamped
    // quotient to the nearest integer, ties to even, in the low bits.
    constexpr uint32_t kMagic = 0x4B400000u;
    const int shift = (int)zero - (int)kMagic;
    uint32_t word = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float q = __builtin_amdgcn_fmed3f(over_scale(v[e]), -zero, 15.f - zero);
        word |= (uint32_t)((int)__float_as_uint(q + __uint_as_float(kMagic)) + shift) << (4 * e);
    }
    scale += bad;
    return word;
}

struct Append {
    const __half *q, *k, *v;
    int64_t ldq, ldk, ldv;
    uint32_t tokens;
    int heads, kv;
    uint32_t q_waves, kv_waves;          // waves over the queries; over the keys, and over the values
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

// APART: a wave's rows are all queries, all keys or all values, so that what differs between those is scalar; else rows lie in the
// order of the tokens.  Measured (us, apart / in order; 32 + 2 x 8 heads of 128): with the transform 1024 tokens 8.5 / 9.2, 2047
// 13.3 / 13.4, 4096 24.3 / 24.6, 16384 95.6 / 93.7; without it 2047 10.7 / 11.1, 4096 19.9 / 20.4, 8192 42.0 / 40.7 (fp16 43.2 / 41.0),
// 16384 80.1 / 76.1 (fp16 83.2 / 75.8).
// (One row per group of lanes: two or four, on their way together, were 2 - 8 % slower up to 4096 tokens and 4 % faster at 16384, before
// waves were told apart.)
template <int D, bool I4, bool PAIRS, bool HAD, bool APART> __global__ __launch_bounds__(256) void rope_kv_append_kernel(Append a)
{
    constexpr int LPR = D / 8, ROWS = 64 / LPR;          // rows of a wave
    const int lane = number_of(threadIdx.x & (LPR - 1));
    bool is_q, is_v;
    uint32_t heads, first;                               // of the rows that this one is among: heads of a token, the wave's first row
    if constexpr (APART) {
        uint32_t wave = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        is_q = wave < a.q_waves, is_v = wave >= a.q_waves + a.kv_waves;
        wave -= is_q ? 0 : is_v ? a.q_waves + a.kv_waves : a.q_waves;
        if (wave >= a.kv_waves && is_v) return;
        heads = is_q ? a.heads : a.kv, first = wave * ROWS;
    } else {
        heads = a.heads + 2 * a.kv, first = blockIdx.x * (4 * ROWS);
    }
    const uint32_t token0 = first / heads, rest = first - token0 * heads + (APART ? threadIdx.x & 63 : threadIdx.x) / LPR;
    // (the quotient, 32 at most, is half a row away from the next whole number)
    const uint32_t on = (uint32_t)(((float)rest + 0.5f) * __builtin_amdgcn_rcpf((float)heads)), token = token0 + on;
    if (token >= a.tokens) return;
    int h = (int)(rest - on * heads);
    if constexpr (!APART) {
        is_q = h < a.heads, is_v = h >= a.heads + a.kv;
        h -= is_q ? 0 : is_v ? a.heads + a.kv : a.heads;
    }
    // (in order, the rows' addresses from the start)
    const uint32_t base = APART ? token0 : token, off = APART ? on : 0, column = h * D + 8 * lane;
    const __half *src = is_q ? a.q + base * a.ldq : is_v ? a.v + base * a.ldv : a.k + base * a.ldk;
    const int64_t ld = is_q ? a.ldq : is_v ? a.ldv : a.ldk;
    Eight x;
    x.v = *reinterpret_cast<const u32x4 *>(src + (off * ld + column));
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
        for (int e = 0; e < 8; e += 2) {
            asm("" : "+v"(v[e]), "+v"(v[e + 1]));        // numbers of fp32: the last product is not to be rounded to fp16 at once
            x.p[e / 2] = f16x2{(_Float16)v[e], (_Float16)v[e + 1]};
        }
    }
    if (is_q) {
        *reinterpret_cast<u32x4 *>(a.qo + base * a.ldqo + (off * a.ldqo + column)) = x.v;
        return;
    }
    if (!is_v && a.ko) *reinterpret_cast<u32x4 *>(a.ko + base * a.ldko + (off * a.ldko + column)) = x.v;
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

// Two rows per group of lanes from eight workgroups on every compute unit on (16384 tokens of 8 heads of 128, 4 bits, 86 MB: 20.4 ->
// 18.5 us, 4096 7.0 -> 6.3; fp16, 134 MB, 28.0 -> 26.7); little gained or lost below (2047 tokens 4.17 -> 4.10).
template <int D, bool I4> hipError_t gather_dim(const Gather &a, hipStream_t st)
{
    constexpr unsigned rows = 256 / (D / 8);
    if (a.rows >= 8 * rows * (unsigned)compute_units()) hipLaunchKernelGGL((kv_gather_kernel<D, I4, 2>), dim3((a.rows + 2 * rows - 1) / (2 * rows)), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((kv_gather_kernel<D, I4, 1>), dim3((a.rows + rows - 1) / rows), dim3(256), 0, st, a);
    return hipGetLastError();
}

inline int shift_of(int64_t page) { return __builtin_ctzll((unsigned long long)page); }

template <int D, bool I4, bool APART> hipError_t append_rows(Append a, bool pairs, bool had, hipStream_t st)
{
    constexpr unsigned rows = 64 / (D / 8);              // of a wave
    a.q_waves = (a.tokens * (unsigned)a.heads + rows - 1) / rows;
    a.kv_waves = (a.tokens * (unsigned)a.kv + rows - 1) / rows;
    const unsigned waves = APART ? a.q_waves + 2 * a.kv_waves : (a.tokens * (unsigned)(a.heads + 2 * a.kv) + rows - 1) / rows;
    const dim3 grid((waves + 3) / 4), block(256);
    if constexpr (!APART) {
        if (pairs) hipLaunchKernelGGL((rope_kv_append_kernel<D, I4, true, false, APART>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((rope_kv_append_kernel<D, I4, false, false, APART>), grid, block, 0, st, a);
    } else if (pairs && had) hipLaunchKernelGGL((rope_kv_append_kernel<D, I4, true, true, APART>), grid, block, 0, st, a);
    else if (pairs) hipLaunchKernelGGL((rope_kv_append_kernel<D, I4, true, false, APART>), grid, block, 0, st, a);
    else if (had) hipLaunchKernelGGL((rope_kv_append_kernel<D, I4, false, true, APART>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((rope_kv_append_kernel<D, I4, false, false, APART>), grid, block, 0, st, a);
    return hipGetLastError();
}
template <int D, bool I4> hipError_t append_dim(const Append &a, bool pairs, bool had, hipStream_t st)
{
    const bool apart = had || (int64_t)a.tokens * (a.heads + 2 * a.kv) <= 1024 * (int64_t)compute_units();
    return apart ? append_rows<D, I4, true>(a, pairs, had, st) : append_rows<D, I4, false>(a, pairs, had, st);
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
    a.tokens = (uint32_t)T;
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

// Attention of one new token per sequence over a paged cache, split over the cache's length and joined.
//
//   s_t = scale q . k_t,   o = sum_t softmax(s)_t v_t     over the tokens t < length whose page exists
//
// Bound by the bytes of the cache.  A workgroup takes one sequence, one key/value head (up to 16 of the query heads that share
// it) and one run of tokens; its four waves walk over tiles of 32 tokens with a running maximum and sum, and meet in LDS.
// Both products run on 16 x 16 x 32 matrix instructions with the query head in the columns:
//
//   S^T = K Q^T   rows = tokens: lane (n, g) = (lane % 16, lane / 16) holds token n of the operand and gets tokens 4 g + r
//   O^T = V^T P^T its k-index is the token: lane (n, g) supplies the eight tokens 4 g + r of two halves of the tile, which are
//                 the ones it got scores for, so the weights go from one product to the next inside the lane
//
// The order of channels in the first product and of columns in the second is free, so both operands are taken as they lie in
// memory, and the sums over codes need no conversion: a code c in bits 4-7 of a half is the subnormal fp16 number c 2^-20, a
// shift and an AND per two codes.  (The matrix pipe takes subnormal operands; measured on random weights, sums over c 2^-20 are
// as exact as over c itself, to 2^-22, while over c 2^-24, bits 0-3, they are off by 2^-14 of a code.)  With scale d and zero z
// per token,
//   s_t = d (q . c - z sum(q)),   o = sum_t w_t (c_t - z_t),   w_t = p_t d_t
// where d goes into the exponent, w = exp2(s log2(e) + log2(d) - maximum): weights then are at most 1 however large or small
// the values are, and lose nothing to the range of fp16.  w is rounded to fp16 for the matrix pipe (half a step, 2^-12, per
// token; the same rounded w multiplies z), sums and maxima are fp32.
#include "sr_common.h"

namespace sr {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
union Frag { f16x8 v; uint32_t w[4]; _Float16 h[8]; };

constexpr int kWaves = 4, kTile = 32;
constexpr float kNone = -__builtin_inff();

struct Decode {
    const _Float16 *q;
    int64_t ldq;
    int heads, kv, group;                // query heads, key/value heads, query heads of one key/value head
    int row_tiles;                       // ceil(group / 16)
    const void *K, *V;
    const float *Kp, *Vp;
    uint32_t n_pages;
    int page_shift;
    const int32_t *table;
    int64_t ld_table;
    int64_t max_len;                     // tokens that the page table covers
    const int32_t *lens;
    float scale;                         // times log2(e)
    int splits, chunk;                   // runs of chunk tokens, a multiple of kWaves * kTile
    _Float16 *o;
    int64_t ldo;
    float *part;                         // [sequence][head][split][D] sums, then [sequence][head][split][2] maximum, total
    float *part_ml;
};

// reduction over the four lanes that share lane % 16
__device__ __forceinline__ float max_of_groups(float v)
{
    v = fmaxf(v, __shfl_xor(v, 16, 64));
    return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ __forceinline__ float sum_of_groups(float v)
{
    v += __shfl_xor(v, 16, 64);
    return v + __shfl_xor(v, 32, 64);
}

__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// nibbles i and i + 4 of a dword as the fp16 numbers code * 2^-20
__device__ __forceinline__ uint32_t nibble_pair(uint32_t w, int i)
{
    return (i == 0 ? w << 4 : w >> (4 * i - 4)) & 0x00F000F0u;
}

// what a wave loads of 32 tokens, as it lies in memory
template <int D, bool I4> struct Tile {
    static constexpr int KW = I4 ? D / 32 : D / 8;       // dwords of a lane's share of a key
    static constexpr int VW = I4 ? 1 : D / 32;           // dwords of a lane's share of a value
    uint32_t k[2][KW], v[2][4][VW];
    f32x4 kp[2][2], vp[2][2];                            // (scale, zero) of tokens 4 g + r
};

template <int D, bool I4> __global__ __launch_bounds__(256) void attn_decode_kernel(Decode a)
{
    constexpr int C = D / 16;                            // output columns per lane and row index: d = C n + j
    using T = Tile<D, I4>;
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t pairs = a.kv * a.row_tiles;
    const uint32_t split = blockIdx.x % (uint32_t)a.splits, rest = blockIdx.x / (uint32_t)a.splits;
    const uint32_t b = rest / pairs, pair = rest - b * pairs;
    const uint32_t h = pair / a.row_tiles, row0 = 16 * (pair - h * a.row_tiles);
    const int64_t len64 = min((int64_t)max(a.lens[b], 0), a.max_len);
    const int len = (int)len64;
    const int first = (int)split * a.chunk, last = min(first + a.chunk, len);
    if (first >= len && a.splits > 1) return;            // the join goes by the length too
    const int rows = min(16, a.group - (int)row0);
    const int head0 = (int)(h * a.group + row0);

    // query row n of the tile in the order that the keys lie in
    Frag q[D / 32];
    float qsum = 0.f;
    {
        const _Float16 *src = a.q + (int64_t)b * a.ldq + (int64_t)(head0 + n) * D;
        const bool there = n < rows;
        if constexpr (I4) {
            constexpr int per = D / 4;                   // codes of a key in one lane, a fragment per dword
            _Float16 x[per];
#pragma unroll
            for (int i = 0; i < per; i += 8) {
                Frag f;
                f.v = there ? *reinterpret_cast<const f16x8 *>(src + per * g + i) : (f16x8)(_Float16)0;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[i + e] = f.h[e];
                    qsum += (float)f.h[e];
                }
            }
#pragma unroll
            for (int p = 0; p < per / 8; ++p)
#pragma unroll
                for (int e = 0; e < 8; ++e) q[p].h[e] = x[8 * p + e / 2 + 4 * (e & 1)];      // halves of nibble_pair()
            qsum = sum_of_groups(qsum);
        } else {
#pragma unroll
            for (int i = 0; i < D / 32; ++i) q[i].v = there ? *reinterpret_cast<const f16x8 *>(src + 32 * i + 8 * g) : (f16x8)(_Float16)0;
        }
    }
    const float score_unit = I4 ? a.scale * 1048576.f : a.scale, qz = qsum * a.scale;

    f32x4 acc[C];
#pragma unroll
    for (int j = 0; j < C; ++j) acc[j] = 0.f;
    float top = kNone, total = 0.f, zsum = 0.f;          // total, zsum: over this lane's tokens

    const int32_t *table = a.table + (int64_t)b * a.ld_table;
    const int page_mask = (1 << a.page_shift) - 1;

    for (int t0 = first + wave * kTile; t0 < last; t0 += kWaves * kTile) {
        T t;
        bool page_there[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            // 16 tokens lie in one page; tokens past the end read the last page there is and count for nothing
            const int tu = min(t0 + 16 * u, (last - 1) & ~15);
            const uint32_t id = (uint32_t)__builtin_amdgcn_readfirstlane(table[tu >> a.page_shift]);
            page_there[u] = id < a.n_pages;
            const int64_t row = ((((int64_t)(page_there[u] ? id : 0u) * a.kv + h) << a.page_shift) + (tu & page_mask));
            if constexpr (I4) {
                const uint32_t *kr = static_cast<const uint32_t *>(a.K) + (row + n) * (D / 8) + g * (D / 32);
#pragma unroll
                for (int i = 0; i < D / 32; ++i) t.k[u][i] = kr[i];
                const uint32_t *vr = static_cast<const uint32_t *>(a.V) + (row + 4 * g) * (D / 8) + (D == 128 ? n : n >> 1);
#pragma unroll
                for (int r = 0; r < 4; ++r) t.v[u][r][0] = vr[r * (D / 8)];
                const f32x4 *kp = reinterpret_cast<const f32x4 *>(a.Kp + (row + 4 * g) * 2), *vp = reinterpret_cast<const f32x4 *>(a.Vp + (row + 4 * g) * 2);
                t.kp[u][0] = kp[0], t.kp[u][1] = kp[1];
                t.vp[u][0] = vp[0], t.vp[u][1] = vp[1];
            } else {
                const u32x4 *kr = reinterpret_cast<const u32x4 *>(static_cast<const _Float16 *>(a.K) + (row + n) * D);
#pragma unroll
                for (int i = 0; i < D / 32; ++i) {
                    const u32x4 x = kr[4 * i + g];
#pragma unroll
                    for (int e = 0; e < 4; ++e) t.k[u][4 * i + e] = x[e];
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const uint32_t *vr = reinterpret_cast<const uint32_t *>(static_cast<const _Float16 *>(a.V) + (row + 4 * g + r) * D) + n * (D / 32);
#pragma unroll
                    for (int e = 0; e < D / 32; ++e) t.v[u][r][e] = vr[e];
                }
            }
        }

        float s[2][4], vscale[2][4], vzero[2][4];
        float most = kNone;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            f32x4 dot = 0.f;
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                Frag f;
#pragma unroll
                for (int e = 0; e < 4; ++e) f.w[e] = I4 ? nibble_pair(t.k[u][i], e) : t.k[u][4 * i + e];
                dot = __builtin_amdgcn_mfma_f32_16x16x32_f16(f.v, q[i].v, dot, 0, 0, 0);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const bool there = page_there[u] && t0 + 16 * u + 4 * g + r < last;
                if constexpr (I4) {
                    const float ks = t.kp[u][r / 2][2 * (r % 2)], kz = t.kp[u][r / 2][2 * (r % 2) + 1];
                    vscale[u][r] = there ? t.vp[u][r / 2][2 * (r % 2)] : 1.f;
                    vzero[u][r] = there ? t.vp[u][r / 2][2 * (r % 2) + 1] : 0.f;
                    const float x = ks * fmaf(dot[r], score_unit, -kz * qz) + __builtin_amdgcn_logf(vscale[u][r]);
                    s[u][r] = there ? x : kNone;
                } else {
                    s[u][r] = there ? dot[r] * score_unit : kNone;
#pragma unroll
                    for (int e = 0; e < D / 32; ++e) t.v[u][r][e] = there ? t.v[u][r][e] : 0u;   // 0 times what lies there
                }
                most = fmaxf(most, s[u][r]);
            }
        }
        most = fmaxf(top, max_of_groups(most));
        const float base = most == kNone ? 0.f : most;
        const float shrink = __builtin_amdgcn_exp2f(top - base);
        total *= shrink;
        zsum *= shrink;
        top = most;
        Frag w;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float p = __builtin_amdgcn_exp2f(s[u][r] - base);
                w.h[4 * u + r] = (_Float16)p;
                if constexpr (I4) {
                    total = fmaf(p, __builtin_amdgcn_rcpf(vscale[u][r]), total);
                    zsum = fmaf((float)w.h[4 * u + r], vzero[u][r], zsum);
                } else {
                    total += p;
                }
            }
#pragma unroll
        for (int j = 0; j < C; ++j) acc[j] *= shrink;
        // half j of the row of token pairs (r, r + 1): two tokens per dword
        uint32_t lo[2][2], hi[2][2];
        if constexpr (I4) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    const uint32_t x = t.v[u][2 * p][0], y = t.v[u][2 * p + 1][0];
                    if constexpr (D == 128) {
                        lo[u][p] = low_halves(x, y), hi[u][p] = high_halves(x, y);
                    } else {
                        lo[u][p] = __builtin_amdgcn_perm(y, x, n & 1 ? 0x07060302u : 0x05040100u), hi[u][p] = 0;
                    }
                }
        }
#pragma unroll
        for (int j = 0; j < C; ++j) {
            Frag f;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    if constexpr (I4) {
                        const uint32_t x = j < 4 ? lo[u][p] : hi[u][p];
                        f.w[2 * u + p] = nibble_pair(x, j & 3);
                    } else {
                        const uint32_t x = t.v[u][2 * p][j / 2], y = t.v[u][2 * p + 1][j / 2];
                        f.w[2 * u + p] = j & 1 ? high_halves(x, y) : low_halves(x, y);
                    }
                }
            acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f.v, w.v, acc[j], 0, 0, 0);
        }
    }

    // the four waves meet: acc[j][r] of lane (n, g) is column d = C (4 g + r) + j of query row n
    __shared__ float s_top[kWaves][16], s_total[kWaves][16];
    __shared__ float s_acc[kWaves][16][D + 4];
    total = sum_of_groups(total);
    zsum = sum_of_groups(zsum);
    if (g == 0) s_top[wave][n] = top, s_total[wave][n] = total;
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < C; ++j) {
            float x = acc[j][r];
            if constexpr (I4) x = x * 1048576.f - zsum;
            s_acc[wave][n][C * (4 * g + r) + j] = x;
        }
    __syncthreads();
    for (int i = threadIdx.x; i < rows * (D / 4); i += 256) {
        const int m = i / (D / 4), d = 4 * (i % (D / 4));
        float most = s_top[0][m];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) most = fmaxf(most, s_top[w][m]);
        const float base = most == kNone ? 0.f : most;
        f32x4 sum = 0.f;
        float all = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float e = __builtin_amdgcn_exp2f(s_top[w][m] - base);
            sum += e * *reinterpret_cast<const f32x4 *>(&s_acc[w][m][d]);
            all += e * s_total[w][m];
        }
        if (a.splits == 1) {
            const float norm = all > 0.f ? 1.f / all : 0.f;
            _Float16 y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = (_Float16)(sum[e] * norm);
            *reinterpret_cast<u32x2 *>(a.o + (int64_t)b * a.ldo + (int64_t)(head0 + m) * D + d) = *reinterpret_cast<u32x2 *>(y);
        } else {
            const int64_t at = ((int64_t)b * a.heads + head0 + m) * a.splits + split;
            *reinterpret_cast<f32x4 *>(a.part + at * D + d) = sum;
            if (d == 0) *reinterpret_cast<float2 *>(a.part_ml + at * 2) = make_float2(most, all);
        }
    }
}

// the runs of one query head, joined by one workgroup: D / 4 threads per part of the runs
template <int D> __global__ __launch_bounds__(256) void attn_join_kernel(Decode a)
{
    constexpr int TPR = D / 4, PARTS = 256 / TPR;
    const uint32_t row = blockIdx.x;                     // sequence * heads + head
    const uint32_t b = row / a.heads, head = row - b * a.heads;
    const int64_t len = min((int64_t)max(a.lens[b], 0), a.max_len);
    const int runs = (int)((len + a.chunk - 1) / a.chunk);
    const int part = threadIdx.x / TPR, d = 4 * (threadIdx.x % TPR);
    const float *ml = a.part_ml + (int64_t)row * a.splits * 2, *sums = a.part + (int64_t)row * a.splits * D;
    float most = kNone, all = 0.f;
    f32x4 sum = 0.f;
    for (int i = part; i < runs; i += PARTS) {
        const float2 x = reinterpret_cast<const float2 *>(ml)[i];
        const f32x4 y = *reinterpret_cast<const f32x4 *>(sums + (int64_t)i * D + d);
        const float now = fmaxf(most, x.x), base = now == kNone ? 0.f : now;
        const float shrink = __builtin_amdgcn_exp2f(most - base), e = __builtin_amdgcn_exp2f(x.x - base);
        sum = sum * shrink + y * e;
        all = all * shrink + x.y * e;
        most = now;
    }
    __shared__ float s_top[PARTS], s_total[PARTS];
    __shared__ f32x4 s_sum[PARTS][TPR];
    if (d == 0) s_top[part] = most, s_total[part] = all;
    s_sum[part][d / 4] = sum;
    __syncthreads();
    if (part) return;
    float top = s_top[0];
#pragma unroll
    for (int p = 1; p < PARTS; ++p) top = fmaxf(top, s_top[p]);
    const float base = top == kNone ? 0.f : top;
    sum = 0.f, all = 0.f;
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
        const float e = __builtin_amdgcn_exp2f(s_top[p] - base);
        sum += s_sum[p][d / 4] * e;
        all += s_total[p] * e;
    }
    const float norm = all > 0.f ? 1.f / all : 0.f;
    _Float16 y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (_Float16)(sum[e] * norm);
    *reinterpret_cast<u32x2 *>(a.o + (int64_t)b * a.ldo + (int64_t)head * D + d) = *reinterpret_cast<u32x2 *>(y);
}

// Runs per sequence: enough workgroups for four on every compute unit, none shorter than one round of the waves.
struct Runs { int splits, chunk; };
Runs runs_of(int64_t n_seqs, int64_t kv, int64_t group, int64_t max_len)
{
    constexpr int64_t round = kWaves * kTile;
    const int64_t pairs = n_seqs * kv * ((group + 15) / 16), want = (int64_t)compute_units() * 4;
    const int64_t rounds = (max_len + round - 1) / round;
    int64_t splits = (want + pairs - 1) / pairs;
    if (splits > rounds) splits = rounds;
    const int64_t chunk = (rounds + splits - 1) / splits * round;
    return {(int)((max_len + chunk - 1) / chunk), (int)chunk};
}

}  // namespace

size_t attn_decode_workspace_bytes(int64_t n_seqs, int64_t n_heads, int64_t kv, int64_t dim, int64_t max_len)
{
    const Runs r = runs_of(n_seqs, kv, n_heads / kv, max_len);
    return r.splits > 1 ? (size_t)n_seqs * n_heads * r.splits * (dim + 2) * 4 : 0;
}

hipError_t launch_attn_decode(const void *Q, int64_t ldq, int64_t n_seqs, int64_t n_heads, const KvCache &c, const int32_t *table,
                              int64_t max_pages, int64_t ld_table, const int32_t *lens, float scale, void *O, int64_t ldo,
                              void *workspace, hipStream_t st)
{
    Decode a;
    const int64_t max_len = max_pages * c.page_size;
    const Runs r = runs_of(n_seqs, c.heads, n_heads / c.heads, max_len);
    a.q = static_cast<const _Float16 *>(Q), a.ldq = ldq;
    a.heads = (int)n_heads, a.kv = (int)c.heads, a.group = (int)(n_heads / c.heads), a.row_tiles = (a.group + 15) / 16;
    a.K = c.K, a.V = c.V, a.Kp = c.Kp, a.Vp = c.Vp;
    a.n_pages = (uint32_t)c.pages, a.page_shift = __builtin_ctzll((unsigned long long)c.page_size);
    a.table = table, a.ld_table = ld_table, a.max_len = max_len, a.lens = lens;
    a.scale = scale * 1.4426950408889634f;
    a.splits = r.splits, a.chunk = r.chunk;
    a.o = static_cast<_Float16 *>(O), a.ldo = ldo;
    a.part = static_cast<float *>(workspace);
    a.part_ml = a.part + (size_t)n_seqs * n_heads * r.splits * c.dim;
    const dim3 grid((unsigned)(n_seqs * c.heads * a.row_tiles * r.splits)), block(kWaves * 64);
    if (c.dim == 128 && c.i4) hipLaunchKernelGGL((attn_decode_kernel<128, true>), grid, block, 0, st, a);
    else if (c.dim == 128) hipLaunchKernelGGL((attn_decode_kernel<128, false>), grid, block, 0, st, a);
    else if (c.i4) hipLaunchKernelGGL((attn_decode_kernel<64, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((attn_decode_kernel<64, false>), grid, block, 0, st, a);
    if (hipError_t e = hipGetLastError(); e != hipSuccess || r.splits == 1) return e;
    const dim3 rows((unsigned)(n_seqs * n_heads));
    if (c.dim == 128) hipLaunchKernelGGL((attn_join_kernel<128>), rows, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((attn_join_kernel<64>), rows, dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace sr

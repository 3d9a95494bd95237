// Attention of whole prompts: packed sequences of different lengths, grouped heads, causal or not.
//
//   o_i = sum_j softmax(scale q_i . k_j) v_j      over the keys j of row i's own sequence, j <= i + (keys - queries) if causal
//
// Bound by the matrix pipe and the exponentials beside it.  A workgroup takes 128 query rows of one head, 32 per wave, and
// walks over its keys 64 at a time with a running maximum and sum; keys and values come into LDS by DMA, one tile ahead.
// Both products run on 32 x 32 x 16 matrix instructions with the query row in the columns:
//
//   S^T = K Q^T   lane (m, g) = (lane % 32, lane / 32) gets the scores of row m and of tokens 8 i + 4 g + (0 .. 3)
//   O^T = V^T P^T its k-index is the token: the eight weights that a lane supplies per instruction are those of tokens
//                 4 g + (0 .. 3) and 8 + 4 g + (0 .. 3) of sixteen, which it got itself
//
// so weights stay in the lane that computed them, a row's maximum and sum are one lane's and its neighbour 32 further, and
// values are read from LDS with the transposing 8-byte read (four tokens of one column per lane).  Weights are rounded to fp16
// for the matrix pipe (they are at most 1: half a step is 2^-12 of one); scores, maxima, sums and outputs are held in fp32.
#include "gemm_common.h"

namespace sr {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
union Frag { f16x8 v; s16x4 s[2]; u32x4 w; _Float16 h[8]; };

constexpr int kRows = 128, kKeys = 64;                   // query rows of a workgroup, keys of a tile
constexpr float kNone = -__builtin_inff();

struct Prefill {
    const _Float16 *q, *k, *v;
    int64_t ldq, ldk, ldv;
    const int32_t *cu_q, *cu_k;
    int n_seqs, tokens_q, tokens_k;
    int heads, kv, tiles;                                // tiles: of query rows, an upper bound
    int causal;
    float scale, per_scale;                              // times log2(e); its reciprocal
    _Float16 *o;
    int64_t ldo;
};

// where sequence i of a packed batch lies; ends that do not fit are cut, never followed
__device__ __forceinline__ void span(const int32_t *cu, int i, int tokens, int &begin, int &length)
{
    begin = min(max(cu[i], 0), tokens);
    length = min(max(cu[i + 1], begin), tokens) - begin;
}

// the sequence that holds the tile-th tile of query rows, and which of its tiles that is; false behind the last
__device__ __forceinline__ bool find_tile(const Prefill &a, int tile, int lane, int &seq, int &local)
{
    for (int s0 = 0; s0 < a.n_seqs; s0 += 64) {
        int n = 0;
        if (s0 + lane < a.n_seqs) {
            int begin, length;
            span(a.cu_q, s0 + lane, a.tokens_q, begin, length);
            n = (length + kRows - 1) / kRows;
        }
        int upto = n;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int other = __shfl_up(upto, d, 64);
            upto += lane >= d ? other : 0;
        }
        const unsigned long long past = __ballot(upto > tile);
        if (past) {
            const int at = __builtin_ctzll(past);
            seq = s0 + at;
            local = __builtin_amdgcn_readfirstlane(tile - __shfl(upto - n, at, 64));
            return true;
        }
        tile -= __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

template <int D> __global__ __launch_bounds__(256, 2) void attn_prefill_kernel(Prefill a)
{
    constexpr int CH = D / 8;                            // 16-byte chunks of a row
    constexpr uint32_t kTileBytes = kKeys * D * 2;
    constexpr int DT = D / 32, LOADS = kKeys * CH / 256; // column tiles; DMA loads of a wave per operand
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)smem;   // [2][keys, values]
    const int lane = threadIdx.x & 63, m = lane & 31, g = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t x = blockIdx.x % (uint32_t)a.heads;
    const int kvh = (int)(x % (uint32_t)a.kv), head = kvh * (a.heads / a.kv) + (int)(x / (uint32_t)a.kv);
    int seq, local;
    if (!find_tile(a, a.tiles - 1 - (int)(blockIdx.x / (uint32_t)a.heads), lane, seq, local)) return;
    int q0, nq, k0, nk;
    span(a.cu_q, seq, a.tokens_q, q0, nq);
    span(a.cu_k, seq, a.tokens_k, k0, nk);
    q0 = __builtin_amdgcn_readfirstlane(q0), nq = __builtin_amdgcn_readfirstlane(nq);
    k0 = __builtin_amdgcn_readfirstlane(k0), nk = __builtin_amdgcn_readfirstlane(nk);
    const int r0 = local * kRows, shift = nk - nq;
    const int end = a.causal ? min(nk, min(r0 + kRows, nq) + shift) : nk;              // keys that any row sees
    const int w0 = r0 + 32 * wave, row = w0 + m;
    const int wend = a.causal ? min(nk, min(w0 + 32, nq) + shift) : nk;                // .. of this wave
    const int rend = a.causal ? min(nk, row + shift + 1) : nk;                         // .. of this lane's row
    const int whole = a.causal ? min(nk, w0 + shift + 1) : nk;                         // keys that every row of the wave sees

    Frag q[D / 16];
    {
        const _Float16 *src = a.q + (int64_t)(q0 + min(row, nq - 1)) * a.ldq + (int64_t)head * D + 8 * g;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) q[i].v = *reinterpret_cast<const f16x8 *>(src + 16 * i);
    }
    f32x16 acc[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) acc[t] = 0.f;
    // Weights are exp2(score - base), a row's largest about 2^7 when base is set, and base is set again only where one would pass
    // 2^15: fp16 has room for that, its subnormals begin 2^-21 below the largest, and most tiles rescale nothing.
    float top = kNone, limit = kNone, base = 0.f, total = 0.f;

    // Tiles lie in LDS by rows, their chunks swapped so that the lanes that read at once meet every bank: keys, read 32 rows
    // of one chunk at a time, by row; values, read 4 rows of four neighbouring chunks, by row in steps of four chunks.
    const uint8_t *kb = reinterpret_cast<const uint8_t *>(a.k + (int64_t)k0 * a.ldk + (int64_t)kvh * D);
    const uint8_t *vb = reinterpret_cast<const uint8_t *>(a.v + (int64_t)k0 * a.ldv + (int64_t)kvh * D);
    auto key_swap = [](int r) { return D == 128 ? r & 15 : (r >> 1) & 7; };
    auto value_swap = [](int r) { return D == 128 ? (r & 3) << 2 : ((r >> 1) & 1) << 2; };
    uint32_t k_off[LOADS], v_off[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int at = (i * 4 + wave) * 64 + lane, r = at / CH, c = at % CH;
        k_off[i] = r * (uint32_t)(a.ldk * 2) + 16 * (c ^ key_swap(r));
        v_off[i] = r * (uint32_t)(a.ldv * 2) + 16 * (c ^ value_swap(r));
    }
    auto load = [&](int t0, int slot) {
        const uint8_t *kt = kb + (int64_t)t0 * a.ldk * 2, *vt = vb + (int64_t)t0 * a.ldv * 2;
        const uint32_t to = lds + slot * 2 * kTileBytes + wave * 1024;
        if (t0 + kKeys <= nk) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                dma16(kt, k_off[i], to + 4096 * i);
                dma16(vt, v_off[i], to + 4096 * i + kTileBytes);
            }
        } else {                                         // rows past the end: the last one again
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int r = ((i * 4 + wave) * 64 + lane) / CH;
                const uint32_t over = (uint32_t)max(r - (nk - 1 - t0), 0);
                dma16(kt, k_off[i] - over * (uint32_t)(a.ldk * 2), to + 4096 * i);
                dma16(vt, v_off[i] - over * (uint32_t)(a.ldv * 2), to + 4096 * i + kTileBytes);
            }
        }
    };

    const int n_tiles = end > 0 ? (end + kKeys - 1) / kKeys : 0, mine = wend > 0 ? (wend + kKeys - 1) / kKeys : 0;
    // the tile that was asked for a round ago is there, and everybody is done with the slot of the next one
    auto turn = [&](int i) {
        wait_vmcnt<0>();
        barrier_nofence();
        if (i + 1 < n_tiles) load((i + 1) * kKeys, (i + 1) & 1);
    };
    if (n_tiles) load(0, 0);
    for (int i = 0; i < mine; ++i) {
        const int t0 = i * kKeys;
        turn(i);
        const uint8_t *ks = smem + (i & 1) * 2 * kTileBytes, *vs = ks + kTileBytes;
        f32x16 s[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            s[u] = 0.f;
            const int r = 32 * u + m;
#pragma unroll
            for (int d = 0; d < D / 16; ++d) {
                Frag k;
                k.v = *reinterpret_cast<const f16x8 *>(ks + r * (D * 2) + 16 * ((2 * d + g) ^ key_swap(r)));
                s[u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k.v, q[d].v, s[u], 0, 0, 0);
            }
        }
        if (t0 + kKeys > whole) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (t0 + 32 * u + 8 * (e / 4) + 4 * g + (e & 3) >= rend) s[u][e] = kNone;
        }
        float most = kNone;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 16; ++e) most = fmaxf(most, s[u][e]);
        if (!__all(most <= limit)) {
            most = fmaxf(fmaxf(most, __shfl_xor(most, 32, 64)), top);
            const float shrink = most == kNone ? 1.f : __builtin_amdgcn_exp2f((top - most) * a.scale);
            total *= shrink;
#pragma unroll
            for (int t = 0; t < DT; ++t) acc[t] *= shrink;
            top = most, limit = most + 8.f * a.per_scale;
            base = most == kNone ? 0.f : most * a.scale - 7.f;
        }
#pragma unroll
        for (int step = 0; step < 4; ++step) {
            Frag w;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float p = __builtin_amdgcn_exp2f(fmaf(s[step / 2][8 * (step & 1) + e], a.scale, -base));
                total += p;
                w.h[e] = (_Float16)p;
            }
#pragma unroll
            for (int t = 0; t < DT; ++t) {
                Frag v;
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int r = 16 * step + 8 * half + 4 * g + ((lane >> 2) & 3);
                    const int c = 4 * t + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
                    const uint8_t *p = vs + r * (D * 2) + 16 * (c ^ value_swap(r)) + 8 * (lane & 1);
                    v.s[half] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)p);
                }
                acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v.v, w.v, acc[t], 0, 0, 0);
            }
        }
    }
    for (int i = mine; i < n_tiles; ++i) turn(i);        // tiles that only later rows see
    total += __shfl_xor(total, 32, 64);
    if (row >= nq) return;
    const float norm = total > 0.f ? 1.f / total : 0.f;
    _Float16 *dst = a.o + (int64_t)(q0 + row) * a.ldo + (int64_t)head * D + 4 * g;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            union { _Float16 h[4]; uint2 u; } y;
#pragma unroll
            for (int r = 0; r < 4; ++r) y.h[r] = (_Float16)(acc[t][4 * e + r] * norm);
            *reinterpret_cast<uint2 *>(dst + 32 * t + 8 * e) = y.u;
        }
}

template <int D> hipError_t launch_dim(const Prefill &a, hipStream_t st)
{
    constexpr int bytes = 4 * kKeys * D * 2;
    if (hipError_t e = allow_dynamic_lds<attn_prefill_kernel<D>>(bytes); e != hipSuccess) return e;
    hipLaunchKernelGGL((attn_prefill_kernel<D>), dim3((unsigned)((int64_t)a.tiles * a.heads)), dim3(256), bytes, st, a);
    return hipGetLastError();
}

}  // namespace

int64_t attn_prefill_workgroups(int64_t T_q, int64_t n_seqs, int64_t n_heads)
{
    return (T_q / kRows + (n_seqs < T_q ? n_seqs : T_q)) * n_heads;      // every sequence may end inside a tile
}

hipError_t launch_attn_prefill(const void *Q, int64_t ldq, const void *K, int64_t ldk, const void *V, int64_t ldv,
                               const int32_t *cu_q, const int32_t *cu_k, int64_t n_seqs, int64_t T_q, int64_t T_k, int64_t n_heads,
                               int64_t kv, int64_t dim, bool causal, float scale, void *O, int64_t ldo, hipStream_t st)
{
    Prefill a;
    a.q = static_cast<const _Float16 *>(Q), a.k = static_cast<const _Float16 *>(K), a.v = static_cast<const _Float16 *>(V);
    a.ldq = ldq, a.ldk = ldk, a.ldv = ldv;
    a.cu_q = cu_q, a.cu_k = cu_k;
    a.n_seqs = (int)n_seqs, a.tokens_q = (int)T_q, a.tokens_k = (int)T_k;
    a.heads = (int)n_heads, a.kv = (int)kv, a.tiles = (int)(attn_prefill_workgroups(T_q, n_seqs, n_heads) / n_heads);
    a.causal = causal, a.scale = scale * 1.4426950408889634f, a.per_scale = 1.f / a.scale;
    a.o = static_cast<_Float16 *>(O), a.ldo = ldo;
    return dim == 128 ? launch_dim<128>(a, st) : launch_dim<64>(a, st);
}

}  // namespace sr

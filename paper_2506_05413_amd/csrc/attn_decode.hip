// Attention of one new token per sequence over a paged cache, split over the cache's length and joined.
//
//   s_t = scale q . k_t,   o = sum_t softmax(s)_t v_t     over the tokens t < length whose page exists
//
// Bound by the bytes of the cache where it is long (4 bits, 8 key/value heads of 128: 64 sequences of 0 .. 8192 tokens, 294 MB, in
// 55 us = 5.3 TB/s; fp16, 32 heads of 64: 24 sequences of 0 .. 2000 tokens, 239 MB, in 45 us), else by the launch and the chain of
// loads and tiles of one sequence (130 tokens 5.5 us, 0.7 us for a wave's tile; 65000 tokens, 75 MB, 21 us with the join).  A workgroup
// takes one key/value head (up to 16 of the query heads that share it) and runs of tokens; its waves walk over tiles of 32 tokens
// with a running maximum and sum, and meet in LDS.  (More query heads to a key/value head are workgroups of their own, each of which
// asks for the cache again: 64 sequences of 0 .. 8192 tokens, 37 MB, 16 query heads on one key/value head 20.5 us, 32 26.9.)  Both products run on 16 x 16 x 32 matrix instructions with the query head in
// the columns:
//
//   S^T = K Q^T   rows = tokens: lane (n, g) = (lane % 16, lane / 16) holds token n of the operand and gets tokens 4 g + r
//   O^T = V^T P^T its k-index is the token: lane (n, g) supplies the eight tokens 4 g + r of two halves of the tile, which are
//                 the ones it got scores for, so the weights go from one product to the next inside the lane
//
// Where up to 4 (8) query heads share a key/value head, the sixteen columns hold 4 (2) copies of them (4 bits), and a copy forms the
// weights of every fourth (of every other pair of) token only, zeros for the rest, so that no lane forms a weight that another has
// too; the copies' sums are added up at the end (64 sequences of 0 .. 8192 tokens 57.3 -> 55.3 us, 16 of 2000 14.7 -> 13.5, 200 of up
// to 500 20.7 -> 18.9).
//
// The order of channels in the first product and of columns in the second is free, so both operands are taken as they lie in
// memory, and the sums over codes need no conversion: a code c in bits 4-7 of a half is the subnormal fp16 number c 2^-20, a
// shift and an AND per two codes.  (The matrix pipe takes subnormal operands; measured on random weights, sums over c 2^-20 are
// as exact as over c itself, to 2^-22, while over c 2^-24, bits 0-3, they are off by 2^-14 of a code.)  With scale d and zero z
// per token,
//   s_t = d (q . c - z sum(q)),   o = sum_t w_t (c_t - z_t),   w_t = p_t d_t
// where p = 2^(s log2(e) - top - lift), top the maximum of the scores and lift that of the tokens' (score - top) + log2(d): weights
// w then are at most 2^8 however large or small the values are, and lose nothing to the range of fp16.  (One sum of the two would
// not do: beside a score of 2^28 it has no room for the other.)  Scores, p, maxima and sums are fp32.  w is rounded to fp16, the type of
// the matrix pipe's operands (half a step, 2^-11 of it; the same rounded w multiplies z): what that leaves would be another operand
// and a second product for every tile, and is less than the rounding of the output (rms distance from 64 bits over normal values
// 2.3e-4 of them, and 2.1e-4 without it).  The denominator is the sum of p as it is: at 4 bits w is p times the token's step, and the sum of
// the rounded w is none of the rounded p.  (Prompts have fp16 values, hence w = p, and divide by the sum of the rounded ones.)
#include "gemm_common.h"

namespace sr {
namespace {

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
union Frag { f16x8 v; uint32_t w[4]; _Float16 h[8]; };

constexpr int kWaves = 4, kTile = 32, kRound = kWaves * kTile;
constexpr float kNone = -__builtin_inff(), kLeastLift = -40.f;

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
    int n_seqs, per_seq;                 // per_seq: key/value heads * row tiles
    int shares;                          // workgroups that share the sequences of one of those; 0: one workgroup per sequence
    _Float16 *o;
    int64_t ldo;
    float *part;                         // [per_seq][share][2][row][D] sums, then [..][row][2] maximum, total
    float *part_ml;
};

// ---- the shares ------------------------------------------------------------------------------------------------------
// The sequences' rounds (of kRound tokens, a tile per wave) lie behind each other in one line, and share w takes the rounds
// [w, w + 1) * size of it: pieces of several sequences, or a piece of one.  Sizes follow from the lengths, which are known on
// the device only, so every wave adds them up itself.  A sequence inside one share is finished there; else the share in which
// it begins leaves a partial result in place 1, the others leave theirs in place 0, and the second kernel joins them.
// (64 sequences of 0 .. 8192 tokens, 8 key/value heads of 128, 4 bits, 294 MB: cutting every sequence into 2, 4 or 8 runs took 1.3
// times as long as the shares, with an earlier form of the tiles.)
__device__ __forceinline__ int length_of(const Decode &a, int b) { return (int)min((int64_t)max(a.lens[b], 0), a.max_len); }
__device__ __forceinline__ int rounds_of(const Decode &a, int b) { return b < a.n_seqs ? (length_of(a, b) + kRound - 1) / kRound : 0; }

// rounds in a share
__device__ __forceinline__ int share_size(const Decode &a, int lane)
{
    int sum = 0;
    for (int b0 = 0; b0 < a.n_seqs; b0 += 64) sum += rounds_of(a, b0 + lane);
    const int all = __builtin_amdgcn_readlane(scan_of_wave(sum), 63);
    return max((all + a.shares - 1) / a.shares, 1);
}
// rounds of the sequences before b
__device__ __forceinline__ int rounds_before(const Decode &a, int b, int lane)
{
    int sum = 0;
    for (int b0 = 0; b0 < b; b0 += 64) sum += b0 + lane < b ? rounds_of(a, b0 + lane) : 0;
    return __builtin_amdgcn_readlane(scan_of_wave(sum), 63);
}
// the sequence that holds round `at` of the line, and the rounds before it; n_seqs behind the last
__device__ __forceinline__ int sequence_at(const Decode &a, int at, int lane, int &before)
{
    before = 0;
    for (int b0 = 0; b0 < a.n_seqs; b0 += 64) {
        const int n = rounds_of(a, b0 + lane), upto = before + scan_of_wave(n);
        const unsigned long long past = __ballot(upto > at);
        if (past) {
            const int l = __builtin_ctzll(past);
            before = __builtin_amdgcn_readlane(upto - n, l);
            return b0 + l;
        }
        before = __builtin_amdgcn_readlane(upto, 63);
    }
    return a.n_seqs;
}

// ---- tiles -----------------------------------------------------------------------------------------------------------
// reductions over the lanes that share a query row: the four with one lane % 16, and the copies of that
template <int COPIES> __device__ __forceinline__ float max_of_groups(float v)
{
    v = fmaxf(v, __shfl_xor(v, 16, 64));
    v = fmaxf(v, __shfl_xor(v, 32, 64));
    if constexpr (COPIES > 1) v = fmaxf(v, lane_perm<0x128>(v));             // rotations by 8 and by 4 of 16
    if constexpr (COPIES > 2) v = fmaxf(v, lane_perm<0x124>(v));
    return v;
}
template <int COPIES> __device__ __forceinline__ float sum_of_copies(float v)
{
    if constexpr (COPIES > 1) v += lane_perm<0x128>(v);
    if constexpr (COPIES > 2) v += lane_perm<0x124>(v);
    return v;
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

// A wave's share of 32 tokens in registers.  Whole runs of 16 tokens lie in one page, so that a half of the tile has one address
// for the wave and fixed offsets per lane.
template <int D, bool I4, int COPIES> struct Tile {
    static constexpr int N = 4 / COPIES;                 // tokens of a half whose weights are this lane's: 4 g + N copy + (0 .. N - 1)
    static constexpr int KW = I4 ? D / 32 : D / 8;       // dwords of a lane's share of a key
    static constexpr int VW = I4 ? 1 : D / 32;           // dwords of a lane's share of a value
    static constexpr int ROW = I4 ? D / 2 : D * 2;       // bytes of a row
    uint32_t k[2][KW], v[2][4][VW];
    float ks[2][N], kz[2][N], vs[2][N], vz[2][N];        // their scales and zeros
};

// 4 bits: a tile waits in LDS as keys, values and parameters (two halves each; keys' first), two tiles per wave
template <int D> struct Stage {
    static constexpr int V = 16 * D, P = 32 * D, BYTES = 32 * D + 512;       // offsets of values and parameters
};

// 16 bytes per lane from addresses of its own to LDS bytes [lds, lds + 1024), in the order of the lanes.  The cache is read once:
// with loads that allocate in the caches 64 sequences of 4096 tokens (303 MB) take 60.7 us, with these 53.5.
__device__ __forceinline__ void dma16_once(const void *p, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off nt" ::"s"(lds), "v"(p) : "memory", "m0");
}

// The query rows of a workgroup, and their state over the tokens that a wave has seen.
template <int D, bool I4, int COPIES> struct Rows {
    static constexpr int C = D / 16;                     // output columns per lane and row index: d = C n + j
    using T = Tile<D, I4, COPIES>;
    static constexpr int N = T::N;
    Frag q[D / 32];
    float unit, qz;                                      // score of one product; its sum(q)
    f32x4 acc[C];                                        // sums of w c 2^-20, or w v
    float top, lift, total, zsum;                        // maximum; sums of p and w z over this lane's tokens

    // row n of q, in the order that the keys lie in; zeros for a row that is not there
    __device__ __forceinline__ void begin(const _Float16 *src, bool there, int g, float scale)
    {
        float qsum = 0.f;
        if constexpr (I4) {
            constexpr int per = D / 4;                   // codes of a key in one lane, a fragment per dword
#pragma unroll
            for (int p = 0; p < per / 8; ++p) {
                Frag f;
                f.v = there ? *reinterpret_cast<const f16x8 *>(src + per * g + 8 * p) : (f16x8)(_Float16)0;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    q[p].h[e] = f.h[e / 2 + 4 * (e & 1)];                    // halves of nibble_pair()
                    qsum += (float)f.h[e];
                }
            }
            qsum = sum_of_groups(qsum);
        } else {
#pragma unroll
            for (int i = 0; i < D / 32; ++i) q[i].v = there ? *reinterpret_cast<const f16x8 *>(src + 32 * i + 8 * g) : (f16x8)(_Float16)0;
        }
        unit = I4 ? scale * 1048576.f : scale, qz = qsum * scale;
#pragma unroll
        for (int j = 0; j < C; ++j) acc[j] = 0.f;
        top = kNone, lift = 0.f, total = 0.f, zsum = 0.f;
    }

    // 32 tokens from `at` on, those before `last` whose page is there (bit u: of half u)
    __device__ __forceinline__ void use(T &t, int at, int last, uint32_t pages_there, int n, int g, int copy)
    {
#pragma clang fp contract(off)                            // a score minus the maximum of the rounded ones is exact near it
        float y[2][N];                                   // scores over log(2)
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
            for (int i = 0; i < N; ++i) {
                const float x = COPIES == 1 ? dot[i] : COPIES == 2 ? (copy ? dot[2 + i] : dot[i]) : copy & 2 ? (copy & 1 ? dot[3] : dot[2]) : copy & 1 ? dot[1] : dot[0];
                y[u][i] = I4 ? fmaf(x, unit, -t.kz[u][i] * qz) * t.ks[u][i] : x * unit;
            }
        }
        if (pages_there != 3 || at + kTile > last) {     // a token that is not there: score minus infinity, a finite value
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int r = 0; r < N; ++r) {
                    const bool there = (pages_there >> u & 1) && at + 16 * u + 4 * g + N * copy + r < last;
                    y[u][r] = there ? y[u][r] : kNone;
                    if constexpr (I4) {
                        t.vs[u][r] = there ? t.vs[u][r] : 1.f;
                        t.vz[u][r] = there ? t.vz[u][r] : 0.f;
                    } else {
#pragma unroll
                        for (int e = 0; e < T::VW; ++e) t.v[u][r][e] = there ? t.v[u][r][e] : 0u;
                    }
                }
        }
        float p[2][N], w[2][N];
        auto weights = [&] {
            float most = 0.f;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int r = 0; r < N; ++r) {
                    p[u][r] = __builtin_amdgcn_exp2f(I4 ? y[u][r] - top - lift : y[u][r] - top);
                    w[u][r] = I4 ? p[u][r] * t.vs[u][r] : p[u][r];
                    most = fmaxf(most, w[u][r]);
                }
            return most;
        };
        // Weights stay below 2^8 relative to a maximum that is replaced only when one does not (the first tile's always): fp16
        // has room for that, and most tiles then rescale nothing.
        if (!__all(weights() <= 256.f && top != kNone)) {
            float most = kNone, raised = kLeastLift;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int r = 0; r < N; ++r) most = fmaxf(most, y[u][r]);
            most = fmaxf(top, max_of_groups<COPIES>(most));
            if constexpr (I4) {
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int r = 0; r < N; ++r)
                        if (most != kNone) raised = fmaxf(raised, y[u][r] - most + __builtin_amdgcn_logf(t.vs[u][r]));
                raised = max_of_groups<COPIES>(raised);
                if (top != kNone) raised = fmaxf(raised, top - most + lift);
            }
            const float shrink = most == kNone ? 1.f : __builtin_amdgcn_exp2f(I4 ? top - most + (lift - raised) : top - most);
            if (I4 && most != kNone) lift = raised;
            total *= shrink;
            zsum *= shrink;
#pragma unroll
            for (int j = 0; j < C; ++j) acc[j] *= shrink;
            top = most == kNone ? 0.f : most;            // minus infinity from itself would be no number
            weights();
            top = most;
        }
        Frag f16w;                                       // of tokens 4 u + r; zeros for those of other copies
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if constexpr (COPIES == 1) {
#pragma unroll
                for (int i = 0; i < 4; ++i) f16w.h[4 * u + i] = (_Float16)w[u][i];
            } else if constexpr (COPIES == 2) {
                const f16x2 pair = {(_Float16)w[u][0], (_Float16)w[u][1]};
                const uint32_t x = __builtin_bit_cast(uint32_t, pair);
                f16w.w[2 * u] = copy ? 0u : x, f16w.w[2 * u + 1] = copy ? x : 0u;
            } else {
                const uint32_t x = (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)w[u][0]) << (16 * (copy & 1));
                f16w.w[2 * u] = copy & 2 ? 0u : x, f16w.w[2 * u + 1] = copy & 2 ? x : 0u;
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                total += p[u][i];
                if constexpr (I4) zsum = fmaf((float)(_Float16)w[u][i], t.vz[u][i], zsum);
            }
        }
        // column j of token pairs (r, r + 1): two tokens per dword
        uint32_t lo[2][2], hi[2][2];
        if constexpr (I4) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint32_t x = t.v[u][2 * i][0], z = t.v[u][2 * i + 1][0];
                    if constexpr (D == 128) {
                        lo[u][i] = low_halves(x, z), hi[u][i] = high_halves(x, z);
                    } else {
                        lo[u][i] = __builtin_amdgcn_perm(z, x, n & 1 ? 0x07060302u : 0x05040100u), hi[u][i] = 0;
                    }
                }
        }
#pragma unroll
        for (int j = 0; j < C; ++j) {
            Frag f;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if constexpr (I4) {
                        f.w[2 * u + i] = nibble_pair(j < 4 ? lo[u][i] : hi[u][i], j & 3);
                    } else {
                        const uint32_t x = t.v[u][2 * i][j / 2], z = t.v[u][2 * i + 1][j / 2];
                        f.w[2 * u + i] = j & 1 ? high_halves(x, z) : low_halves(x, z);
                    }
                }
            acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f.v, f16w.v, acc[j], 0, 0, 0);
        }
    }
};

// Tokens [first, last) of sequence b over a wave's tiles, `smem` the wave's own stages (4 bits).
template <int D, bool I4, int COPIES, int WAVES>
__device__ __forceinline__ void walk(const Decode &a, Rows<D, I4, COPIES> &rows, int b, int h, int first, int last, uint8_t *smem, int wave, int lane)
{
    using T = Tile<D, I4, COPIES>;
    constexpr int ROUND = WAVES * kTile;
    const int n = lane & 15, g = lane >> 4, copy = n / (16 / COPIES);
    // (constant while the kernel runs: scalar loads, which the vector counter does not see)
    const auto *table = (const __attribute__((address_space(4))) int32_t *)(uintptr_t)(a.table + (int64_t)b * a.ld_table);
    const int page_mask = (1 << a.page_shift) - 1;
    // Tokens past the end read the last rows there are and count for nothing; so do those of a page that does not exist, from
    // page 0.  `there`: bit u, the page of half u exists.
    struct Where { int64_t row0, row1; uint32_t there; };
    struct Pages { int id[2]; };
    auto half_at = [&](int t0, int u) { return min(t0 + 16 * u, (last - 1) & ~15); };
    auto pages_of = [&](int t0) {
        Pages p;
#pragma unroll
        for (int u = 0; u < 2; ++u) p.id[u] = table[half_at(t0, u) >> a.page_shift];
        return p;
    };
    auto where = [&](int t0, const Pages &p) {
        Where w;
        w.there = 0;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint32_t id = (uint32_t)__builtin_amdgcn_readfirstlane(p.id[u]);
            const bool there = id < a.n_pages;
            w.there |= there ? 1u << u : 0u;
            (u ? w.row1 : w.row0) = (((int64_t)(there ? id : 0u) * a.kv + h) << a.page_shift) + (half_at(t0, u) & page_mask);
        }
        return w;
    };
    auto half_of = [&](const void *side, int64_t row) { return static_cast<const uint8_t *>(side) + row * T::ROW; };

    int t0 = first + wave * kTile;
    if (t0 >= last) return;
    if constexpr (I4) {
        // Rows come by DMA into two stages of the wave's own, a tile being loaded while another waits: registers hold one tile.
        // Page numbers are fetched a tile before that.  Lanes load in the order of memory; keys land with the chunks of row n
        // swapped by n / 4 and values with the rows in the order 4 (t % 4) + t / 4, so that both are read back without bank
        // conflicts.  A stage is loaded again behind a wait for the reads of it.
        constexpr int CPR = D / 32;                      // 16-byte chunks of a row
        const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)smem;
        const int row = (lane / CPR) & 15, chunk = lane % CPR;
        const uint32_t k_off = row * T::ROW + 16 * (D == 128 ? chunk ^ (row >> 2) : chunk);
        const uint32_t v_off = (D == 128 ? 4 * (row & 3) + (row >> 2) : row) * T::ROW + 16 * chunk;
        auto load = [&](int slot, const Where &w) {
            const uint32_t to = lds + slot * Stage<D>::BYTES;
            if constexpr (D == 128) {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    dma16_once(half_of(a.K, u ? w.row1 : w.row0) + k_off, to + 1024 * u);
                    dma16_once(half_of(a.V, u ? w.row1 : w.row0) + v_off, to + Stage<D>::V + 1024 * u);
                }
            } else {                                     // both halves at once
                dma16_once(half_of(a.K, w.row0 + (lane < 32 ? 0 : w.row1 - w.row0)) + k_off, to);
                dma16_once(half_of(a.V, w.row0 + (lane < 32 ? 0 : w.row1 - w.row0)) + v_off, to + Stage<D>::V);
            }
            if (lane < 32)                               // keys' two halves, then values'
                dma16_once(reinterpret_cast<const uint8_t *>(lane < 16 ? a.Kp : a.Vp) + (w.row0 + (lane & 8 ? w.row1 - w.row0 : 0)) * 8 + 16 * (lane & 7), to + Stage<D>::P);
        };
        constexpr int LOADS = D == 128 ? 5 : 3;          // of a tile
        auto fetch = [&](T &t, int slot) {
            const uint8_t *from = smem + slot * Stage<D>::BYTES;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if constexpr (D == 128) {
                    const u32x4 x = *reinterpret_cast<const u32x4 *>(from + 1024 * u + 64 * n + 16 * (g ^ (n >> 2)));
#pragma unroll
                    for (int i = 0; i < 4; ++i) t.k[u][i] = x[i];
                } else {
                    const u32x2 x = *reinterpret_cast<const u32x2 *>(from + 512 * u + 32 * n + 8 * g);
                    t.k[u][0] = x[0], t.k[u][1] = x[1];
                }
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    t.v[u][r][0] = *reinterpret_cast<const uint32_t *>(from + Stage<D>::V + (D == 128 ? 1024 * u + 64 * (4 * r + g) + 4 * n : 512 * u + 32 * (4 * g + r) + 4 * (n >> 1)));
                const uint8_t *params = from + Stage<D>::P + 128 * u + 32 * g;
                if constexpr (COPIES == 4) {
                    const float2 kp = *reinterpret_cast<const float2 *>(params + 8 * copy), vp = *reinterpret_cast<const float2 *>(params + 256 + 8 * copy);
                    t.ks[u][0] = kp.x, t.kz[u][0] = kp.y, t.vs[u][0] = vp.x, t.vz[u][0] = vp.y;
                } else {
#pragma unroll
                    for (int i = 0; i < T::N / 2; ++i) {
                        const f32x4 kp = *reinterpret_cast<const f32x4 *>(params + 16 * (i + copy)), vp = *reinterpret_cast<const f32x4 *>(params + 256 + 16 * (i + copy));
                        t.ks[u][2 * i] = kp[0], t.kz[u][2 * i] = kp[1], t.ks[u][2 * i + 1] = kp[2], t.kz[u][2 * i + 1] = kp[3];
                        t.vs[u][2 * i] = vp[0], t.vz[u][2 * i] = vp[1], t.vs[u][2 * i + 1] = vp[2], t.vz[u][2 * i + 1] = vp[3];
                    }
                }
            }
        };
        Where w = where(t0, pages_of(t0));
        uint32_t there = w.there, there_next = 0;
        load(0, w);
        if (t0 + ROUND < last) {
            w = where(t0 + ROUND, pages_of(t0 + ROUND));
            there_next = w.there;
            load(1, w);
        }
        Pages next = pages_of(t0 + 2 * ROUND);
        for (int slot = 0; t0 < last; t0 += ROUND, slot ^= 1) {
            T t;
            if (t0 + ROUND < last) wait_vmcnt<LOADS>();
            else wait_vmcnt<0>();
            fetch(t, slot);
            const uint32_t here = there;
            there = there_next;
            if (t0 + 2 * ROUND < last) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                w = where(t0 + 2 * ROUND, next);
                there_next = w.there;
                load(slot, w);
                next = pages_of(t0 + 3 * ROUND);
            }
            rows.use(t, t0, last, here, n, g, copy);
        }
    } else {
        for (; t0 < last; t0 += ROUND) {
            T t;
            const Where w = where(t0, pages_of(t0));
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint8_t *kb = half_of(a.K, u ? w.row1 : w.row0), *vb = half_of(a.V, u ? w.row1 : w.row0);
#pragma unroll
                for (int i = 0; i < D / 32; ++i) {
                    const u32x4 x = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(kb + (uint32_t)(n * T::ROW + 16 * g + 64 * i)));
#pragma unroll
                    for (int e = 0; e < 4; ++e) t.k[u][4 * i + e] = x[e];
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const uint8_t *p = vb + (uint32_t)((4 * g + r) * T::ROW + n * (D / 8));
                    if constexpr (D == 128) {
                        const u32x4 x = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p));
#pragma unroll
                        for (int e = 0; e < 4; ++e) t.v[u][r][e] = x[e];
                    } else {
                        const u32x2 x = __builtin_nontemporal_load(reinterpret_cast<const u32x2 *>(p));
                        t.v[u][r][0] = x[0], t.v[u][r][1] = x[1];
                    }
                }
            }
            rows.use(t, t0, last, w.there, n, g, copy);
        }
    }
}

template <int D> __device__ __forceinline__ void store_row(_Float16 *dst, f32x4 sum, float total)
{
    const float norm = total > 0.f ? 1.f / total : 0.f;
    union { _Float16 h[4]; u32x2 v; } y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y.h[e] = (_Float16)(sum[e] * norm);
    *reinterpret_cast<u32x2 *>(dst) = y.v;
}

template <int D, bool I4, int COPIES, int WAVES> __global__ __launch_bounds__(WAVES * 64, 2) void attn_decode_kernel(Decode a)
{
    constexpr int C = D / 16, ROUND = WAVES * kTile;     // (kRound where there are shares)
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // Neighbouring workgroups take different heads, so that an XCD, every eighth workgroup of a launch, gets as much as any.
    const int block = (int)(blockIdx.x / (uint32_t)a.per_seq), pair = (int)blockIdx.x - block * a.per_seq;
    const int h = pair / a.row_tiles, row0 = 16 * (pair - h * a.row_tiles);
    const int n_rows = min(16, a.group - row0), head0 = h * a.group + row0;
    int b = block, before = 0, from = 0, to = 0;         // sequence, rounds before it; the rounds of this share
    if (a.shares) {
        const int size = share_size(a, lane);
        from = block * size, to = from + size;
        b = sequence_at(a, from, lane, before);
        if (b == a.n_seqs) return;
    }
    for (;;) {
        const int len = length_of(a, b), rounds = (len + ROUND - 1) / ROUND;
        const int r0 = max(from - before, 0), r1 = a.shares ? min(to - before, rounds) : rounds;
        const bool whole = r0 == 0 && r1 == rounds;
        Rows<D, I4, COPIES> rows;
        rows.begin(a.q + (int64_t)b * a.ldq + (int64_t)(head0 + n % (16 / COPIES)) * D, n % (16 / COPIES) < n_rows, g, a.scale);
        walk<D, I4, COPIES, WAVES>(a, rows, b, h, r0 * ROUND, min(r1 * ROUND, len), smem + wave * (2 * Stage<D>::BYTES), wave, lane);
        __syncthreads();                                 // the stages' area is used again

        // the waves meet: acc[j][r] of lane (n, g) is column d = C (4 g + r) + j of query row n
        float(*s_top)[16] = reinterpret_cast<float(*)[16]>(smem), (*s_total)[16] = s_top + WAVES;
        float(*s_acc)[16][D + 4] = reinterpret_cast<float(*)[16][D + 4]>(s_total + WAVES);
        const float back = I4 ? __builtin_amdgcn_exp2f(rows.lift) : 1.f, total = sum_of_copies<COPIES>(sum_of_groups(rows.total)) * back,
                    zsum = sum_of_copies<COPIES>(sum_of_groups(rows.zsum));
        if (g == 0) s_top[wave][n] = rows.top, s_total[wave][n] = total;
        if constexpr (COPIES > 1) {
#pragma unroll
            for (int j = 0; j < C; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) rows.acc[j][r] = sum_of_copies<COPIES>(rows.acc[j][r]);
        }
        if (n < n_rows) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int j = 0; j < C; j += 4) {
                    f32x4 x;
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = I4 ? (rows.acc[j + e][r] * 1048576.f - zsum) * back : rows.acc[j + e][r];
                    *reinterpret_cast<f32x4 *>(&s_acc[wave][n][C * (4 * g + r) + j]) = x;
                }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < n_rows * (D / 4); i += WAVES * 64) {
            const int m = i / (D / 4), d = 4 * (i % (D / 4));
            float most = s_top[0][m];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) most = fmaxf(most, s_top[w][m]);
            const float base = most == kNone ? 0.f : most;
            f32x4 sum = 0.f;
            float all = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float e = __builtin_amdgcn_exp2f(s_top[w][m] - base);
                sum += e * *reinterpret_cast<const f32x4 *>(&s_acc[w][m][d]);
                all += e * s_total[w][m];
            }
            if (whole) {
                store_row<D>(a.o + (int64_t)b * a.ldo + (int64_t)(head0 + m) * D + d, sum, all);
            } else {
                const int64_t at = (((int64_t)pair * a.shares + block) * 2 + (r0 == 0)) * min(16, a.group) + m;
                *reinterpret_cast<f32x4 *>(a.part + at * D + d) = sum;
                if (d == 0) *reinterpret_cast<float2 *>(a.part_ml + at * 2) = make_float2(most, all);
            }
        }
        if (!a.shares) return;
        // on to the next sequence of the share that has tokens
        do before += rounds_of(a, b++);
        while (b < a.n_seqs && before < to && rounds_of(a, b) == 0);
        if (b >= a.n_seqs || before >= to) return;
        __syncthreads();
    }
}

// The pieces of query heads joined: D / 4 lanes take four columns each of every PARTS-th piece of a head, four pieces in flight;
// the parts of a head meet in LDS.  Sequences without tokens get their zeros here too.
template <int D, int PARTS> __global__ __launch_bounds__(256) void attn_join_kernel(Decode a, uint32_t n_rows)
{
    constexpr int TPR = D / 4, ROWS = 256 / (TPR * PARTS), DEEP = 4;
    const int lane = threadIdx.x % TPR, part = threadIdx.x / TPR % PARTS, mine = threadIdx.x / (TPR * PARTS), d = 4 * lane;
    const uint32_t row = min(blockIdx.x * ROWS + mine, n_rows - 1);          // sequence * heads + head
    const int b = (int)(row / a.heads), head = (int)(row - (uint32_t)b * a.heads);
    int pieces = 0, first = 0;                                               // of this row's sequence; the first one's share
    {
        // the rows of a workgroup may belong to several sequences: one after the other, by every wave
        const int size = share_size(a, threadIdx.x & 63);
        const int b_low = (int)(min(blockIdx.x * ROWS, n_rows - 1) / a.heads), b_high = (int)(min(blockIdx.x * ROWS + ROWS - 1, n_rows - 1) / a.heads);
        int before = rounds_before(a, b_low, threadIdx.x & 63);
        for (int s = b_low; s <= b_high; ++s) {
            const int rounds = rounds_of(a, s);
            if (s == b) {
                first = before / size;
                pieces = rounds ? (before + rounds - 1) / size - first + 1 : 0;
            }
            before += rounds;
        }
    }
    const int h = head / a.group, in_group = head - h * a.group, group_rows = min(16, a.group);
    const int64_t place = ((int64_t)(h * a.row_tiles + in_group / 16) * a.shares + first) * 2;
    auto at = [&](int i) { return (place + 2 * i + (i == 0)) * group_rows + in_group % 16; };
    const float2 *ml = reinterpret_cast<const float2 *>(a.part_ml);
    float most = kNone, all = 0.f;
    f32x4 sum = 0.f;
    for (int i0 = pieces > 1 ? part : pieces; i0 < pieces; i0 += PARTS * DEEP) {   // (a sequence in one piece is done)
        float2 x[DEEP];
        f32x4 y[DEEP];
#pragma unroll
        for (int k = 0; k < DEEP; ++k) {
            const int64_t p = at(min(i0 + PARTS * k, pieces - 1));
            x[k] = ml[p];
            y[k] = *reinterpret_cast<const f32x4 *>(a.part + p * D + d);
        }
        float now = most;
#pragma unroll
        for (int k = 0; k < DEEP; ++k) {
            x[k].x = i0 + PARTS * k < pieces ? x[k].x : kNone;
            now = fmaxf(now, x[k].x);
        }
        const float base = now == kNone ? 0.f : now, shrink = __builtin_amdgcn_exp2f(most - base);
        sum *= shrink;
        all *= shrink;
#pragma unroll
        for (int k = 0; k < DEEP; ++k) {
            const float e = __builtin_amdgcn_exp2f(x[k].x - base);
            sum += y[k] * e;
            all += x[k].y * e;
        }
        most = now;
    }
    if constexpr (PARTS > 1) {
        __shared__ float s_top[ROWS][PARTS], s_total[ROWS][PARTS];
        __shared__ f32x4 s_sum[ROWS][PARTS][TPR];
        if (lane == 0) s_top[mine][part] = most, s_total[mine][part] = all;
        s_sum[mine][part][lane] = sum;
        __syncthreads();
        if (part) return;
#pragma unroll
        for (int p = 1; p < PARTS; ++p) most = fmaxf(most, s_top[mine][p]);
        const float base = most == kNone ? 0.f : most;
        sum = 0.f, all = 0.f;
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            const float e = __builtin_amdgcn_exp2f(s_top[mine][p] - base);
            sum += s_sum[mine][p][lane] * e;
            all += s_total[mine][p] * e;
        }
    }
    if (pieces == 1 || blockIdx.x * ROWS + mine >= n_rows) return;
    store_row<D>(a.o + (int64_t)b * a.ldo + (int64_t)head * D + d, sum, all);
}

template <int D, bool I4, int COPIES, int WAVES> hipError_t launch_waves(const Decode &a, hipStream_t st)
{
    constexpr int meet = WAVES * 16 * (D + 4 + 2) * 4, stages = I4 ? WAVES * 2 * Stage<D>::BYTES : 0;
    constexpr int lds = meet > stages ? meet : stages;
    static_assert(lds <= 160 * 1024, "within what a workgroup may have");
    if constexpr (lds > 65536)
        if (hipError_t e = allow_dynamic_lds<attn_decode_kernel<D, I4, COPIES, WAVES>>(lds); e != hipSuccess) return e;
    const dim3 grid((unsigned)(a.shares ? a.shares : a.n_seqs) * (unsigned)a.per_seq);
    hipLaunchKernelGGL((attn_decode_kernel<D, I4, COPIES, WAVES>), grid, dim3(WAVES * 64), lds, st, a);
    return hipGetLastError();
}

// Eight waves where a workgroup has a unit to itself and a whole sequence to do (4 bits; us, 4 waves / 8: one sequence of 500 tokens 7.1
// / 7.0, of 1000 9.9 / 9.0, 16 of 2000 16.2 / 13.6, 32 of up to 2000 16.1 / 13.6; 64 of 500 11.3 / 11.9, 200 of up to 500 18.9 / 24.6.  Sixteen
// were slower than eight everywhere, and fp16 gained nothing, 32 of 1000, when that was measured on an earlier form of the kernel).
template <int D, bool I4, int COPIES> hipError_t launch_copies(const Decode &a, hipStream_t st)
{
    if constexpr (I4)
        if (!a.shares && (int64_t)a.n_seqs * a.per_seq <= compute_units() && a.max_len > 2 * kRound) return launch_waves<D, I4, COPIES, 8>(a, st);
    return launch_waves<D, I4, COPIES, 4>(a, st);
}

template <int D, bool I4> hipError_t launch_shares(const Decode &a, hipStream_t st)
{
    if constexpr (I4) {
        if (a.group <= 4) return launch_copies<D, I4, 4>(a, st);
        if (a.group <= 8) return launch_copies<D, I4, 2>(a, st);
    }
    return launch_copies<D, I4, 1>(a, st);
}

template <int D> hipError_t launch_join(const Decode &a, hipStream_t st)
{
    constexpr int groups = 256 / (D / 4);
    const uint32_t n_rows = (uint32_t)a.n_seqs * (uint32_t)a.heads;
    if (a.shares > 4 * a.n_seqs) hipLaunchKernelGGL((attn_join_kernel<D, groups>), dim3(n_rows), dim3(256), 0, st, a, n_rows);
    else hipLaunchKernelGGL((attn_join_kernel<D, 1>), dim3((n_rows + groups - 1) / groups), dim3(256), 0, st, a, n_rows);
    return hipGetLastError();
}

// Shares of the sequences of one key/value head and row tile; 0: a workgroup per sequence does it all, which needs no second
// kernel (4 us) and no change from one sequence to the next, but takes as long as the longest sequence: 0.7 us a round (4 bits; with
// eight waves 0.5 for as many tokens; fp16, which keeps one tile of a wave on its way, 1.4), or what the bytes take.  Measured (us,
// shares / a workgroup each; * where the rule takes the slower one):
//   4 bits, 8 key/value heads of 128:  1 sequence of 500 tokens 8.8 / 7.0, 896 8.9 / 8.3, 1000 9.1 / 9.0;  8 of 1000 10.8 / 9.4, 1300
//     14.1 / 10.6, up to 2000 10.7 / 13.0;  16 of 2000 14.5 / 13.6, up to 3000 15.8 / 16.9 *, 4000 19.1 / 20.6;  32 of up to 3000 21.6 / 17.5,
//     4000 24.9 / 21.2 *;  64 of up to 2000 27.0 / 19.5, 8192 55.0 / 65.3;  128 of up to 2000 37.8 / 32.7, 4096 62.2 / 64.1
//   fp16:  1 of 384 8.7 / 7.8;  8 of 500 10.4 / 11.2;  32 of 500 19.7 / 15.7, 1000 28.3 / 24.6 *;  64 of up to 1000 27.2 / 30.9
// The rule goes by counts, since lengths are not known here.  Where there are no shares for the number of sequences, one long
// sequence among many short ones is a workgroup's for each of its heads: 65000 tokens beside 254 sequences of up to 300 take 60 us, beside
// 255 of them, eight pairs to a unit, 359.
int shares_of(int64_t n_seqs, int64_t per_seq, int64_t max_len, bool i4)
{
    const int64_t units = compute_units(), rounds = (max_len + kRound - 1) / kRound, shares = 2 * units / per_seq;
    const int64_t pairs = n_seqs * per_seq;
    if (rounds <= (i4 ? (pairs > units ? 16 : pairs >= units / 2 ? 24 : pairs >= units / 4 ? 12 : 7) : pairs >= units / 2 ? 6 : 3)) return 0;
    // a wave adds up 64 lengths at a time, and rounds are counted in 32 bits
    if (shares < 2 || n_seqs > 1024 || pairs >= 8 * units || n_seqs * rounds >= 1 << 30) return 0;
    return (int)shares;
}

}  // namespace

size_t attn_decode_workspace_bytes(int64_t n_seqs, int64_t n_heads, int64_t kv, int64_t dim, int64_t max_len, bool i4)
{
    const int64_t group = n_heads / kv, per_seq = kv * ((group + 15) / 16);
    return (size_t)(per_seq * shares_of(n_seqs, per_seq, max_len, i4) * 2 * (group < 16 ? group : 16) * (dim + 2) * 4);
}

hipError_t launch_attn_decode(const void *Q, int64_t ldq, int64_t n_seqs, int64_t n_heads, const KvCache &c, const int32_t *table,
                              int64_t max_pages, int64_t ld_table, const int32_t *lens, float scale, void *O, int64_t ldo,
                              void *workspace, hipStream_t st)
{
    Decode a;
    a.q = static_cast<const _Float16 *>(Q), a.ldq = ldq;
    a.heads = (int)n_heads, a.kv = (int)c.heads, a.group = (int)(n_heads / c.heads), a.row_tiles = (a.group + 15) / 16;
    a.K = c.K, a.V = c.V, a.Kp = c.Kp, a.Vp = c.Vp;
    a.n_pages = (uint32_t)c.pages, a.page_shift = __builtin_ctzll((unsigned long long)c.page_size);
    a.table = table, a.ld_table = ld_table, a.max_len = max_pages * c.page_size, a.lens = lens;
    a.scale = scale * 1.4426950408889634f;
    a.n_seqs = (int)n_seqs, a.per_seq = a.kv * a.row_tiles, a.shares = shares_of(n_seqs, a.per_seq, a.max_len, c.i4);
    a.o = static_cast<_Float16 *>(O), a.ldo = ldo;
    a.part = static_cast<float *>(workspace);
    a.part_ml = a.part + (size_t)a.per_seq * a.shares * 2 * (a.group < 16 ? a.group : 16) * c.dim;
    const hipError_t e = c.dim == 128 ? (c.i4 ? launch_shares<128, true>(a, st) : launch_shares<128, false>(a, st))
                                      : (c.i4 ? launch_shares<64, true>(a, st) : launch_shares<64, false>(a, st));
    if (e != hipSuccess || !a.shares) return e;
    return c.dim == 128 ? launch_join<128>(a, st) : launch_join<64>(a, st);
}

}  // namespace sr

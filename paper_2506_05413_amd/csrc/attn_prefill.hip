// Attention of whole prompts: packed sequences of different lengths, grouped heads, causal or not.
//
//   o_i = sum_j softmax(scale q_i . k_j) v_j      over the keys j of row i's own sequence, j <= i + (keys - queries) if causal
//
// A row wave takes 32 query rows of a head, a workgroup's row waves heads that share a key/value head or further rows, and walks
// over their keys 64 (or 32) at a time with running sums; keys and values come into LDS by DMA, one tile ahead.  Both products run
// on 32 x 32 x 16 matrix instructions with the query row in the columns:
//
//   S^T = K Q^T   lane (m, g) = (lane % 32, lane / 32) gets the scores of row m and of tokens 8 i + 4 g + (0 .. 3)
//   O^T = V^T P^T its k-index is the token: the eight weights that a lane supplies per instruction are those of tokens
//                 4 g + (0 .. 3) and 8 + 4 g + (0 .. 3) of sixteen, which it got itself
//
// so weights stay in the lane that computed them, a row's sum is one lane's and its neighbour 32 further, and values are read
// from LDS with the transposing 8-byte read (four tokens of one column per lane).
//
// Weights are w = 2^(7 + log2(e) scale (q . k - top)), top a row's largest q . k when it was set, and it is set again only where a
// weight might pass 2^16: the sum of a tile's weights, which is needed anyhow, shows it, so that a tile needs no maximum, and most
// tiles rescale nothing.  The products of a tile are summed up from -top on, so that a difference is rounded as the score is,
// however large.  Weights are rounded to fp16 for the matrix pipe (half a step, 2^-11 of each; subnormal below 2^-21 of the
// largest at least), and the sum in the denominator is that of the rounded ones, so that equal values come out as they are.  (The
// rest of a weight would be another operand and a second product for every tile; the outputs' own rounding is as large: rms distance
// from 64 bits over normal values 2.3e-4 of them, and 2.0e-4 without it.)  Scores, sums and outputs are held in fp32.
//
// What bounds it: long prompts the power the chip may draw (8192 tokens, 32 heads of 128, causal: the clock is 1.83 GHz of 2.4 and
// the matrix pipe busy for half of the cycles), the others the chain of a row's tiles.  Per 64 keys and SIMD, two waves there, the
// products alone take 0.85 us, with the weights 1.05, with the reads from LDS 1.3; one wave takes 1.05.  Hence four shapes of
// workgroup (us; 32 and 8 heads of 128, causal, one prompt of T tokens; 8 and 8 heads; nine prompts of T tokens together):
//                                               T = 512   1024   2048   4096   8192  |  3000   4096   6000  |   400   1000
//   8 row waves  a tile loaded once for 256        17.7   31.2   58.4    139    518  |    70     95    134  |   7.6   10.9
//   4 row waves  two workgroups on a unit          13.4   23.9   48.0    147    535  |    52     70    108  |   6.4   10.0
//   2 x 2 sets   the sets take every other tile    11.1   23.3   64.3    202    752  |    37     55    114  |  11.7   18.5
//                and meet in LDS at the end
//   2 x 4 sets   tiles of 32 keys                  11.2   23.0   62.1    193    718  |    33     51    106  |  11.7   19.3
// Products interleaved with the weights of the tile before (three tiles in flight) were 9 % slower at 8192 tokens and 15 % at
// 1024, 64 rows per wave (one wave per SIMD) 30 % slower, and two halves of a workgroup that multiply and weigh in turn, by
// barriers, 6 .. 30 % slower.
#include <algorithm>

#include "gemm_common.h"

namespace sr {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
union Frag { f16x8 v; s16x4 s[2]; f16x2 p[4]; };

constexpr int kMatrix = 0x8, kRead = 0x100;              // groups of instructions for the scheduler: matrix products, reads from LDS
constexpr float kNone = -__builtin_inff();
// Workgroups of one row of the grid: a launch of 2^32 and more work items along one dimension is not refused, it wraps.
constexpr int kGridShift = 22;

struct Prefill {
    const _Float16 *q, *k, *v;
    int64_t ldq, ldk, ldv;
    const int32_t *cu_q, *cu_k;
    int n_seqs, tokens_q, tokens_k;
    int heads, kv, group;                                // group: query heads of one key/value head
    int head_shift, row_shift;                           // log2 of the heads and of the rows of one that a workgroup takes
    int tiles;                                           // of query rows, an upper bound
    int at_once;                                         // tiles whose workgroups fill half of the places
    int causal;
    float scale;                                         // times log2(e)
    _Float16 *o;
    int64_t ldo;
};

// where a sequence of a packed batch lies; ends that do not fit are cut, never followed
__device__ __forceinline__ void span(int from, int to, int tokens, int &begin, int &length)
{
    begin = min(max(from, 0), tokens);
    length = min(max(to, begin), tokens) - begin;
}

// a tile of query rows: its sequence's queries and keys, and its number among that sequence's tiles
struct Place { int q0, nq, k0, nk, local; };

__device__ __forceinline__ void take(Place &p, int lane_of, int q0, int nq, int k0, int nk)
{
    p.q0 = __builtin_amdgcn_readlane(q0, lane_of), p.nq = __builtin_amdgcn_readlane(nq, lane_of);
    p.k0 = __builtin_amdgcn_readlane(k0, lane_of), p.nk = __builtin_amdgcn_readlane(nk, lane_of);
}

// The tile-th tile of rows of the batch, those with the most keys first; false behind the last.  A lane looks at a sequence.
// (Nine prompts of 26 .. 541 tokens: 29.3 -> 25.7 us.)  Up to 64 sequences: tile i of a sequence that has `ahead` more keys than
// queries is on level i + 1 + ahead / (rows of a tile), and a level is found by bisection over the number of tiles above it.  Where every workgroup has its place at once (`at_once` tiles are
// half of the places), the second half of them is dealt out from the other end, so that a compute unit's two workgroups are a
// long and a short one (one prompt of 2048 tokens, 32 heads of 128: 48.6 -> 47.4 us).  More sequences: the last one's last first.
__device__ __forceinline__ bool find_tile(const Prefill &a, int tile, int lane, Place &p)
{
    auto tiles_in = [&](int rows) { return (int)(((uint32_t)rows + (1u << a.row_shift) - 1) >> a.row_shift); };
    if (a.n_seqs <= 64) {
        const int s = min(lane, a.n_seqs - 1);
        const int q_from = a.cu_q[s], q_to = a.cu_q[s + 1], k_from = a.cu_k[s], k_to = a.cu_k[s + 1];
        int q0, nq, k0, nk;
        span(q_from, q_to, a.tokens_q, q0, nq);
        span(k_from, k_to, a.tokens_k, k0, nk);
        const int n = lane < a.n_seqs ? tiles_in(nq) : 0;
        const int ahead = max(nk - nq, 0) >> a.row_shift;
        auto above = [&](int level) { return __builtin_amdgcn_readlane(scan_of_wave(min(max(ahead + n - level, 0), n)), 63); };
        const int all = above(0);
        if (tile >= all) return false;
        if (all <= 2 * a.at_once && tile >= a.at_once) tile = all - 1 - (tile - a.at_once);
        int low = 0, high = ((a.tokens_k > a.tokens_q ? a.tokens_k : a.tokens_q) >> a.row_shift) + 1;   // above(low) > tile >= above(high)
        while (high - low > 1) {
            const int mid = low + (high - low) / 2;
            if (above(mid) > tile) low = mid;
            else high = mid;
        }
        // the tile is on level `high`
        const int rank = tile - above(high);
        const bool here = high > ahead && high <= ahead + n;
        const unsigned long long mask = __ballot(here);
        const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
        const int at = __builtin_ctzll(__ballot(here && before == rank));
        take(p, at, q0, nq, k0, nk);
        p.local = high - 1 - __builtin_amdgcn_readlane(ahead, at);
        return true;
    }
    tile = a.tiles - 1 - tile;
    if (tile < 0) return false;                          // (a workgroup that only rounds the grid up)
    for (int s0 = 0; s0 < a.n_seqs; s0 += 64) {
        const int s = min(s0 + lane, a.n_seqs - 1);
        const int q_from = a.cu_q[s], q_to = a.cu_q[s + 1], k_from = a.cu_k[s], k_to = a.cu_k[s + 1];
        int q0, nq, k0, nk;
        span(q_from, q_to, a.tokens_q, q0, nq);
        span(k_from, k_to, a.tokens_k, k0, nk);
        const int n = s0 + lane < a.n_seqs ? tiles_in(nq) : 0;
        const int upto = scan_of_wave(n);
        const unsigned long long past = __ballot(upto > tile);
        if (past) {
            const int at = __builtin_ctzll(past);
            take(p, at, q0, nq, k0, nk);
            p.local = tile - __builtin_amdgcn_readlane(upto - n, at);
            return true;
        }
        tile -= __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

// SETS sets of waves, each with every SETS-th tile of KEYS keys
template <int D, int W, int SETS, int KEYS> __global__ __launch_bounds__(64 * W * SETS, D == 64 && SETS == 4 ? 4 : 2) void attn_prefill_kernel(Prefill a)
{
    constexpr int CH = D / 8;                            // 16-byte chunks of a row
    constexpr uint32_t kTileBytes = KEYS * D * 2;
    constexpr int DT = D / 32, LOADS = KEYS * CH / (64 * W);    // column tiles; DMA loads of a wave per operand
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];   // per set: [2][keys, values]
    const int lane = threadIdx.x & 63, m = lane & 31, g = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane((threadIdx.x >> 6) % W), set = __builtin_amdgcn_readfirstlane((threadIdx.x >> 6) / W);
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)smem + set * 4 * kTileBytes;
    const uint8_t *tiles = smem + set * 4 * kTileBytes;
    // neighbouring workgroups take different key/value heads: an XCD, every eighth of them, keeps few heads' keys in its L2
    const uint32_t blocks = (uint32_t)a.heads >> a.head_shift, number = (blockIdx.y << kGridShift) + blockIdx.x, x = number % blocks;
    const int kvh = (int)(x % (uint32_t)a.kv);
    const int head = kvh * a.group + ((int)(x / (uint32_t)a.kv) << a.head_shift) + (wave & ((1 << a.head_shift) - 1));
    Place p;
    if (!find_tile(a, (int)(number / blocks), lane, p)) return;
    const int rows = 1 << a.row_shift, r0 = p.local << a.row_shift, shift = p.nk - p.nq;
    const int end = a.causal ? min(p.nk, min(r0 + rows, p.nq) + shift) : p.nk;         // keys that any row sees
    const int w0 = r0 + 32 * (wave >> a.head_shift), row = w0 + m;
    const int wend = w0 >= p.nq ? 0 : a.causal ? min(p.nk, min(w0 + 32, p.nq) + shift) : p.nk;   // .. of this wave
    const int rend = a.causal ? min(p.nk, row + shift + 1) : p.nk;                     // .. of this lane's row
    const int whole = a.causal ? min(p.nk, w0 + shift + 1) : p.nk;                     // keys that every row of the wave sees

    // Tiles lie in LDS by rows, their chunks swapped so that the lanes that read at once meet every bank: keys, read 32 rows
    // of one chunk at a time, by row; values, read 4 rows of four neighbouring chunks, by row in steps of four chunks.
    const uint8_t *kb = reinterpret_cast<const uint8_t *>(a.k + (int64_t)p.k0 * a.ldk + (int64_t)kvh * D);
    const uint8_t *vb = reinterpret_cast<const uint8_t *>(a.v + (int64_t)p.k0 * a.ldv + (int64_t)kvh * D);
    auto key_swap = [](int r) { return D == 128 ? r & 15 : (r >> 1) & 7; };
    auto value_swap = [](int r) { return D == 128 ? (r & 3) << 2 : ((r >> 1) & 1) << 2; };
    uint32_t k_off[LOADS], v_off[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int at = (i * W + wave) * 64 + lane, r = at / CH, c = at % CH;
        k_off[i] = r * (uint32_t)(a.ldk * 2) + 16 * (c ^ key_swap(r));
        v_off[i] = r * (uint32_t)(a.ldv * 2) + 16 * (c ^ value_swap(r));
    }
    auto load = [&](int t0, int slot) {
        const uint8_t *kt = kb + (int64_t)t0 * a.ldk * 2, *vt = vb + (int64_t)t0 * a.ldv * 2;
        const uint32_t to = lds + slot * 2 * kTileBytes + wave * 1024;
        if (t0 + KEYS <= p.nk) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                dma16(kt, k_off[i], to + W * 1024 * i);
                dma16(vt, v_off[i], to + W * 1024 * i + kTileBytes);
            }
        } else {                                         // rows past the end: the last one again
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int r = ((i * W + wave) * 64 + lane) / CH;
                const uint32_t over = (uint32_t)max(r - (p.nk - 1 - t0), 0);
                dma16(kt, k_off[i] - over * (uint32_t)(a.ldk * 2), to + W * 1024 * i);
                dma16(vt, v_off[i] - over * (uint32_t)(a.ldv * 2), to + W * 1024 * i + kTileBytes);
            }
        }
    };
    const int n_tiles = end > 0 ? (end + KEYS - 1) / KEYS : 0, mine = wend > 0 ? (wend + KEYS - 1) / KEYS : 0;
    const int rounds = (n_tiles + SETS - 1) / SETS;
    // A wave's query rows come the same way, whole rows at a time, through the stage of the second tile (and past it: 8 row waves).
    // Taken from memory in the order of the operand, every line of a row would be asked for four times.
    constexpr int Q_LOADS = CH / 2;
    constexpr uint32_t kQueries = 2 * kTileBytes;
    {
        const int b0 = min(w0, p.nq - 1);
        const uint8_t *from = reinterpret_cast<const uint8_t *>(a.q + (int64_t)(p.q0 + b0) * a.ldq + (int64_t)head * D);
#pragma unroll
        for (int i = 0; i < Q_LOADS; ++i) {
            const int at = i * 64 + lane, r = at / CH, c = at % CH;
            dma16(from, (uint32_t)min(r, p.nq - 1 - b0) * (uint32_t)(a.ldq * 2) + 16 * (c ^ key_swap(r)), lds + kQueries + wave * (32 * D * 2) + 1024 * i);
        }
    }
    Frag q[D / 16];
    if (set < n_tiles) {
        load(set * KEYS, 0);
        wait_vmcnt<2 * LOADS>();
    } else {
        wait_vmcnt<0>();
    }
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
        q[i].v = *reinterpret_cast<const f16x8 *>(tiles + kQueries + wave * (32 * D * 2) + m * (D * 2) + 16 * ((2 * i + g) ^ key_swap(m)));
    // have them here: a wait for them inside the loop below would be one for everything that is in flight there
#pragma unroll
    for (int i = 0; i < D / 16; ++i) asm volatile("" : "+v"(q[i].v));
    f32x16 acc[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) acc[t] = 0.f;
    f32x16 below = 0.f;                                  // minus the score that weights are relative to
    float top = kNone, limit = -1.f, total = 0.f;

    // what was asked for a round ago is there, and everybody is done with the slot that is asked for now
    auto turn = [&](int round) {
        wait_vmcnt<0>();
        barrier_nofence();
        const int next = (round + 1) * SETS + set;
        if (next < n_tiles) load(next * KEYS, (round + 1) & 1);
    };
    int round = 0;
    for (; round * SETS + set < mine; ++round) {
        turn(round);
        const int t0 = (round * SETS + set) * KEYS;
        const uint8_t *ks = tiles + (round & 1) * 2 * kTileBytes, *vs = ks + kTileBytes;
        auto value = [&](int step, int t) {
            Frag v;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int r = 16 * step + 8 * half + 4 * g + ((lane >> 2) & 3);
                const int c = 4 * t + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
                const uint8_t *from = vs + r * (D * 2) + 16 * (c ^ value_swap(r)) + 8 * (lane & 1);
                v.s[half] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)from);
            }
            return v;
        };
        f32x16 s[KEYS / 32];
#pragma unroll
        for (int u = 0; u < KEYS / 32; ++u) {
            s[u] = below;
            const int r = 32 * u + m;
#pragma unroll
            for (int d = 0; d < D / 16; ++d) {
                Frag k;
                k.v = *reinterpret_cast<const f16x8 *>(ks + r * (D * 2) + 16 * ((2 * d + g) ^ key_swap(r)));
                s[u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k.v, q[d].v, s[u], 0, 0, 0);
            }
        }
        // reads of keys ahead of the products, one more with each
        constexpr int SCORES = KEYS / 32 * (D / 16), AHEAD = SCORES > 8 ? 6 : SCORES / 2;
        __builtin_amdgcn_sched_group_barrier(kRead, AHEAD, 0);
#pragma unroll
        for (int i = 0; i < SCORES - AHEAD; ++i) {
            __builtin_amdgcn_sched_group_barrier(kMatrix, 1, 0);
            __builtin_amdgcn_sched_group_barrier(kRead, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(kMatrix, AHEAD, 0);
        if (t0 + KEYS > whole) {
#pragma unroll
            for (int u = 0; u < KEYS / 32; ++u)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (t0 + 32 * u + 8 * (e / 4) + 4 * g + (e & 3) >= rend) s[u][e] = kNone;
        }
        Frag w[KEYS / 16];                               // of 16 tokens each
        float sum;
        auto weigh = [&] {
            sum = 0.f;
#pragma unroll
            for (int u = 0; u < KEYS / 32; ++u)
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    f16x2 &pair = w[2 * u + e / 8].p[e / 2 % 4];
                    pair = f16x2{(_Float16)__builtin_amdgcn_exp2f(fmaf(s[u][e], a.scale, 7.f)), (_Float16)__builtin_amdgcn_exp2f(fmaf(s[u][e + 1], a.scale, 7.f))};
                    sum = __builtin_amdgcn_fdot2(pair, f16x2{(_Float16)1.f, (_Float16)1.f}, sum, false);
                }
        };
        weigh();
        if (!__all(sum <= limit)) {                      // (a weight beyond fp16 is infinite, and so is the sum)
            float most = kNone;
#pragma unroll
            for (int u = 0; u < KEYS / 32; ++u)
#pragma unroll
                for (int e = 0; e < 16; ++e) most = fmaxf(most, s[u][e]);
            most = fmaxf(most, __shfl_xor(most, 32, 64));
            const float up = top == kNone ? most : fmaxf(most, 0.f);
            if (up != kNone) {
                const float shrink = top == kNone ? 1.f : __builtin_amdgcn_exp2f(-up * a.scale);
                total *= shrink;
#pragma unroll
                for (int t = 0; t < DT; ++t) acc[t] *= shrink;
#pragma unroll
                for (int u = 0; u < KEYS / 32; ++u) s[u] -= up;
                below -= up, top = -below[0], limit = 32768.f;
            }
            weigh();
        }
        total += sum;
#pragma unroll
        for (int step = 0; step < KEYS / 16; ++step)
#pragma unroll
            for (int t = 0; t < DT; ++t) acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(value(step, t).v, w[step].v, acc[t], 0, 0, 0);
        // the reads of some products ahead, two more with each
        constexpr int VALUES = KEYS / 16 * DT, BEFORE = VALUES > 4 ? 4 : 2;
        __builtin_amdgcn_sched_group_barrier(kRead, 2 * BEFORE, 1);
#pragma unroll
        for (int i = 0; i < VALUES - BEFORE; ++i) {
            __builtin_amdgcn_sched_group_barrier(kMatrix, 1, 1);
            __builtin_amdgcn_sched_group_barrier(kRead, 2, 1);
        }
        __builtin_amdgcn_sched_group_barrier(kMatrix, BEFORE, 1);
    }
    for (; round < rounds; ++round) turn(round);         // tiles that only other waves need

    // Outputs leave as they came, whole rows at a time: a lane has four columns of a row (part i: those from 8 i + 4 g on) and
    // stores eight of another one.
    constexpr int PARTS = D / 8;
    auto part = [&](int i) { return f32x4{acc[i / 4][4 * (i % 4)], acc[i / 4][4 * (i % 4) + 1], acc[i / 4][4 * (i % 4) + 2], acc[i / 4][4 * (i % 4) + 3]}; };
    auto store = [&](int r, int c, f16x8 y) {
        if (w0 + r < p.nq) *reinterpret_cast<f16x8 *>(a.o + (int64_t)(p.q0 + w0 + r) * a.ldo + (int64_t)head * D + 8 * c) = y;
    };
    barrier_nofence();
    if constexpr (SETS == 1) {
        total += __shfl_xor(total, 32, 64);
        const float norm = total > 0.f ? 1.f / total : 0.f;
        // chunks swapped by row, their halves by rows 16 and up
        uint8_t *area = smem + wave * (32 * D * 2);
#pragma unroll
        for (int i = 0; i < PARTS; ++i) {
            union { _Float16 h[4]; uint2 u; } y;
            const f32x4 x = part(i) * norm;
#pragma unroll
            for (int e = 0; e < 4; ++e) y.h[e] = (_Float16)x[e];
            *reinterpret_cast<uint2 *>(area + m * (D * 2) + 16 * (i ^ (m & (CH - 1))) + 8 * (g ^ (m >> 4))) = y.u;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int j = 0; j < CH / 2; ++j) {
            const int r = (j * 64 + lane) / CH, c = lane % CH;
            f16x8 y = *reinterpret_cast<const f16x8 *>(area + r * (D * 2) + 16 * (c ^ (r & (CH - 1))));
            if (j >= CH / 4) y = __builtin_shufflevector(y, y, 4, 5, 6, 7, 0, 1, 2, 3);
            store(r, c, y);
        }
    } else {
        // the sets lay down what they have (part i of a lane beside those of others, in an order of its own), and each joins its
        // share of the rows
        f32x4 *area = reinterpret_cast<f32x4 *>(smem) + wave * (PARTS * 64);
        float2 *state = reinterpret_cast<float2 *>(smem + SETS * W * (PARTS * 1024)) + wave * 64;
#pragma unroll
        for (int i = 0; i < PARTS; ++i) area[(set * W * PARTS + i) * 64 + (lane ^ i)] = part(i);
        state[set * W * 64 + lane] = make_float2(top, total);
        __syncthreads();
#pragma unroll
        for (int j = 0; j < CH / 2 / SETS; ++j) {
            const int r = ((set * (CH / 2 / SETS) + j) * 64 + lane) / CH, c = lane % CH;
            float both = kNone, all = 0.f;
            f32x4 lo = 0.f, hi = 0.f;
#pragma unroll
            for (int n = 0; n < SETS; ++n) both = fmaxf(both, state[n * W * 64 + r].x);
#pragma unroll
            for (int n = 0; n < SETS; ++n) {
                const float2 one = state[n * W * 64 + r];
                const float by = one.x == kNone ? 0.f : __builtin_amdgcn_exp2f((one.x - both) * a.scale);
                all += (one.y + state[n * W * 64 + r + 32].y) * by;
                lo += area[(n * W * PARTS + c) * 64 + (r ^ c)] * by;
                hi += area[(n * W * PARTS + c) * 64 + ((r + 32) ^ c)] * by;
            }
            const float norm = all > 0.f ? 1.f / all : 0.f;
            f16x8 y;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = (_Float16)(lo[e] * norm), y[4 + e] = (_Float16)(hi[e] * norm);
            store(r, c, y);
        }
    }
}

// tiles of rows, at most: every sequence may end inside one
int64_t tiles_of(int64_t T_q, int64_t n_seqs, int64_t rows) { return T_q / rows + (n_seqs < T_q ? n_seqs : T_q); }

// Heads of a key/value head for the row waves of a workgroup: as many as come out even, so that a tile has few rows of each
// (nine prompts of 2500 tokens, 32 and 8 heads 26.0 -> 22.5 us, sixty 27.5 -> 17.3; one prompt the same).
int group_even(int group, int waves)
{
    int heads = 1;
    while (2 * heads <= waves && group % (2 * heads) == 0) heads *= 2;
    return heads;
}

template <int D, int W, int SETS, int KEYS> hipError_t launch_dim(Prefill a, int64_t n_seqs, bool balance, hipStream_t st)
{
    constexpr int tiles = SETS * 4 * KEYS * D * 2, queries = 2 * KEYS * D * 2 + W * 32 * D * 2;
    constexpr int join = SETS == 1 ? 0 : SETS * W * (D / 8 * 1024 + 512), most = tiles > join ? tiles : join, bytes = most > queries ? most : queries;
    if (hipError_t e = allow_dynamic_lds<attn_prefill_kernel<D, W, SETS, KEYS>>(bytes); e != hipSuccess) return e;
    a.head_shift = __builtin_ctz(group_even(a.group, W));
    a.row_shift = __builtin_ctz(32 * W) - a.head_shift;
    const int64_t blocks = a.heads >> a.head_shift;
    a.tiles = (int)tiles_of(a.tokens_q, n_seqs, 1 << a.row_shift);
    a.at_once = balance ? (int)((compute_units() + blocks - 1) / blocks) : 0;
    static_assert((64ll * W * SETS << kGridShift) < 1ll << 32, "a row of the grid");
    const int64_t all = a.tiles * blocks, row = std::min(all, (int64_t)1 << kGridShift);
    hipLaunchKernelGGL((attn_prefill_kernel<D, W, SETS, KEYS>), dim3((unsigned)row, (unsigned)((all + row - 1) / row)), dim3(64 * W * SETS), bytes, st, a);
    return hipGetLastError();
}

}  // namespace

int64_t attn_prefill_workgroups(int64_t T_q, int64_t n_seqs, int64_t n_heads) { return tiles_of(T_q, n_seqs, 64) * n_heads; }

hipError_t launch_attn_prefill(const void *Q, int64_t ldq, const void *K, int64_t ldk, const void *V, int64_t ldv,
                               const int32_t *cu_q, const int32_t *cu_k, int64_t n_seqs, int64_t T_q, int64_t T_k, int64_t n_heads,
                               int64_t kv, int64_t dim, bool causal, float scale, void *O, int64_t ldo, hipStream_t st)
{
    Prefill a;
    a.q = static_cast<const _Float16 *>(Q), a.k = static_cast<const _Float16 *>(K), a.v = static_cast<const _Float16 *>(V);
    a.ldq = ldq, a.ldk = ldk, a.ldv = ldv;
    a.cu_q = cu_q, a.cu_k = cu_k;
    a.n_seqs = (int)n_seqs, a.tokens_q = (int)T_q, a.tokens_k = (int)T_k;
    a.heads = (int)n_heads, a.kv = (int)kv, a.group = (int)(n_heads / kv);
    a.causal = causal, a.scale = scale * 1.4426950408889634f;
    a.o = static_cast<_Float16 *>(O), a.ldo = ldo;
    // Sets of waves over the keys while the workgroups of two row waves (load: how many there are for a place) are few for how
    // long a row's keys are, four sets for long ones (heads of 64, which have two workgroups on a unit: where not even all
    // places are taken).  Heads of 64 gain nothing from 256 rows a workgroup (4096 tokens, 32 heads 84 us for 85).
    const int64_t units = compute_units();
    const double rows = (double)T_q * n_heads, keys = (double)T_k / n_seqs;
    const int share = group_even(a.group, 2);            // heads of such a workgroup
    const double load = ((double)T_q + (n_seqs - 1.0) * (32 / share)) * n_heads / (64.0 * units * (128 / dim));
    if (keys > 64 && load <= std::min(0.75 + keys / 700, 2.25)) {
        if (keys >= 1024 && (dim == 128 || load <= 0.75)) return dim == 128 ? launch_dim<128, 2, 4, 32>(a, n_seqs, false, st) : launch_dim<64, 2, 4, 32>(a, n_seqs, false, st);
        return dim == 128 ? launch_dim<128, 2, 2, 64>(a, n_seqs, false, st) : launch_dim<64, 2, 2, 64>(a, n_seqs, false, st);
    }
    if (dim == 128 && rows >= 512.0 * units && T_q >= 2048 * n_seqs) return launch_dim<128, 8, 1, 64>(a, n_seqs, false, st);
    return dim == 128 ? launch_dim<128, 4, 1, 64>(a, n_seqs, true, st) : launch_dim<64, 4, 1, 64>(a, n_seqs, true, st);
}

}  // namespace sr

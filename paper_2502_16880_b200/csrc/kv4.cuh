// A paged cache of keys and values held in 4 bits, and attention of few queries over it.
//
// A group of 32, 64 or 128 columns of a token's head is held as codes 0..15 of a step and a lowest value (both of the element type):
//   low = min x, step = round((max x - min x) / 15), code = round((x - low) / step) in 0..15, x ~ low + step code.
// With x split that way the score of a token needs whole numbers as operands only:
//   q . k = sum over groups of step_g (sum of q code) + low_g (sum of q)
// and so does the output, with p the weights of the softmax:
//   out = sum over tokens of (p step_g) code + sum of p low_g.
// Codes go to the warp MMA as fp16 subnormals (two operations a pair, no arithmetic); what is rounded is p step_g, to fp16, as p
// would be for 16-bit values.
//
// Layout: tokens in blocks of 16, [page][head][block of 16]: keys, values, (step, low) pairs of keys [group][16], of values.
//   keys:   [16][4 lanes] of D / 8 bytes: column c is nibble c % 8 of word c / 32 of lane (c / 8) % 4
//   values: [2][8 columns][4 pairs of tokens][2] of D / 16 bytes: column c is nibble c / 8 of column place c % 8
// so that a lane's MMA operands are one 16-byte (D = 64: 8-byte) shared-memory load each, without bank conflicts, and no two tokens
// share a byte.
#pragma once
#include <type_traits>

#include "mbarrier.cuh"
#include "q4_prims.cuh"

namespace coral {

constexpr int kKv4Block = 16;                       // tokens of a block

struct Kv4Cache {
    unsigned char* base;
    int slots;                                      // pages * page
    int n_k, page, groups;
    __host__ __device__ int block_bytes(int D) const { return kKv4Block * D + 128 * groups; }
    // start of the block that holds slot `slot` of head `head`
    __device__ __forceinline__ unsigned char* block(int slot, int head, int D) const {
        const int subs = page / kKv4Block, sub = slot / kKv4Block, page_at = sub / subs;
        return base + (((long long)page_at * n_k + head) * subs + (sub - page_at * subs)) * block_bytes(D);
    }
};

template <typename T> __device__ __forceinline__ uint32_t kv4_bits(float v);
template <> __device__ __forceinline__ uint32_t kv4_bits<__nv_bfloat16>(float v) { return __bfloat16_as_ushort(__float2bfloat16_rn(v)); }
template <> __device__ __forceinline__ uint32_t kv4_bits<__half>(float v) { return __half_as_ushort(__float2half_rn(v)); }
// step and low of a pair
template <typename T> __device__ __forceinline__ float2 kv4_pair(uint32_t w);
template <> __device__ __forceinline__ float2 kv4_pair<__nv_bfloat16>(uint32_t w) { return make_float2(bf16_lo(w), bf16_hi(w)); }
template <> __device__ __forceinline__ float2 kv4_pair<__half>(uint32_t w) { return __half22float2(*reinterpret_cast<__half2*>(&w)); }

// ---- tokens into the cache and out of it ---------------------------------------------------------------------
constexpr int kKv4RowThreads = 256;
struct Kv4Rows {
    const int64_t* slots;
    int rows;                                       // tokens * heads
    void *k, *v;                                    // inputs of a store, outputs of a load
    long long ld_k, ld_v;
};

// D / 8 threads a row of a head, eight columns each.  grid: (rows, keys and values).
template <typename T, int D>
__global__ void __launch_bounds__(kKv4RowThreads) kv4_store_kernel(Kv4Cache c, Kv4Rows a) {
    constexpr int L = D / 8;
    pdl_wait();
    const int row = (int)(blockIdx.x * (kKv4RowThreads / L) + threadIdx.x / L);
    const int lane = threadIdx.x & 31, l = lane & (L - 1);
    const bool is_v = blockIdx.y != 0;
    const int token = row / c.n_k, head = row - token * c.n_k;
    const int64_t at = row < a.rows ? a.slots[token] : -1;
    const bool on = at >= 0 && at < c.slots;
    const int slot = (int)at;
    float x[8] = {};
    if (on) Elem<T>::load8(static_cast<const T*>(is_v ? a.v : a.k) + token * (is_v ? a.ld_v : a.ld_k) + head * D + 8 * l, x);
    float low = x[0], high = x[0], bad = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        low = fminf(low, x[i]);
        high = fmaxf(high, x[i]);
        bad += x[i] * 0.f;                          // NaN for an infinity or a NaN
    }
    const int per = L / c.groups;                   // threads of a group
    for (int o = 1; o < per; o <<= 1) {
        low = fminf(low, __shfl_xor_sync(0xffffffffu, low, o));
        high = fmaxf(high, __shfl_xor_sync(0xffffffffu, high, o));
        bad += __shfl_xor_sync(0xffffffffu, bad, o);
    }
    const uint32_t step_bits = kv4_bits<T>((high - low) / 15.f + bad);
    const float step = kv4_pair<T>(step_bits).x;
    uint32_t word = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float n = step > 0.f ? fminf(fmaxf(rintf((x[i] - low) / step), 0.f), 15.f) : 0.f;
        word |= (uint32_t)n << (4 * i);
    }
    if (is_v) {                                     // from eight columns a thread to one column place a thread
        uint32_t turned = 0;
        const int first = lane & ~(L - 1), n = l & 7, half = l & 8;
#pragma unroll
        for (int j = 0; j < 8; ++j) turned |= (__shfl_sync(0xffffffffu, word, first + half + j) >> (4 * n) & 15u) << (4 * j);
        word = turned;
    }
    if (!on) return;
    unsigned char* blk = c.block(slot, head, D);
    const int t = (int)(slot & 15);
    if (!is_v) {
        *reinterpret_cast<uint32_t*>(blk + (t * 4 + (l & 3)) * (D / 8) + 4 * (l >> 2)) = word;
    } else {
        const int n = l & 7;
        *reinterpret_cast<uint32_t*>(blk + 8 * D + (t >> 3) * (4 * D) + ((n * 4 + ((t & 7) >> 1)) * 2 + (t & 1)) * (D / 16) + 4 * (l >> 3)) = word;
    }
    if (l % per == 0)
        reinterpret_cast<uint32_t*>(blk + 16 * D)[((is_v ? c.groups : 0) + l / per) * 16 + t] = step_bits | kv4_bits<T>(low + bad) << 16;
}

template <typename T, int D>
__global__ void __launch_bounds__(kKv4RowThreads) kv4_load_kernel(Kv4Cache c, Kv4Rows a) {
    constexpr int L = D / 8;
    pdl_wait();
    if (!(blockIdx.y ? a.v : a.k)) return;
    const int row = (int)(blockIdx.x * (kKv4RowThreads / L) + threadIdx.x / L);
    const int lane = threadIdx.x & 31, l = lane & (L - 1);
    const bool is_v = blockIdx.y != 0;
    const int token = row / c.n_k, head = row - token * c.n_k;
    const int64_t at = row < a.rows ? a.slots[token] : -1;
    const bool on = at >= 0 && at < c.slots;
    const int slot = (int)at;
    uint32_t word = 0, pair = 0;
    if (on) {
        const unsigned char* blk = c.block(slot, head, D);
        const int t = (int)(slot & 15), n = l & 7;
        word = *reinterpret_cast<const uint32_t*>(
            !is_v ? blk + (t * 4 + (l & 3)) * (D / 8) + 4 * (l >> 2)
                  : blk + 8 * D + (t >> 3) * (4 * D) + ((n * 4 + ((t & 7) >> 1)) * 2 + (t & 1)) * (D / 16) + 4 * (l >> 3));
        pair = reinterpret_cast<const uint32_t*>(blk + 16 * D)[((is_v ? c.groups : 0) + l / (L / c.groups)) * 16 + t];
    }
    if (is_v) {
        uint32_t turned = 0;
        const int first = lane & ~(L - 1), i = l & 7, half = l & 8;
#pragma unroll
        for (int n = 0; n < 8; ++n) turned |= (__shfl_sync(0xffffffffu, word, first + half + n) >> (4 * i) & 15u) << (4 * n);
        word = turned;
    }
    if (row >= a.rows) return;
    const float2 s = kv4_pair<T>(pair);
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = fmaf((float)(word >> (4 * j) & 15u), s.x, s.y);
    T* to = static_cast<T*>(is_v ? a.v : a.k) + token * (is_v ? a.ld_v : a.ld_k) + head * D + 8 * l;
    Elem<T>::store8(to, x);
}

// ---- attention -----------------------------------------------------------------------------------------------
// A block takes up to 8 NR row_groups rows (query tokens of a sequence times the query heads of one key head) and a span of the
// sequence's cache.  Its producer warp brings stages of eight blocks of 16 tokens into a ring, one bulk copy a block (whatever
// the page size); eight warps, in row groups that share the tokens of a stage, take a block of 16 tokens each:
//   scores  [16 tokens x 8 rows] = K (operand A, unpacked) Q^T,   out [D x 8 rows] += V^T (operand A, unpacked) P^T
// with tokens and columns on the MMA's long side, so one sequence's few rows cost no more than 8 and an unpacked operand serves
// NR MMAs.  The running maximum is a reference, moved only when a score passes it by 2^8, so that most blocks need a vote and no
// shuffles.  Long caches are split over blocks, and kv4_join_kernel adds the parts up.
constexpr int kKv4Warps = 8;
constexpr int kKv4Threads = (kKv4Warps + 1) * 32;
constexpr int kKv4Stages = 4;
constexpr int kKv4StageTokens = 8 * kKv4Block;
constexpr int kKv4MaxTree = 64;                     // query tokens under a tree mask

struct Kv4Args {
    Kv4Cache c;
    int n_seq, n_rows, max_q, n_q, G, width, n_pages;
    int row_groups, row_blocks, splits;
    float scale2;                                   // scale log2(e)
    long long ld_table, ld_q, ld_out;
    const void* q;
    const int32_t *table, *lens;
    const int64_t* q_offsets;                       // null: max_q rows a sequence
    const unsigned long long* tree;
    void* out;
    float* lse;
    float* part_o;                                  // [split][row][head][D], unnormalised
    float2* part_ml;                                // [split][row][head] reference maximum (log2) and sum
    DeviceState* st;
};

// First row and number of rows of a sequence; no more than max_q of them are worked on.
__device__ __forceinline__ void kv4_rows_of(const Kv4Args& a, int seq, int* first, int* n) {
    if (a.q_offsets) {
        clamped_range(a.q_offsets, seq, a.n_rows, first, n);
    } else {
        *first = seq * a.max_q;
        *n = a.max_q;
    }
}

__device__ __forceinline__ float exp2_fast(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ uint32_t half_pair(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// The transpose of an 8 x 8 tile of 16-bit values, a row's pair a thread.
__device__ __forceinline__ uint32_t tile_transpose(uint32_t v) {
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}

template <typename T, int D, int NG, int NR>
__global__ void __launch_bounds__(kKv4Threads, NR == 1 ? 2 : 1) kv4_attention_kernel(const Kv4Args a) {
    constexpr int kBytes = kKv4Block * D + 128 * NG;          // of a block of 16 tokens
    constexpr int kStage = 8 * kBytes;
    constexpr int W = D / 32, J = D / 16;                     // words of a lane and token; tiles of 16 columns
    // fp16 outputs: what the rounding of p step loses is made good at the middle of the codes, so that it weighs code - 7.5 and not
    // code (0.0005 -> 0.0003 of the output; bf16 outputs, rounded to 0.0017, do not show it)
    constexpr bool kCentre = std::is_same_v<T, __half>;
    static_assert(kKv4Warps * 8 * NR * D * 4 <= kKv4Stages * kStage, "the warps' outputs fit the ring");
    extern __shared__ __align__(128) unsigned char kv4_smem[];
    __shared__ __align__(8) uint64_t full[kKv4Stages], empty[kKv4Stages];
    __shared__ uint32_t present[kKv4Stages];                  // which blocks of a stage there are
    __shared__ float2 s_ml[kKv4Warps][8 * NR];
    __shared__ volatile int abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kKv4Stages; ++i) {
            mbar_init(smem_u32(&full[i]), 1);
            mbar_init(smem_u32(&empty[i]), kKv4Warps);
        }
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncthreads();
    pdl_wait();
    if (blockIdx.x == 0 && threadIdx.x == 0) a.st->status = 0;      // a wait would have to fail millions of polls before this

    unsigned unit = blockIdx.x;
    const int split = unit % a.splits;
    unit /= a.splits;
    const int row_block = unit % a.row_blocks;
    unit /= a.row_blocks;
    const int head = unit % a.c.n_k, seq = unit / a.c.n_k;
    int q0, n;
    kv4_rows_of(a, seq, &q0, &n);
    const int rows = min(n, a.max_q) * a.G, row0 = row_block * 8 * NR * a.row_groups;
    if (row0 >= rows) return;
    const long long most = (long long)a.width * a.c.page;
    const int len = (int)max(0LL, min((long long)a.lens[seq], most));
    const int all = (len + kKv4StageTokens - 1) / kKv4StageTokens, per = (all + a.splits - 1) / a.splits;
    const int from = min(split * per, all), to = min(from + per, all);

    const int parts = kKv4Warps / a.row_groups;               // warps that share a row group's tokens
    const int group = warp / parts, mine = warp - group * parts;
    float acc[NR][J][4] = {};
    float m[NR][2], l[NR][2] = {}, corr[NR][NG][2] = {}, lost[NR][NG][2] = {};
    uint32_t limit = 0, f_exp = 127;                          // steps up to `limit` (bits) fit the scale of p step, 2^(127 - f_exp)

    if (warp == kKv4Warps) {
        const int32_t* table = a.table + seq * a.ld_table;
        const int subs = a.c.page / kKv4Block;
        // page of the block of 16 tokens that this lane copies of stage i, -1: none
        auto page_of = [&](int i) {
            const int sub = i * 8 + lane;
            return lane < 8 && i < to && sub * kKv4Block < len ? __ldg(table + sub / subs) : -1;
        };
        int next = page_of(from), stage = 0;
        uint32_t phase = 0;
        for (int i = from; i < to; ++i) {
            const int page = next;
            next = page_of(i + 1);
            const bool there = page >= 0 && page < a.n_pages;
            const uint32_t which = __ballot_sync(0xffffffffu, there);
            mbar_wait(smem_u32(&empty[stage]), phase ^ 1u, &abort_flag, a.st);
            const uint32_t bar = smem_u32(&full[stage]);
            if (lane == 0) {
                present[stage] = which;
                mbar_expect_tx(bar, __popc(which) * kBytes);
            }
            __syncwarp();
            if (there) {
                const int sub = i * 8 + lane;
                const unsigned char* src = a.c.base + (((long long)page * a.c.n_k + head) * subs + sub % subs) * kBytes;
                bulk_g2s(smem_u32(kv4_smem + stage * kStage + lane * kBytes), src, kBytes, bar);
            }
            if (++stage == kKv4Stages) { stage = 0; phase ^= 1u; }
        }
        // nothing is left on its way when the ring is used again or the block ends, an expired wait elsewhere included
        for (int i = max(from, to - kKv4Stages); i < to; ++i)
            mbar_wait(smem_u32(&full[(i - from) % kKv4Stages]), (uint32_t)((i - from) / kKv4Stages) & 1u, &abort_flag, a.st);
    } else {
        const int g = lane >> 2, c = lane & 3;
        // Operand B of the scores: this lane's rows g (one a tile), columns 32 w + 8 c ..., brought into fp16's range by a power of two.
        uint4 qf[NR][W];
        float lows[NR][NG][2];                                // sums of the scaled queries of rows 2c, 2c + 1, times 2^-24
        float back1[NR][2], back2[NR][2];                     // what turns a raw score of these rows into one in powers of two
        int node[NR][2];
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            const int row = row0 + (group * NR + r) * 8 + g;
            float f[W][8] = {};
            if (row < rows) {
                const int tok = row / a.G;
                const T* q = static_cast<const T*>(a.q) + (q0 + tok) * a.ld_q + (long long)(head * a.G + row - tok * a.G) * D + 8 * c;
#pragma unroll
                for (int w = 0; w < W; ++w) Elem<T>::load8(q + 32 * w, f[w]);
            }
            uint32_t big = 0;
#pragma unroll
            for (int w = 0; w < W; ++w)
#pragma unroll
                for (int i = 0; i < 8; ++i) big = max(big, __float_as_uint(f[w][i]) & 0x7fffffffu);
            big = max(big, __shfl_xor_sync(0xffffffffu, big, 1));
            big = max(big, __shfl_xor_sync(0xffffffffu, big, 2));
            const int e = q4_exponent(big);
            const Q4Power up(e), down(24 - e);
            float sum[NG] = {};
#pragma unroll
            for (int w = 0; w < W; ++w) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    f[w][i] = up(f[w][i]);
                    sum[w * NG / W] += f[w][i];
                }
                qf[r][w] = q4_operand(f[w]);
            }
#pragma unroll
            for (int i = 0; i < NG; ++i) {
                sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 1);
                sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 2);
                sum[i] *= 0x1p-24f;
            }
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int of = (2 * c + s) * 4;
#pragma unroll
                for (int i = 0; i < NG; ++i) lows[r][i][s] = __shfl_sync(0xffffffffu, sum[i], of);
                back1[r][s] = __shfl_sync(0xffffffffu, down.a, of);
                back2[r][s] = __shfl_sync(0xffffffffu, down.b, of) * a.scale2;
                node[r][s] = (row0 + (group * NR + r) * 8 + 2 * c + s) / a.G;
                m[r][s] = kNegInf;
            }
        }

        // Sixteen tokens from `token` on, at `blk`.  CUT: not every row sees all of them.
        auto work = [&](const unsigned char* blk, int token, auto cut) {
            constexpr bool CUT = decltype(cut)::value;
            float s[NR][4];
            const uint32_t* pk = reinterpret_cast<const uint32_t*>(blk + 16 * D) + g;
            {
                uint32_t kw[2][W];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const unsigned char* p = blk + h * 4 * D + lane * (D / 8);
                    if constexpr (D == 128) *reinterpret_cast<uint4*>(kw[h]) = *reinterpret_cast<const uint4*>(p);
                    else *reinterpret_cast<uint2*>(kw[h]) = *reinterpret_cast<const uint2*>(p);
                }
#pragma unroll
                for (int i = 0; i < NG; ++i) {
                    float d[NR][4] = {};
#pragma unroll
                    for (int w = i * W / NG; w < (i + 1) * W / NG; ++w) {
                        uint32_t u[4], v[4];
                        q4_spread(kw[0][w], u);
                        q4_spread(kw[1][w], v);
                        const uint32_t a0[4] = {u[0], v[0], u[1], v[1]}, a1[4] = {u[2], v[2], u[3], v[3]};
#pragma unroll
                        for (int r = 0; r < NR; ++r) {
                            q4_mma(d[r], a0, qf[r][w].x, qf[r][w].y);
                            q4_mma(d[r], a1, qf[r][w].z, qf[r][w].w);
                        }
                    }
                    const float2 p0 = kv4_pair<T>(pk[i * 16]), p1 = kv4_pair<T>(pk[i * 16 + 8]);
#pragma unroll
                    for (int r = 0; r < NR; ++r)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float2 p = e < 2 ? p0 : p1;
                            const float x = fmaf(p.x, d[r][e], p.y * lows[r][i][e & 1]);
                            s[r][e] = i == 0 ? x : s[r][e] + x;
                        }
                }
            }
            uint32_t seen = ~0u;                              // bit 4 r + e
            bool above = false;
#pragma unroll
            for (int r = 0; r < NR; ++r)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[r][e] = s[r][e] * back1[r][e & 1] * back2[r][e & 1];
                    if constexpr (CUT) {
                        const int t = token + g + (e < 2 ? 0 : 8), at = t - (len - n), row = node[r][e & 1];
                        bool see = t < len && (row0 + (group * NR + r) * 8 + 2 * c + (e & 1)) < rows;
                        if (see && at >= 0) see = a.tree ? at < kKv4MaxTree && __ldg(a.tree + q0 + row) >> at & 1ull : at <= row;
                        if (!see) {
                            seen &= ~(1u << (4 * r + e));
                            s[r][e] = kNegInf;
                        }
                    }
                    above |= s[r][e] > m[r][e & 1] + 8.f;
                }
            if (__any_sync(0xffffffffu, above)) {
#pragma unroll
                for (int r = 0; r < NR; ++r)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float t = fmaxf(m[r][h], fmaxf(s[r][h], s[r][2 + h]));
#pragma unroll
                        for (int o = 4; o < 32; o <<= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, o));
                        const float f = m[r][h] == t ? 1.f : exp2_fast(m[r][h] - t);
                        m[r][h] = t;
                        l[r][h] *= f;
#pragma unroll
                        for (int i = 0; i < NG; ++i) {
                            corr[r][i][h] *= f;
                            if constexpr (kCentre) lost[r][i][h] *= f;
                        }
#pragma unroll
                        for (int j = 0; j < J; ++j) {
                            acc[r][j][h] *= f;
                            acc[r][j][2 + h] *= f;
                        }
                    }
            }
#pragma unroll
            for (int r = 0; r < NR; ++r)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[r][e] = exp2_fast(s[r][e] - (m[r][e & 1] == kNegInf ? 0.f : m[r][e & 1]));
                    l[r][e & 1] += s[r][e];
                }
            // The scale of p step: 2^(127 - f_exp) brings the largest step so far to at most 2^6, and p is at most 2^8.
            uint32_t vp[NG][2], top = 0;
#pragma unroll
            for (int i = 0; i < NG; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    vp[i][h] = pk[(NG + i) * 16 + 8 * h];
                    const uint32_t b = __float_as_uint(kv4_pair<T>(vp[i][h]).x);
                    if ((!CUT || token + g + 8 * h < len) && b < 0x7f800000u) top = max(top, b);
                }
            top = __reduce_max_sync(0xffffffffu, top);
            if (top > limit) {
                const uint32_t e = max(1u, min(top >> 23, 253u));
                const Q4Power f((int)f_exp - (int)e);
                f_exp = e;
                limit = e + 6 < 254 ? (e + 6) << 23 : 0x7f7fffffu;
#pragma unroll
                for (int r = 0; r < NR; ++r)
#pragma unroll
                    for (int j = 0; j < J; ++j)
#pragma unroll
                        for (int x = 0; x < 4; ++x) acc[r][j][x] = f(acc[r][j][x]);
                if constexpr (kCentre) {
#pragma unroll
                    for (int r = 0; r < NR; ++r)
#pragma unroll
                        for (int i = 0; i < NG; ++i)
#pragma unroll
                            for (int h = 0; h < 2; ++h) lost[r][i][h] = f(lost[r][i][h]);
                }
            }
            const float f = __uint_as_float((254u - f_exp) << 23);
            uint32_t b0[NR][NG], b1[NR][NG];
#pragma unroll
            for (int i = 0; i < NG; ++i) {
                const float2 p0 = kv4_pair<T>(vp[i][0]), p1 = kv4_pair<T>(vp[i][1]);
#pragma unroll
                for (int r = 0; r < NR; ++r) {
                    float x[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float2 p = e < 2 ? p0 : p1;
                        x[e] = s[r][e] * (p.x * f);
                        float y = s[r][e] * p.y;
                        if (CUT && !(seen >> (4 * r + e) & 1u)) x[e] = y = 0.f;      // a step or lowest value that is not finite
                        corr[r][i][e & 1] += y;
                    }
                    const uint32_t h0 = half_pair(x[0], x[1]), h1 = half_pair(x[2], x[3]);
                    if constexpr (kCentre) {
                        const float2 f0 = kv4_pair<__half>(h0), f1 = kv4_pair<__half>(h1);
                        lost[r][i][0] += (x[0] - f0.x) + (x[2] - f1.x);
                        lost[r][i][1] += (x[1] - f0.y) + (x[3] - f1.y);
                    }
                    b0[r][i] = tile_transpose(h0);
                    b1[r][i] = tile_transpose(h1);
                }
            }
            uint32_t vw[2][2][W / 2];                         // [eight tokens][token of the pair][word]
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const unsigned char* p = blk + 8 * D + h * 4 * D + lane * (D / 8);
                if constexpr (D == 128) *reinterpret_cast<uint4*>(vw[h]) = *reinterpret_cast<const uint4*>(p);
                else *reinterpret_cast<uint2*>(vw[h]) = *reinterpret_cast<const uint2*>(p);
            }
#pragma unroll
            for (int w = 0; w < W / 2; ++w)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    uint32_t u[4], v[4];
                    q4_spread(__byte_perm(vw[0][0][w], vw[0][1][w], half ? 0x7632 : 0x5410), u);
                    q4_spread(__byte_perm(vw[1][0][w], vw[1][1][w], half ? 0x7632 : 0x5410), v);
                    const uint32_t a0[4] = {u[0], u[1], v[0], v[1]}, a1[4] = {u[2], u[3], v[2], v[3]};
                    const int j = 4 * w + 2 * half;
#pragma unroll
                    for (int r = 0; r < NR; ++r) {
                        q4_mma(acc[r][j], a0, b0[r][j * NG / J], b1[r][j * NG / J]);
                        q4_mma(acc[r][j + 1], a1, b0[r][(j + 1) * NG / J], b1[r][(j + 1) * NG / J]);
                    }
                }
        };

        const bool live = row0 + group * NR * 8 < rows;
        const int open = len - n + (a.tree ? 0 : 1);          // every row sees the tokens before this one
        int stage = 0;
        uint32_t phase = 0;
        for (int i = from; i < to; ++i) {
            mbar_wait(smem_u32(&full[stage]), phase, &abort_flag, a.st);
            const uint32_t which = abort_flag ? 0u : present[stage];
            if (live)
                for (int b = mine; b < 8; b += parts)
                    if (which >> b & 1u) {
                        const int token = (i * 8 + b) * kKv4Block;
                        const unsigned char* blk = kv4_smem + stage * kStage + b * kBytes;
                        if (token + kKv4Block <= open) work(blk, token, std::false_type{});
                        else work(blk, token, std::true_type{});
                    }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // read here, refilled by a bulk copy
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&empty[stage]));
            if (++stage == kKv4Stages) { stage = 0; phase ^= 1u; }
        }
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) {
                    l[r][h] += __shfl_xor_sync(0xffffffffu, l[r][h], o);
#pragma unroll
                    for (int i = 0; i < NG; ++i) corr[r][i][h] += __shfl_xor_sync(0xffffffffu, corr[r][i][h], o);
                }
        if constexpr (kCentre) {
            const Q4Power undo((int)f_exp - 127);
#pragma unroll
            for (int r = 0; r < NR; ++r)
#pragma unroll
                for (int i = 0; i < NG; ++i)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float x = undo(lost[r][i][h]) * 7.5f;
#pragma unroll
                        for (int o = 4; o < 32; o <<= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
                        corr[r][i][h] += x;
                    }
        }
    }
    __syncthreads();                                          // every warp is done with the ring
    float* s_out = reinterpret_cast<float*>(kv4_smem);        // [warp][row of its group][D]
    if (warp < kKv4Warps) {
        const int g = lane >> 2, c = lane & 3;
        const Q4Power undo((int)f_exp - 127 + 24);
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = r * 8 + 2 * c + h;
                float* o = s_out + (warp * 8 * NR + row) * D;
                if (g == 0) s_ml[warp][row] = make_float2(m[r][h], l[r][h]);
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    o[16 * j + g] = undo(acc[r][j][h]) + corr[r][j * NG / J][h];
                    o[16 * j + 8 + g] = undo(acc[r][j][2 + h]) * 0.0625f + corr[r][j * NG / J][h];
                }
            }
    }
    __syncthreads();
    // the warps of a row group, four columns a thread
    for (int i = threadIdx.x; i < a.row_groups * 8 * NR * (D / 4); i += kKv4Threads) {
        const int local = i / (D / 4), col = (i - local * (D / 4)) * 4;
        const int grp = local / (8 * NR), r = local - grp * 8 * NR, row = row0 + local;
        if (row >= rows) continue;
        float top = kNegInf;
        for (int w = 0; w < parts; ++w) top = fmaxf(top, s_ml[grp * parts + w][r].x);
        float sum = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int w = 0; w < parts; ++w) {
            const float2 ml = s_ml[grp * parts + w][r];
            if (ml.x == kNegInf && ml.y == 0.f) continue;
            const float f = ml.x == top ? 1.f : exp2_fast(ml.x - top);
            const float4 v = *reinterpret_cast<const float4*>(s_out + ((grp * parts + w) * 8 * NR + r) * D + col);
            sum += f * ml.y;
            o.x += f * v.x; o.y += f * v.y; o.z += f * v.z; o.w += f * v.w;
        }
        const int tok = row / a.G;
        const long long at = (long long)(q0 + tok) * a.n_q + head * a.G + row - tok * a.G;
        if (a.splits > 1) {
            const long long p = (long long)split * a.n_rows * a.n_q + at;
            *reinterpret_cast<float4*>(a.part_o + p * D + col) = o;
            if (col == 0) a.part_ml[p] = make_float2(top, sum);
        } else {
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            T* to_out = static_cast<T*>(a.out) + (long long)(q0 + tok) * a.ld_out + (long long)(head * a.G + row - tok * a.G) * D + col;
            const T v[4] = {Elem<T>::down(o.x * inv), Elem<T>::down(o.y * inv), Elem<T>::down(o.z * inv), Elem<T>::down(o.w * inv)};
            *reinterpret_cast<uint2*>(to_out) = *reinterpret_cast<const uint2*>(v);
            if (a.lse && col == 0) a.lse[at] = sum == 0.f ? kNegInf : (top + log2f(sum)) * 0.69314718055994531f;
        }
    }
    pdl_launch_dependents();
}

// Adds up the parts of split caches.  A warp a row and head, D / 32 columns a lane.
template <typename T, int D>
__global__ void __launch_bounds__(256) kv4_join_kernel(const Kv4Args a) {
    constexpr int N = D / 32;
    const long long i = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    pdl_wait();
    const int head = (int)(i % a.n_q);
    const long long node = i / a.n_q;
    const long long seq = node / a.max_q;
    if (seq >= a.n_seq) return;
    int q0, n;
    kv4_rows_of(a, (int)seq, &q0, &n);
    const int tok = (int)(node - seq * a.max_q);
    if (tok >= min(n, a.max_q)) return;
    const long long at = (long long)(q0 + tok) * a.n_q + head, step = (long long)a.n_rows * a.n_q;
    float top = kNegInf;
    for (int s = lane; s < a.splits; s += 32) top = fmaxf(top, __ldcg(&a.part_ml[s * step + at]).x);
    top = warp_max(top);
    float sum = 0.f, o[N] = {};
    for (int s = 0; s < a.splits; ++s) {
        const float2 ml = __ldcg(&a.part_ml[s * step + at]);
        if (ml.x == kNegInf && ml.y == 0.f) continue;
        const float f = ml.x == top ? 1.f : exp2_fast(ml.x - top);
        sum += f * ml.y;
        const float* p = a.part_o + (s * step + at) * D + lane * N;
        if constexpr (N == 4) {
            const float4 v = __ldcg(reinterpret_cast<const float4*>(p));
            o[0] += f * v.x; o[1] += f * v.y; o[2] += f * v.z; o[3] += f * v.w;
        } else {
            const float2 v = __ldcg(reinterpret_cast<const float2*>(p));
            o[0] += f * v.x; o[1] += f * v.y;
        }
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    T v[N];
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = Elem<T>::down(o[j] * inv);
    T* out = static_cast<T*>(a.out) + (long long)(q0 + tok) * a.ld_out + (long long)head * D + lane * N;
    if constexpr (N == 4) *reinterpret_cast<uint2*>(out) = *reinterpret_cast<const uint2*>(v);
    else *reinterpret_cast<uint32_t*>(out) = *reinterpret_cast<const uint32_t*>(v);
    if (a.lse && lane == 0) a.lse[at] = sum == 0.f ? kNegInf : (top + log2f(sum)) * 0.69314718055994531f;
}

}  // namespace coral

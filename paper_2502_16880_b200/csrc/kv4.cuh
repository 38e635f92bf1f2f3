// A paged cache of keys and values held in 4 bits, and attention of few queries over it.
//
// A group of 32, 64 or 128 columns of a token's head is held as codes 0..15 of a step and a lowest value (both of the element type):
//   low = min x, step = round((max x - min x) / 15), code = round((x - low) / step) in 0..15, x ~ low + step code.
// With x split that way the score of a token needs whole numbers as operands only:
//   q . k = sum over groups of step_g (sum of q code) + low_g (sum of q)
// and so does the output, with p the weights of the softmax:
//   out = sum over tokens of (p step_g) code + sum of p low_g.
// Codes go to the warp MMA as fp16 subnormals (two operations a pair, no arithmetic); what is rounded is p step_g, to fp16, as p
// would be for 16-bit values, times a power of two that follows the row's and the group's own largest p step_g: what a row does not
// see, or gives next to no weight, or what other groups hold, takes no bits from it.
//
// Layout: tokens in blocks of 16, [page][head][block of 16]: keys, values, (step, low) pairs of keys [group][16], of values.
//   keys:   [16][4 lanes] of D / 8 bytes: column c is nibble c % 8 of word c / 32 of lane (c / 8) % 4
//   values: [2][8 column places][4 pairs of tokens][D / 32][2 tokens] 16-bit pieces: column c is nibble (c / 8) % 4 of piece c / 32 of place c % 8
// so that a lane's MMA operands are one 16-byte (D = 64: 8-byte) shared-memory load each, without bank conflicts, the two tokens of
// an operand's pair lie in the halves of a word, and no two tokens share a byte.
#pragma once
#include <type_traits>

#include "mbarrier.cuh"
#include "q4_prims.cuh"

namespace coral {

constexpr int kKv4Block = 16;                       // tokens of a block

// Quotients by a divisor known on the host: n / d = (umulhi(n, m) + n) >> s for n below 2^31, with s = ceil(log2 d) and
// m = floor(2^32 (2^s - d) / d) + 1 (the multiply-and-shift division of Granlund and Montgomery).
struct Divide {
    uint32_t m, s, d;
    Divide() = default;
    __host__ explicit Divide(uint32_t by) : m(0), s(0), d(by) {
        while ((1u << s) < by) ++s;
        m = (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << s) - by)) / by + 1);
    }
    __device__ __forceinline__ int operator()(int n) const { return (int)((__umulhi((uint32_t)n, m) + (uint32_t)n) >> s); }
};

struct Kv4Cache {
    unsigned char* base;
    int slots;                                      // pages * page
    int n_k, page, groups, share;                   // share: log2 of the threads, of eight columns each, that have a group
    Divide heads, subs;                             // by n_k, and by the blocks of a page
    __host__ __device__ int block_bytes(int D) const { return kKv4Block * D + 128 * groups; }
    // start of the block that holds slot `slot` of head `head`
    __device__ __forceinline__ unsigned char* block(int slot, int head, int D) const {
        const int sub = slot / kKv4Block, page_at = subs(sub), per = (int)subs.d;
        return base + (long long)((page_at * n_k + head) * per + (sub - page_at * per)) * block_bytes(D);
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
// Bound by instructions: eight columns a thread, whose codes (and their way to the values' layout) are integer work.  16384 tokens of 8 heads
// of 128 stored and read back, bf16: 60 us (26 of bytes), 80 and 72 % of the issue slots; 113 with codes by division and
// values transposed number by number, 75 with groups found by division instead of shifts.
constexpr int kKv4RowThreads = 256;
struct Kv4Rows {
    const int64_t* slots;
    int rows;                                       // tokens * heads
    void *k, *v;                                    // inputs of a store, outputs of a load
    long long ld_k, ld_v;
};

// Eight 4-bit numbers of eight threads, transposed: thread i's word of numbers n becomes thread n's word of numbers i.
__device__ __forceinline__ uint32_t nibbles_transposed(uint32_t w, int lane) {
    // by distance 4, 2, 1: the half of the numbers that belongs to the partner goes there
    uint32_t o = __shfl_xor_sync(0xffffffffu, w, 4);
    w = lane & 4 ? (w & 0xffff0000u) | o >> 16 : (w & 0x0000ffffu) | o << 16;
    o = __shfl_xor_sync(0xffffffffu, w, 2);
    w = lane & 2 ? (w & 0xff00ff00u) | (o >> 8 & 0x00ff00ffu) : (w & 0x00ff00ffu) | (o & 0x00ff00ffu) << 8;
    o = __shfl_xor_sync(0xffffffffu, w, 1);
    return lane & 1 ? (w & 0xf0f0f0f0u) | (o >> 4 & 0x0f0f0f0fu) : (w & 0x0f0f0f0fu) | (o & 0x0f0f0f0fu) << 4;
}

// What a thread of D / 8 a row of a head works on: eight columns of the keys (blockIdx.y 0) or values (1).
template <int D>
struct Kv4Place {
    static constexpr int L = D / 8;
    int row, token, head, l, slot;
    bool is_v, on;
    __device__ __forceinline__ Kv4Place(const Kv4Cache& c, const Kv4Rows& a) {
        row = (int)(blockIdx.x * (kKv4RowThreads / L) + threadIdx.x / L);
        l = threadIdx.x & (L - 1);
        is_v = blockIdx.y != 0;
        token = c.heads(row);
        head = row - token * c.n_k;
        const int64_t at = row < a.rows ? a.slots[token] : -1;
        on = at >= 0 && at < c.slots;
        slot = (int)at;
    }
    template <typename T>
    __device__ __forceinline__ T* columns(const Kv4Rows& a) const {
        return static_cast<T*>(is_v ? a.v : a.k) + token * (is_v ? a.ld_v : a.ld_k) + head * D + 8 * l;
    }
    // The thread's word of codes: eight columns of the keys, or two pieces of a column place of the values.
    __device__ __forceinline__ uint32_t* keys(unsigned char* blk) const {
        return reinterpret_cast<uint32_t*>(blk + ((slot & 15) * 4 + (l & 3)) * (D / 8) + 4 * (l >> 2));
    }
    __device__ __forceinline__ uint16_t* values(unsigned char* blk) const {
        const int t = slot & 15;
        return reinterpret_cast<uint16_t*>(blk + 8 * D + (t >> 3) * (4 * D) + ((l & 7) * 4 + ((t & 7) >> 1)) * (D / 8) + 8 * (l >> 3)) + (t & 1);
    }
    __device__ __forceinline__ void put(unsigned char* blk, uint32_t word) const {
        if (is_v) {
            values(blk)[0] = (uint16_t)word;
            values(blk)[2] = (uint16_t)(word >> 16);
        } else {
            *keys(blk) = word;
        }
    }
    __device__ __forceinline__ uint32_t get(unsigned char* blk) const { return is_v ? values(blk)[0] | (uint32_t)values(blk)[2] << 16 : *keys(blk); }
    // its group's (step, low)
    __device__ __forceinline__ uint32_t* pair(unsigned char* blk, const Kv4Cache& c) const {
        return reinterpret_cast<uint32_t*>(blk + 16 * D) + ((is_v ? c.groups : 0) + (l >> c.share)) * 16 + (slot & 15);
    }
};

// (lowest, - highest) of eight elements; a NaN stays one.
template <typename T> struct Kv4Range;
template <> struct Kv4Range<__nv_bfloat16> {
    using Two = __nv_bfloat162;
    static __device__ __forceinline__ Two min2(Two a, Two b) { return __hmin2_nan(a, b); }
    static __device__ __forceinline__ Two max2(Two a, Two b) { return __hmax2_nan(a, b); }
    static __device__ __forceinline__ Two ends(Two low, Two high) {
        const __nv_bfloat16 l = __hmin_nan(low.x, low.y), h = __hmax_nan(high.x, high.y);
        return __halves2bfloat162(l, __hneg(h));
    }
};
template <> struct Kv4Range<__half> {
    using Two = __half2;
    static __device__ __forceinline__ Two min2(Two a, Two b) { return __hmin2_nan(a, b); }
    static __device__ __forceinline__ Two max2(Two a, Two b) { return __hmax2_nan(a, b); }
    static __device__ __forceinline__ Two ends(Two low, Two high) {
        const __half l = __hmin_nan(__low2half(low), __high2half(low)), h = __hmax_nan(__low2half(high), __high2half(high));
        return __halves2half2(l, __hneg(h));
    }
};

template <typename T, int D>
__global__ void __launch_bounds__(kKv4RowThreads) kv4_store_kernel(const __grid_constant__ Kv4Cache c, const __grid_constant__ Kv4Rows a) {
    constexpr int L = D / 8;
    using Range = Kv4Range<T>;
    using Two = typename Range::Two;
    pdl_wait();
    const Kv4Place<D> p(c, a);
    uint32_t raw[4] = {};
    if (p.on) *reinterpret_cast<uint4*>(raw) = *reinterpret_cast<const uint4*>(p.template columns<T>(a));
    const Two* r2 = reinterpret_cast<const Two*>(raw);
    Two ends = Range::ends(Range::min2(Range::min2(r2[0], r2[1]), Range::min2(r2[2], r2[3])), Range::max2(Range::max2(r2[0], r2[1]), Range::max2(r2[2], r2[3])));
    const int per = 1 << c.share;                   // threads of a group
#pragma unroll
    for (int o = 1; o < L; o <<= 1)
        if (o < per) {
            const uint32_t other = __shfl_xor_sync(0xffffffffu, *reinterpret_cast<uint32_t*>(&ends), o);
            ends = Range::min2(ends, *reinterpret_cast<const Two*>(&other));
        }
    const float2 lh = kv4_pair<T>(*reinterpret_cast<uint32_t*>(&ends));
    const float range = -lh.y - lh.x, bad = range * 0.f;       // NaN for an infinity or a NaN, and for a range that fp32 does not hold
    const uint32_t step_bits = kv4_bits<T>(range / 15.f + bad);
    const float step = kv4_pair<T>(step_bits).x;
    // Codes by the reciprocal and one step towards the quotient, rounded by adding 1.5 2^23.  A quotient in the middle between two
    // codes has few bits and comes out exact.  (A subnormal step has no reciprocal in fp32.)
    const float inv = step > 1e-37f ? __frcp_rn(step) : 0.f;
    constexpr float kRound = 12582912.f;
    const unsigned long long inv2 = pair_of(inv, inv), low2 = pair_of(-lh.x, -lh.x), step2 = pair_of(-step, -step), round2 = pair_of(kRound, kRound);
    uint32_t word = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 x = kv4_pair<T>(raw[i]);
        const unsigned long long d = add2(pair_of(x.x, x.y), low2), q = mul2(d, inv2);
        const float2 f = halves(fma2(fma2(q, step2, d), inv2, q));
        const float2 n = halves(add2(pair_of(fminf(f.x, 15.f), fminf(f.y, 15.f)), round2));
        word += __float_as_uint(n.x) << (8 * i);
        word += __float_as_uint(n.y) << (8 * i + 4);
    }
    constexpr uint32_t kBits = 0x4b400000u;         // of kRound: what each code has added
    word -= kBits * 0x11111111u;
    if (step > 0.f && !(step > 1e-37f)) {
        word = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 x = kv4_pair<T>(raw[i / 2]);
            word |= (uint32_t)fminf(rintf(((i & 1 ? x.y : x.x) - lh.x) / step), 15.f) << (4 * i);
        }
    }
    if (p.is_v) word = nibbles_transposed(word, p.l);
    if (!p.on) return;
    unsigned char* blk = c.block(p.slot, p.head, D);
    p.put(blk, word);
    if ((p.l & (per - 1)) == 0) *p.pair(blk, c) = step_bits | kv4_bits<T>(lh.x + bad) << 16;
}

template <typename T, int D>
__global__ void __launch_bounds__(kKv4RowThreads) kv4_load_kernel(const __grid_constant__ Kv4Cache c, const __grid_constant__ Kv4Rows a) {
    pdl_wait();
    if (!(blockIdx.y ? a.v : a.k)) return;
    const Kv4Place<D> p(c, a);
    uint32_t word = 0, pair = 0;
    if (p.on) {
        unsigned char* blk = c.block(p.slot, p.head, D);
        word = p.get(blk);
        pair = *p.pair(blk, c);
    }
    if (p.is_v) word = nibbles_transposed(word, p.l);
    if (p.row >= a.rows) return;
    const float2 s = kv4_pair<T>(pair);
    constexpr uint32_t kBits = 0x4b000000u;         // 2^23: a code in its lowest bits becomes a number without a conversion
    const unsigned long long less = pair_of(-8388608.f, -8388608.f), step = pair_of(s.x, s.x), low = pair_of(s.y, s.y);
    V8 x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float n0 = __uint_as_float((word >> (8 * i) & 15u) | kBits), n1 = __uint_as_float((word >> (8 * i + 4) & 15u) | kBits);
        x.p[i] = fma2(add2(pair_of(n0, n1), less), step, low);
    }
    store8v<T>(p.template columns<T>(a), x);
}

// ---- attention -----------------------------------------------------------------------------------------------
// A block takes all rows of a key head (query tokens of a sequence times the query heads; 8 NR row_groups at most, with row_groups 1 or 2) and a
// span of the sequence's cache.  Its eight warps are row groups of `parts` warps; warp i of each group takes every parts-th chunk of U blocks
// of 16 tokens, so the warps of one number share a stream of chunks and the others do without them:
//   scores  [16 tokens x 8 rows] = K (operand A, unpacked) Q^T,   out [D x 8 rows] += V^T (operand A, unpacked) P^T
// with tokens and columns on the MMA's long side, so one sequence's few rows cost no more than 8 and an unpacked operand serves
// NR MMAs.  A stream has a ring of chunks, filled by its first warp with one bulk copy a block (whatever the page size).  The running
// maximum is a reference, moved only when a score passes it by 2^8, so that most chunks need one vote and no shuffles.  Long
// caches are split over blocks, and kv4_join_kernel adds the parts up.
// 131072 tokens of 8 heads of 128, 4 rows each, bf16: 39 us with the join, 56 % of the copy bandwidth measured; 64 sequences of up to 4096
// tokens, 4 heads, 7 rows: 36 us, 49 %.  (One power of two a warp, by the steps of all its tokens, took 38.9 and 35.2 against 39.1 and 35.9, but
// left rows without their bits beside a token or group of much larger values.)  What bounds it: the chain of unpacking, MMA, weights and MMA of a
// chunk, of which 128 registers leave 16 warps a SM (48 % of the issue slots), and its start, end and join, 5 to 9 us.
constexpr int kKv4Warps = 8;
constexpr int kKv4Threads = kKv4Warps * 32;
constexpr int kKv4SpanBlocks = 16;                  // spans of a split are a multiple of so many blocks of 16 tokens
constexpr int kKv4MaxSplits = 256;
constexpr int kKv4MaxTree = 64;                     // query tokens under a tree mask

struct Kv4Args {
    Kv4Cache c;
    int n_seq, n_rows, max_q, n_q, G, width, n_pages;
    int row_groups, splits, slots;                  // (up to 32 rows) row groups, and chunks of a stream's ring
    int row_blocks;                                 // (more) blocks that share a key head's rows
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
__device__ __forceinline__ uint32_t half2_minus(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
// The transpose of an 8 x 8 tile of 16-bit values, a row's pair a thread.
__device__ __forceinline__ uint32_t tile_transpose(uint32_t v) {
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}

constexpr float kKv4NoMax = -3e38f;                 // the reference before any score; finite, so that nothing is inf - inf

// What a warp keeps of its 8 NR rows.  Accumulators of the MMA: columns 16 j + g and + 8 (times 16), rows 2c and 2c + 1 of a tile, with
// g = lane / 4, c = lane % 4; everything a row has is kept for the pair of rows 2c, 2c + 1.
template <typename T, int D, int NG, int NR>
struct Kv4Rowset {
    static constexpr int kBytes = kKv4Block * D + 128 * NG;  // of a block of 16 tokens
    static constexpr int W = D / 32, J = D / 16;             // words of a lane and token; tiles of 16 columns
    // fp16 outputs: the values' operand is code - 8 (exact as well), so that the rounding of p step weighs that and not code
    // (0.0005 -> 0.0003 of the output; bf16 outputs, rounded to 0.0017, do not show it)
    static constexpr bool kCentre = std::is_same_v<T, __half>;
    using Pair = unsigned long long;
    // A row moves when one of its p passes 2^8 or an operand 2^15 (fp16 ends below 2^16); its largest p step so far is then brought to
    // 2^6..2^7, so that what fp16's subnormals lose of an operand is 2^-31 of that at most.
    static constexpr int kMostPower = 126, kMoved = 6;
    static constexpr float kMostP = 256.f, kMostOperand = 32768.f;

    float acc[NR][J][4];
    float m[NR][2];
    Pair l[NR], corr[NR][NG];
    Pair power[NR][NG];                                      // powers of two: acc is in units of 2^-24 / power, operand B is p step power
    // operand B of the scores, sums of the scaled queries (times 2^-24), and what makes a raw score one in powers of two
    uint4 qf[NR][W];
    Pair low[NR][NG], back[NR];
    int node[NR][2];                                         // query token of a row, past all of them for rows that do not exist

    static __device__ __forceinline__ Pair both(float v) { return pair_of(v, v); }

    // Rows row0 ... of the sequence whose first query row is q0; columns 32 w + 8 c ... of row g are this lane's part of operand B.
    __device__ __forceinline__ void begin(const Kv4Args& a, int q0, int head, int row0, int rows) {
        const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            const int row = row0 + r * 8 + g;
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
            const int e = q4_exponent(big);                  // the power of two that brings the row into fp16's range
            const Q4Power up(e), down(24 - e);
            const float undo = a.scale2 * down.a * down.b;
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
                low[r][i] = pair_of(__shfl_sync(0xffffffffu, sum[i], 8 * c), __shfl_sync(0xffffffffu, sum[i], 8 * c + 4));
                corr[r][i] = 0;
                power[r][i] = both(exp2_int(kMostPower));
            }
            back[r] = pair_of(__shfl_sync(0xffffffffu, undo, 8 * c), __shfl_sync(0xffffffffu, undo, 8 * c + 4));
            l[r] = 0;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int at = row0 + r * 8 + 2 * c + s;
                node[r][s] = at < rows ? at / a.G : 0x7fffffff;
                m[r][s] = kKv4NoMax;
            }
#pragma unroll
            for (int j = 0; j < J; ++j)
#pragma unroll
                for (int x = 0; x < 4; ++x) acc[r][j][x] = 0.f;
        }
    }

    // Raw scores of a block's tokens g and g + 8: s[row tile][token].
    __device__ __forceinline__ void scores(const unsigned char* blk, Pair (&s)[NR][2]) const {
        const int lane = threadIdx.x & 31;
        const uint32_t* pk = reinterpret_cast<const uint32_t*>(blk + 16 * D) + (lane >> 2);
        uint32_t kw[2][W];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const unsigned char* p = blk + h * 4 * D + lane * (D / 8);
            if constexpr (D == 128) *reinterpret_cast<uint4*>(kw[h]) = *reinterpret_cast<const uint4*>(p);
            else *reinterpret_cast<uint2*>(kw[h]) = *reinterpret_cast<const uint2*>(p);
        }
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            float d[NR][2][4] = {};                           // two chains of MMAs
#pragma unroll
            for (int w = i * W / NG; w < (i + 1) * W / NG; ++w) {
                uint32_t u[4], v[4];
                q4_spread(kw[0][w], u);
                q4_spread(kw[1][w], v);
                const uint32_t a0[4] = {u[0], v[0], u[1], v[1]}, a1[4] = {u[2], v[2], u[3], v[3]};
#pragma unroll
                for (int r = 0; r < NR; ++r) {
                    q4_mma(d[r][0], a0, qf[r][w].x, qf[r][w].y);
                    q4_mma(d[r][W / NG > 1 ? 1 : 0], a1, qf[r][w].z, qf[r][w].w);
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float2 p = kv4_pair<T>(pk[i * 16 + 8 * h]);
#pragma unroll
                for (int r = 0; r < NR; ++r) {
                    Pair x = pair_of(d[r][0][2 * h], d[r][0][2 * h + 1]);
                    if (W / NG > 1) x = add2(x, pair_of(d[r][1][2 * h], d[r][1][2 * h + 1]));
                    const Pair y = i == 0 ? mul2(both(p.y), low[r][i]) : fma2(both(p.y), low[r][i], s[r][h]);
                    s[r][h] = fma2(both(p.x), x, y);
                }
            }
        }
    }

    // The reference of the maximum and the powers of rows whose p or operands ask for it: p anew from the raw scores s of the tokens that are
    // seen (bit ((u NR + r) 2 + h) 2 + e), vp their steps.  A row goes by its own tokens alone: the rest of the warp keeps its bits.
    template <int U>
    __device__ __forceinline__ void move(const Pair (&s)[U][NR][2], Pair (&p)[U][NR][2], const uint32_t (&vp)[U][NG][2], uint32_t seen) {
        const uint32_t mine = 0x11111111u << (threadIdx.x & 3);             // the lanes that have this one's rows
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            float f[2];
            bool moves[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float t = m[r][e], most = 0.f, operand = 0.f;
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float2 raw = halves(mul2(s[u][r][h], back[r])), now = halves(p[u][r][h]);
                        if (seen >> (((u * NR + r) * 2 + h) * 2 + e) & 1u) t = fmaxf(t, e ? raw.y : raw.x);
                        most = fmaxf(most, e ? now.y : now.x);
#pragma unroll
                        for (int i = 0; i < NG; ++i) {
                            const float2 w = halves(mul2(mul2(p[u][r][h], both(kv4_pair<T>(vp[u][i][h]).x)), power[r][i]));
                            operand = fmaxf(operand, e ? w.y : w.x);
                        }
                    }
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, o));
                moves[e] = (__ballot_sync(0xffffffffu, most > kMostP || operand > kMostOperand) & mine) != 0;
                f[e] = !moves[e] || m[r][e] == t ? 1.f : exp2_fast(m[r][e] - t);
                if (moves[e]) m[r][e] = t;
            }
            const Pair f2 = pair_of(f[0], f[1]);
            l[r] = mul2(l[r], f2);
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    // (the product rounded as in the maximum: of scores beyond 2^24, one fused step would leave more than the 2^8 that p has room for)
                    const float2 old = halves(p[u][r][h]), x = halves(add2(mul2(s[u][r][h], back[r]), pair_of(-m[r][0], -m[r][1])));
                    const uint32_t on = seen >> (((u * NR + r) * 2 + h) * 2);
                    p[u][r][h] = pair_of(!moves[0] ? old.x : on & 1u ? exp2_fast(x.x) : 0.f, !moves[1] ? old.y : on & 2u ? exp2_fast(x.y) : 0.f);
                }
#pragma unroll
            for (int i = 0; i < NG; ++i) {
                corr[r][i] = mul2(corr[r][i], f2);
                const float2 had = halves(power[r][i]);
                float now[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    // what had the old power's 2^kMoved (or more) counts with what it is now, 2^(kMoved - exponent) f
                    const int old = (int)(__float_as_uint(e ? had.y : had.x) >> 23);
                    float largest = exp2_int(kMoved + 127 - old) * f[e];
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const float2 w = halves(mul2(p[u][r][h], both(kv4_pair<T>(vp[u][i][h]).x)));     // p is at most 1 here: no overflow
                            largest = fmaxf(largest, e ? w.y : w.x);
                        }
#pragma unroll
                    for (int o = 4; o < 32; o <<= 1) largest = fmaxf(largest, __shfl_xor_sync(0xffffffffu, largest, o));
                    const int next = moves[e] ? min(max(2 * 127 + kMoved - (int)(__float_as_uint(largest) >> 23), 127 - kMostPower + kMoved), 127 + kMostPower) : old;
                    now[e] = __uint_as_float((uint32_t)next << 23);
                    const Q4Power by(next - old);
#pragma unroll
                    for (int j = i * J / NG; j < (i + 1) * J / NG; ++j)
#pragma unroll
                        for (int k = 0; k < 2; ++k) acc[r][j][2 * k + e] = by(acc[r][j][2 * k + e] * f[e]);
                }
                power[r][i] = pair_of(now[0], now[1]);
            }
        }
    }

    // U blocks of 16 tokens from `token` on, side by side at blk.  CUT: not every row sees all of them (past: tokens that all rows see, len:
    // tokens of the sequence, there: which of the U blocks there are).
    template <int U, bool CUT>
    __device__ __forceinline__ void work(const Kv4Args& a, const unsigned char* blk, int token, int q0, int past, int len, uint32_t there) {
        const int lane = threadIdx.x & 31, g = lane >> 2;
        Pair s[U][NR][2], p[U][NR][2];
#pragma unroll
        for (int u = 0; u < U; ++u) scores(blk + u * kBytes, s[u]);
        float above = 0.f, operand = 0.f, step_top[NG] = {};  // (a NaN is passed over)
        float2 p_top[NR] = {};
        uint32_t vp[U][NG][2], seen = ~0u;                    // bit ((u NR + r) 2 + h) 2 + e
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t* pv = reinterpret_cast<const uint32_t*>(blk + u * kBytes + 16 * D) + NG * 16 + g;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int t = token + 16 * u + 8 * h + g;
                const bool real = !CUT || (t < len && (there >> u & 1u));
#pragma unroll
                for (int i = 0; i < NG; ++i) {
                    vp[u][i][h] = pv[i * 16 + 8 * h];
                    step_top[i] = fmaxf(step_top[i], kv4_pair<T>(vp[u][i][h]).x);
                }
#pragma unroll
                for (int r = 0; r < NR; ++r) {
                    float2 v = halves(fma2(s[u][r][h], back[r], pair_of(-m[r][0], -m[r][1])));
                    if constexpr (CUT) {
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int at = t - past, row = node[r][e];
                            bool see = real && row != 0x7fffffff;
                            if (see && at >= 0) see = a.tree ? at < kKv4MaxTree && __ldg(a.tree + q0 + row) >> at & 1ull : at <= row;
                            if (!see) {
                                seen &= ~(1u << (((u * NR + r) * 2 + h) * 2 + e));
                                (e ? v.y : v.x) = kNegInf;
                            }
                        }
                    }
                    v = make_float2(exp2_fast(v.x), exp2_fast(v.y));
                    p_top[r] = make_float2(fmaxf(p_top[r].x, v.x), fmaxf(p_top[r].y, v.y));
                    p[u][r][h] = pair_of(v.x, v.y);
                }
            }
        }
        // Operands are at most the largest p of a row times the largest step, whichever tokens have them (and see them): move() looks closer.
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            above = fmaxf(above, fmaxf(p_top[r].x, p_top[r].y));
#pragma unroll
            for (int i = 0; i < NG; ++i) {
                const float2 w = halves(mul2(mul2(pair_of(p_top[r].x, p_top[r].y), both(step_top[i])), power[r][i]));
                operand = fmaxf(operand, fmaxf(w.x, w.y));
            }
        }
        if (__any_sync(0xffffffffu, above > kMostP || operand > kMostOperand)) move<U>(s, p, vp, seen);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            uint32_t b[NR][NG][2];
#pragma unroll
            for (int r = 0; r < NR; ++r)
#pragma unroll
                for (int h = 0; h < 2; ++h) l[r] = add2(l[r], p[u][r][h]);
#pragma unroll
            for (int i = 0; i < NG; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float2 pr = kv4_pair<T>(vp[u][i][h]);
                    const Pair step = both(pr.x), lowest = both(kCentre ? fmaf(8.f, pr.x, pr.y) : pr.y);
#pragma unroll
                    for (int r = 0; r < NR; ++r) {
                        float2 w;
                        if constexpr (CUT) {                  // a step or lowest value that is not finite has no part in what is not seen
                            const uint32_t on = seen >> (((u * NR + r) * 2 + h) * 2);
                            const float2 q = halves(mul2(mul2(p[u][r][h], step), power[r][i])), y = halves(mul2(p[u][r][h], lowest));
                            w = make_float2(on & 1u ? q.x : 0.f, on & 2u ? q.y : 0.f);
                            corr[r][i] = add2(corr[r][i], pair_of(on & 1u ? y.x : 0.f, on & 2u ? y.y : 0.f));
                        } else {
                            w = halves(mul2(mul2(p[u][r][h], step), power[r][i]));
                            corr[r][i] = fma2(p[u][r][h], lowest, corr[r][i]);
                        }
                        b[r][i][h] = tile_transpose(half_pair(w.x, w.y));
                    }
                }
            uint32_t vw[2][W];                                // [eight tokens][four columns of a pair of tokens]
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const unsigned char* at = blk + u * kBytes + 8 * D + h * 4 * D + lane * (D / 8);
                if constexpr (D == 128) *reinterpret_cast<uint4*>(vw[h]) = *reinterpret_cast<const uint4*>(at);
                else *reinterpret_cast<uint2*>(vw[h]) = *reinterpret_cast<const uint2*>(at);
            }
#pragma unroll
            for (int w = 0; w < W; ++w) {
                uint32_t c[4], d[4];
                q4_spread(vw[0][w], c);
                q4_spread(vw[1][w], d);
                if constexpr (kCentre)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        c[k] = half2_minus(c[k], k & 1 ? 0x00800080u : 0x00080008u);
                        d[k] = half2_minus(d[k], k & 1 ? 0x00800080u : 0x00080008u);
                    }
                const uint32_t a0[4] = {c[0], c[1], d[0], d[1]}, a1[4] = {c[2], c[3], d[2], d[3]};
                const int j = 2 * w;
#pragma unroll
                    for (int r = 0; r < NR; ++r) {
                        q4_mma(acc[r][j], a0, b[r][j * NG / J][0], b[r][j * NG / J][1]);
                        q4_mma(acc[r][j + 1], a1, b[r][(j + 1) * NG / J][0], b[r][(j + 1) * NG / J][1]);
                    }
            }
        }
    }

    // Sums over the lanes of a row; out [row of the set][D] unnormalised and ml [row] (reference, sum).
    __device__ __forceinline__ void end(float* out, float2* ml) {
        const int lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
        auto over_lanes = [](Pair v) {
            float2 f = halves(v);
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) {
                f.x += __shfl_xor_sync(0xffffffffu, f.x, o);
                f.y += __shfl_xor_sync(0xffffffffu, f.y, o);
            }
            return f;
        };
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            float fix[NG][2];
            Q4Power undo[NG][2];
#pragma unroll
            for (int i = 0; i < NG; ++i) {
                const float2 v = over_lanes(corr[r][i]);
                fix[i][0] = v.x;
                fix[i][1] = v.y;
                const float2 had = halves(power[r][i]);
                undo[i][0] = Q4Power(127 + 24 - (int)(__float_as_uint(had.x) >> 23));
                undo[i][1] = Q4Power(127 + 24 - (int)(__float_as_uint(had.y) >> 23));
            }
            const float2 sum = over_lanes(l[r]);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = r * 8 + 2 * c + h;
                if (g == 0) ml[row] = make_float2(m[r][h], h ? sum.y : sum.x);
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    out[row * D + 16 * j + g] = undo[j * NG / J][h](acc[r][j][h]) + fix[j * NG / J][h];
                    out[row * D + 16 * j + 8 + g] = undo[j * NG / J][h](acc[r][j][2 + h]) * 0.0625f + fix[j * NG / J][h];
                }
            }
        }
    }
};

// Blocks of 16 tokens a chunk, ring of a block in bytes: two blocks a SM where a warp has eight rows.
template <int NG, int NR> constexpr int kKv4Chunk = NR == 1 && NG < 4 ? 2 : 1;
template <int NR> constexpr int kKv4Ring = NR == 1 ? 108 * 1024 : 192 * 1024;
constexpr int kKv4MaxSlots = 12;

template <typename T, int D, int NG, int NR>
__global__ void __launch_bounds__(kKv4Threads, NR == 1 ? 2 : 1) kv4_attention_kernel(const __grid_constant__ Kv4Args a) {
    using Rowset = Kv4Rowset<T, D, NG, NR>;
    constexpr int kBytes = Rowset::kBytes, U = kKv4Chunk<NG, NR>;
    extern __shared__ __align__(128) unsigned char kv4_smem[];
    __shared__ __align__(8) uint64_t full[kKv4Warps * kKv4MaxSlots], empty[kKv4Warps * kKv4MaxSlots];
    __shared__ uint32_t present[kKv4Warps * kKv4MaxSlots];    // which blocks of a chunk there are
    __shared__ float2 s_ml[kKv4Warps][8 * NR];
    __shared__ volatile int abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int parts = kKv4Warps / a.row_groups, group = warp / parts, mine = warp - group * parts;
    if (threadIdx.x == 0) abort_flag = 0;
    for (int i = threadIdx.x; i < parts * a.slots; i += kKv4Threads) {
        mbar_init(smem_u32(&full[i]), 1);
        mbar_init(smem_u32(&empty[i]), a.row_groups);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();
    pdl_wait();
    if (blockIdx.x == 0 && threadIdx.x == 0) a.st->status = 0;      // a wait would have to fail millions of polls before this

    unsigned unit = blockIdx.x;
    const int split = unit % a.splits;
    unit /= a.splits;
    const int head = unit % a.c.n_k, seq = unit / a.c.n_k;
    int q0, n;
    kv4_rows_of(a, seq, &q0, &n);
    const int rows = min(n, a.max_q) * a.G;
    if (rows == 0) return;
    const int len = (int)max(0LL, min((long long)a.lens[seq], min((long long)a.width * a.c.page, 0x7fff0000LL)));
    const int spans = (len + kKv4SpanBlocks * kKv4Block - 1) / (kKv4SpanBlocks * kKv4Block), per = (spans + a.splits - 1) / a.splits;
    // chunks of this block, and those of this warp's stream: from + mine, from + mine + parts, ...
    const int from = min(split * per, spans) * (kKv4SpanBlocks / U), to = min(min(split * per, spans) + per, spans) * (kKv4SpanBlocks / U);
    const int chunks = (to - from - mine + parts - 1) / parts;

    unsigned char* ring = kv4_smem + mine * a.slots * (U * kBytes);
    const int bar0 = mine * a.slots;
    const int32_t* table = a.table + seq * a.ld_table;
    // Where the stream's blocks lie in the cache, 32 of them at a time, one a lane (-1: none).
    int place = -1;
    auto look_up = [&](int i) {
        const int k = i + lane / U, sub = (from + mine + k * parts) * U + lane % U, at = a.c.subs(sub), subs = (int)a.c.subs.d;
        const int page = k < chunks && sub * kKv4Block < len ? __ldg(table + at) : -1;
        place = page >= 0 && page < a.n_pages ? (page * a.c.n_k + head) * subs + sub - at * subs : -1;
    };
    auto copy = [&](int i, int slot) {
        if (i % (32 / U) == 0) look_up(i);
        const int at = __shfl_sync(0xffffffffu, place, (i * U + lane) & 31);
        const bool there = lane < U && at >= 0;
        const uint32_t which = __ballot_sync(0xffffffffu, there), bar = smem_u32(&full[bar0 + slot]);
        if (lane == 0) {
            present[bar0 + slot] = which;
            mbar_expect_tx(bar, __popc(which) * kBytes);
        }
        __syncwarp();
        if (there) bulk_g2s(smem_u32(ring + (slot * U + lane) * kBytes), a.c.base + (long long)at * kBytes, kBytes, bar);
    };
    if (group == 0)
        for (int i = 0; i < min(a.slots, chunks); ++i) copy(i, i);
    Rowset set;
    set.begin(a, q0, head, group * 8 * NR, rows);
    const bool live = group * NR * 8 < rows;
    const int past = len - n, open = past + (a.tree ? 0 : 1);          // every row sees the tokens before `open`
    int slot = 0;
    uint32_t phase = 0;
#pragma unroll 1
    for (int i = 0; i < chunks; ++i) {
        mbar_wait(smem_u32(&full[bar0 + slot]), phase, &abort_flag, a.st);
        const uint32_t there = abort_flag || !live ? 0u : present[bar0 + slot];
        const int token = (from + mine + i * parts) * U * kKv4Block;
        const unsigned char* blk = ring + slot * (U * kBytes);
        if (there == (1u << U) - 1 && token + U * kKv4Block <= open) set.template work<U, false>(a, blk, token, q0, past, len, there);
        else if (there) set.template work<U, true>(a, blk, token, q0, past, len, there);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // read here, refilled by a bulk copy
        __syncwarp();
        if (a.row_groups == 1) {
            if (i + a.slots < chunks) copy(i + a.slots, slot);
        } else {
            if (lane == 0) mbar_arrive(smem_u32(&empty[bar0 + slot]));
            // the chunk before this one, which the stream's other warps have left by now, as a rule
            const int last = slot ? slot - 1 : a.slots - 1;
            if (group == 0 && i > 0 && i - 1 + a.slots < chunks) {
                mbar_wait(smem_u32(&empty[bar0 + last]), slot ? phase : phase ^ 1u, &abort_flag, a.st);
                copy(i - 1 + a.slots, last);
            }
        }
        if (++slot == a.slots) { slot = 0; phase ^= 1u; }
    }
    __syncthreads();                                          // every warp is done with the ring
    float* s_out = reinterpret_cast<float*>(kv4_smem);        // [warp][row of its group][D]
    set.end(s_out + warp * 8 * NR * D, s_ml[warp]);
    __syncthreads();
    // the warps of a row group, four columns a thread
    for (int i = threadIdx.x; i < a.row_groups * 8 * NR * (D / 4); i += kKv4Threads) {
        const int row = i / (D / 4), col = (i - row * (D / 4)) * 4;
        const int grp = row / (8 * NR), r = row - grp * 8 * NR;
        if (row >= rows) continue;
        float top = kNegInf;
        for (int w = 0; w < parts; ++w) top = fmaxf(top, s_ml[grp * parts + w][r].x);
        float sum = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int w = 0; w < parts; ++w) {
            const float2 ml = s_ml[grp * parts + w][r];
            if (ml.y == 0.f) continue;                        // saw nothing
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

// Adds up the parts of split caches, in a fixed order: WAYS warps a row and head (each every WAYS-th part), D / 32 columns a lane.
constexpr int kKv4JoinWarps = 4;
template <typename T, int D, int WAYS>
__global__ void __launch_bounds__(kKv4JoinWarps * 32) kv4_join_kernel(const __grid_constant__ Kv4Args a) {
    constexpr int N = D / 32;
    __shared__ float s_o[kKv4JoinWarps][D];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, way = warp % WAYS;
    const int unit = blockIdx.x * (kKv4JoinWarps / WAYS) + warp / WAYS;
    pdl_wait();
    const int node = unit / a.n_q, head = unit - node * a.n_q, seq = node / a.max_q, tok = node - seq * a.max_q;
    int q0 = 0, n = 0;
    if (seq < a.n_seq) kv4_rows_of(a, seq, &q0, &n);
    const bool live = tok < min(n, a.max_q);
    const long long at = (long long)(q0 + tok) * a.n_q + head, step = (long long)a.n_rows * a.n_q;
    constexpr int kMost = WAYS == 1 ? 1 : kKv4MaxSplits / 32;
    float2 ml[kMost];                                         // part 32 i + lane
    float top = kNegInf;
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        const int s = i * 32 + lane;
        ml[i] = live && s < a.splits ? __ldcg(&a.part_ml[s * step + at]) : make_float2(kNegInf, 0.f);
        if (ml[i].y != 0.f) top = fmaxf(top, ml[i].x);        // parts that saw nothing have a sum of 0
    }
    top = warp_max(top);
    float sum = 0.f, o[N] = {};
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        const float f = ml[i].y == 0.f ? 0.f : ml[i].x == top ? 1.f : exp2_fast(ml[i].x - top);
        sum += f * ml[i].y;
        if (i * 32 >= a.splits) break;
#pragma unroll
        for (int j = 0; j < 32 / WAYS; ++j) {
            const int s = i * 32 + j * WAYS + way;
            if (WAYS == 1 && s >= a.splits) break;
            const float g = __shfl_sync(0xffffffffu, f, j * WAYS + way);
            if (s >= a.splits || g == 0.f) continue;
            const float* p = a.part_o + (s * step + at) * D + lane * N;
            if constexpr (N == 4) {
                const float4 v = __ldcg(reinterpret_cast<const float4*>(p));
                o[0] += g * v.x; o[1] += g * v.y; o[2] += g * v.z; o[3] += g * v.w;
            } else {
                const float2 v = __ldcg(reinterpret_cast<const float2*>(p));
                o[0] += g * v.x; o[1] += g * v.y;
            }
        }
    }
    sum = warp_sum(sum);
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    if constexpr (WAYS > 1) {
#pragma unroll
        for (int j = 0; j < N; ++j) s_o[warp][lane * N + j] = o[j];
        __syncthreads();
#pragma unroll
        for (int j = 0; j < N; ++j) {
            o[j] = 0.f;
#pragma unroll
            for (int w = 0; w < WAYS; ++w) o[j] += s_o[w][lane * N + j];
        }
    }
    if (!live || way != 0) return;
    T v[N];
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = Elem<T>::down(o[j] * inv);
    T* out = static_cast<T*>(a.out) + (long long)(q0 + tok) * a.ld_out + head * D + lane * N;
    if constexpr (N == 4) *reinterpret_cast<uint2*>(out) = *reinterpret_cast<const uint2*>(v);
    else *reinterpret_cast<uint32_t*>(out) = *reinterpret_cast<const uint32_t*>(v);
    if (a.lse && lane == 0) a.lse[at] = sum == 0.f ? kNegInf : (top + log2f(sum)) * 0.69314718055994531f;
}

}  // namespace coral

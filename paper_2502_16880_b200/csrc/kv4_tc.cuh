// Attention of many rows (the nodes of draft trees, times the heads of a group) over the 4-bit cache, on the 5th-generation tensor cores: the
// products of prompt_attention.cuh, two tiles of 128 rows a block, with keys and values unpacked by eight warps instead of copied.
//   * a warp brings the packed blocks of 64 tokens a step into a ring of their own, one bulk copy each,
//   * a warp finds the powers of two that bring the step's largest key and value to 2^14..2^15,
//   * eight warps unpack the step to fp16 tiles, low + step code, times those powers.  Keys take two tiles, what fp16 holds and what is
//     left of it, so that scores are exact to fp32's sums (one tile would move them, and with them every weight, by 2^-12 of their
//     terms); values are rounded once, to 2^-12 of themselves,
//   * a thread of the softmax has a row: P = exp2(S c kf - m) in fp16 (for fp16 outputs in two parts), with the step's key power kf in the
//     factor and its value power in the reference m, which so follows the largest score and the largest value; P stays below 2^15 whatever
//     the values' size,
//   * fp16 holds 40 powers of two: where a token's key, or a group of its values, lies so far below a step's or a former step's largest ones (which
//     a row may not even see) that bits of them would be lost, a warp computes each row that meets them again, in fp32 (kt_row_again);
//     also scores beyond kPaFar, and results that are not finite, unless values that the row sees are the only such ones in sight.
// Columns lie in another order than in memory: 0 4 1 5 2 6 3 7 within eight (queries and keys alike, for the sums it is all one), and
// place by place for the values (column 8 i + n at n D / 8 + ...), which the outputs undo.
// 8 sequences x 8 key heads, trees of 60 nodes x 4 heads, 3001 tokens, fp16: 71 us with the join (11 at the tensor cores' measured rate), of which
// the question why a row is not finite costs 0.6; when that took 70, 66 with one part of a weight, 60 with one tile of the keys too, whose log of sums was off by 5e-4 where few tokens are seen.  What bounds it: 64 tokens
// take 3500 cycles, of which the products' operands read shared memory for 2500 (2.5 times those of prompt_attention.cuh, since keys count
// twice), and an unpacking warp is busy all the time, keys 1700 and values 1000 (with one tile of rows it alone sets the 3100 cycles).
#pragma once
#include "kv4.cuh"
#include "prompt_attention.cuh"

namespace coral {

constexpr int kKtUnpack = 8;                       // unpacking warps, eight tokens of a step each
// Registers a thread: 96 at launch (640 threads); the softmax's two warpgroups take what the other three give up.
constexpr int kKtRegsMany = 136, kKtRegsFew = 64;
static_assert(2 * kKtRegsMany + 3 * kKtRegsFew <= 5 * 96, "a split above the launch's registers would wait forever");
constexpr int kKtThreads = (12 + kKtUnpack) * 32;  // warps 0..7 softmax, 8 and 9 MMAs of a tile each, 10 copies, 11 powers, 12.. unpacking
constexpr int kKtRaw = 4;                          // steps of packed tokens in flight
constexpr int kKtBlocks = kPaKeys / kKv4Block;     // blocks of 16 tokens a step
constexpr int kKtPowers = 8;                       // steps whose powers are kept
constexpr int kKtPresent = 16;
// Parts of a weight: what fp16 holds, and for fp16 outputs what is left (bf16's 2^-9 hides a weight's 2^-12).
template <typename T> constexpr int kKtParts = std::is_same_v<T, __half> ? 2 : 1;
template <int D> constexpr int kKtStages = D == 128 ? 7 : 10;
template <int D, int NG> constexpr size_t kt_smem_bytes() {
    return 1024 + (size_t)2 * 128 * D * 2 + (size_t)kKtStages<D> * kPaKeys * D * 2 + (size_t)kKtRaw * kKtBlocks * (kKv4Block * D + 128 * NG);
}

// The largest of |low| and |low + 15 step| (a NaN is passed over), and from it the power of two that undoes the one which brings it to
// 2^14..2^15; that one's bits are kt_inverse's.
template <typename T>
__device__ __forceinline__ float kt_largest(float top, uint32_t pair) {
    const float2 p = kv4_pair<T>(pair);
    return fmaxf(top, fmaxf(fabsf(p.y), fabsf(fmaf(15.f, p.x, p.y))));
}
// Whether a token's key, or a group of its values (which has outputs of its own), whose largest is `own` would lose bits next to `top`: fp16 holds
// 2^-25 of what `top` brings to 2^14 or more, which has to be 2^-22 of the key and 2^-13 of the group.
__device__ __forceinline__ bool kt_lost(float own, float top, bool value) { return own > 0.f && own < top * (value ? 0x1p-26f : 0x1p-17f); }
__device__ __forceinline__ float kt_power(float top) {
    const int e = min(max((int)(__float_as_uint(top) >> 23), 16), 254);
    return __uint_as_float((uint32_t)(e - 14) << 23);
}
__device__ __forceinline__ float kt_inverse(float power) { return __uint_as_float((254u << 23) - __float_as_uint(power)); }
// A word's eight codes as values, pairs (0,4), (1,5), (2,6), (3,7): step and low as fp16 pairs, one rounding.
__device__ __forceinline__ uint4 kt_values(uint32_t w, uint32_t step, uint32_t low) {
    uint32_t r[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t bits = ((k < 2 ? w : w >> 8) & (k & 1 ? 0x00f000f0u : 0x000f000fu)) | 0x64006400u;    // 1024 + code, or + 16 code
        uint32_t code;
        if (k & 1) asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(code) : "r"(bits), "r"(0x2c002c00u), "r"(0xd400d400u));     // / 16 - 64
        else asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(code) : "r"(bits), "r"(0x64006400u));
        asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r[k]) : "r"(code), "r"(step), "r"(low));
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
}
// The same in fp32, as what fp16 holds of them and the rest.
struct KtTwo {
    uint4 high, rest;
};
__device__ __forceinline__ KtTwo kt_values_two(uint32_t w, unsigned long long step, unsigned long long low) {
    uint32_t h[4], l[4];
    constexpr uint32_t kBits = 0x4b000000u;         // 2^23: a code in its lowest bits becomes a number without a conversion
    const unsigned long long less = pair_of(-8388608.f, -8388608.f), minus = pair_of(-1.f, -1.f);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const unsigned long long code = add2(pair_of(__uint_as_float((w >> (4 * k) & 15u) | kBits), __uint_as_float((w >> (4 * k + 16) & 15u) | kBits)), less);
        const unsigned long long v = fma2(code, step, low);
        const float2 f = halves(v);
        h[k] = half_pair(f.x, f.y);
        const float2 held = kv4_pair<__half>(h[k]), rest = halves(fma2(pair_of(held.x, held.y), minus, v));
        l[k] = half_pair(rest.x, rest.y);
    }
    return KtTwo{make_uint4(h[0], h[1], h[2], h[3]), make_uint4(l[0], l[1], l[2], l[3])};
}
// Where chunk `chunk` (eight columns) of row `row` lies in a tile of `rows` rows, 64 columns a part, 128-byte swizzle.
__device__ __forceinline__ uint32_t kt_chunk(int row, int chunk, int rows) { return (chunk >> 3) * rows * 128 + row * 128 + ((chunk ^ row) & 7) * 16; }

// Tokens `from` to `len` of a row, by a warp in fp32, from the packed tokens that it sees: the reference m (a power of two), the sum of the weights
// 2^(score - m), and the weighted sum of the values, D / 32 columns a lane.  ASK: only if it is not values that the row sees, and no others, that
// are not finite (false: what the row has is right).
template <typename T, int D, int NG>
__device__ __forceinline__ bool kt_row_again(const Kv4Args& a, bool ask, const int32_t* table, int head, const T* q, int from, int len, int past, int node,
                                          unsigned long long tree, float* m, float* sum, float* acc) {
    const int lane = threadIdx.x & 31;
    constexpr int N = D / 32;
    // where the block of token j lies (-1: there is none, or it is not seen)
    auto seen = [&](int j) {
        const int at = j - past;
        return j < len && (at < 0 || (a.tree ? at < kKv4MaxTree && tree >> at & 1ull : at <= node));
    };
    auto block_of = [&](int j) -> long long {
        const int sub = j / kKv4Block, per = (int)a.c.subs.d, page_at = a.c.subs(sub), page = __ldg(table + page_at);
        if (page < 0 || page >= a.n_pages) return -1;
        return (((long long)page * a.c.n_k + head) * per + sub - page_at * per) * (kKv4Block * D + 128 * NG);
    };
    if (ask) {
        // 1: a value that the row sees is not finite, 2: one that it does not
        auto bad = [&](int j) {
            const long long block = j < len ? block_of(j) : -1;
            if (block < 0) return 0;
            float odd = 0.f;
            for (int g = 0; g < NG; ++g) odd = fmaf(0.f, kv4_pair<T>(reinterpret_cast<const uint32_t*>(a.c.base + block + 16 * D)[(NG + g) * 16 + (j & 15)]).y, odd);
            return odd == 0.f ? 0 : seen(j) ? 1 : 2;
        };
        int found = 0;
        for (int j = max(from, past); j < len; j += 32) found |= bad(j + lane);
        found = __reduce_or_sync(0xffffffffu, found);
        for (int j = from; !found && j < min(past, len); j += 32) found = __any_sync(0xffffffffu, j + lane < past && bad(j + lane));
        if (found == 1) return false;
    }
    // this lane's token j: its score
    auto score = [&](int j, long long* block) {
        *block = seen(j) ? block_of(j) : -1;
        if (*block < 0) return kNegInf;
        const unsigned char* blk = a.c.base + *block;
        float s = 0.f;
        for (int c = 0; c < D; ++c) {
            const float2 pr = kv4_pair<T>(reinterpret_cast<const uint32_t*>(blk + 16 * D)[c * NG / D * 16 + (j & 15)]);
            const uint32_t w = *reinterpret_cast<const uint32_t*>(blk + ((j & 15) * 4 + (c >> 3 & 3)) * (D / 8) + 4 * (c >> 5));
            s = fmaf(Elem<T>::up(q[c]), fmaf((float)(w >> (4 * (c & 7)) & 15u), pr.x, pr.y), s);
        }
        return __fmul_rn(s, a.scale2);                         // rounded once for the maximum and the weight, whatever its size
    };
    long long block;
    float top = kNegInf;
    for (int j = from + lane; j < len; j += 32) top = fmaxf(top, score(j, &block));
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (top == kNegInf) top = 0.f;
    float all = 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e) acc[e] = 0.f;
    for (int j0 = from; j0 < len; j0 += 32) {
        const float s = score(j0 + lane, &block);
        const float p = block >= 0 ? exp2_fast(s - top) : 0.f;
        all += p;
        for (uint32_t todo = __ballot_sync(0xffffffffu, block >= 0); todo; todo &= todo - 1) {
            const int i = __ffs(todo) - 1, t = (j0 + i) & 15;
            const float w = __shfl_sync(0xffffffffu, p, i);
            const unsigned char* blk = a.c.base + __shfl_sync(0xffffffffu, block, i);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const int c = lane * N + e, n = c & 7, k = c >> 3;
                const float2 pr = kv4_pair<T>(reinterpret_cast<const uint32_t*>(blk + 16 * D)[(NG + c * NG / D) * 16 + t]);
                const uint16_t piece = reinterpret_cast<const uint16_t*>(blk + 8 * D + (t >> 3) * (4 * D) + (n * 4 + ((t & 7) >> 1)) * (D / 8) + 4 * (k >> 2))[t & 1];
                acc[e] = fmaf(w, fmaf((float)(piece >> (4 * (k & 3)) & 15u), pr.x, pr.y), acc[e]);
            }
        }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
    *m = top;
    *sum = all;
    return true;
}

// The rows of a warp that are to be computed again: those of `todo`, without a question those of `lost`.  Tokens from .. to of this block's part.
template <typename T, int D, int NG>
__device__ __noinline__ void kt_rows_again(const Kv4Args& a, uint32_t todo, uint32_t lost, const int32_t* table, int head, int split, int q0, int tok, int q_head,
                                           unsigned long long tree, int from, int to, int past) {
    const int lane = threadIdx.x & 31;
    const bool whole = a.splits == 1;
    for (; todo; todo &= todo - 1) {
        const int r = __ffs(todo) - 1, tok_r = __shfl_sync(0xffffffffu, tok, r), head_r = __shfl_sync(0xffffffffu, q_head, r);
        const unsigned long long tree_r = __shfl_sync(0xffffffffu, tree, r);
        float acc[D / 32], m, sum;
        if (!kt_row_again<T, D, NG>(a, !(lost >> r & 1u), table, head, static_cast<const T*>(a.q) + (q0 + tok_r) * a.ld_q + (long long)head_r * D, from, to, past, tok_r,
                                    tree_r, &m, &sum, acc))
            continue;
        const long long at = (long long)(q0 + tok_r) * a.n_q + head_r, part = (long long)split * a.n_rows * a.n_q + at;
#pragma unroll
        for (int e = 0; e < D / 32; ++e) {
            if (whole) static_cast<T*>(a.out)[(long long)(q0 + tok_r) * a.ld_out + (long long)head_r * D + lane * (D / 32) + e] = Elem<T>::down(sum == 0.f ? 0.f : acc[e] / sum);
            else a.part_o[part * D + lane * (D / 32) + e] = acc[e];
        }
        if (lane == 0) {
            if (!whole) a.part_ml[part] = make_float2(sum == 0.f ? kKv4NoMax : m, sum);
            else if (a.lse) a.lse[at] = sum == 0.f ? kNegInf : (m + log2f(sum)) * 0.69314718055994531f;
        }
    }
}

template <typename T, int D, int NG>
__global__ void __launch_bounds__(kKtThreads, 1) kv4_many_kernel(const __grid_constant__ Kv4Args a) {
    constexpr int STAGES = kKtStages<D>, kTile = 128 * D * 2, kStep = kPaKeys * D * 2, kBytes = kKv4Block * D + 128 * NG, W = D / 32, DB = D / 64;
    constexpr int PARTS = kKtParts<T>;
    extern __shared__ unsigned char kt_smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(kt_smem_raw) + 1023) & ~(uintptr_t)1023);
    unsigned char *s_kv = smem + 2 * kTile, *s_raw = s_kv + STAGES * kStep;
    __shared__ __align__(8) uint64_t q_full, kv_full[STAGES], kv_empty[STAGES], s_full[4], p_full[4], pv_done[4];
    __shared__ __align__(8) uint64_t raw_full[kKtRaw], raw_empty[kKtRaw], power_full[kKtPowers];
    __shared__ uint32_t present[kKtPresent];
    __shared__ float2 s_power[kKtPowers];                     // of a step's keys and values
    __shared__ uint32_t s_lost[kKtPowers];                    // not 0: some of the step's tokens are too far below its largest
    __shared__ uint32_t tmem_slot;
    __shared__ volatile int abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        mbar_init(smem_u32(&q_full), 8);
        for (int i = 0; i < STAGES; ++i) {
            mbar_init(smem_u32(&kv_full[i]), kKtUnpack);
            mbar_init(smem_u32(&kv_empty[i]), 2);
        }
        for (int i = 0; i < 4; ++i) {
            mbar_init(smem_u32(&s_full[i]), 1);
            mbar_init(smem_u32(&p_full[i]), 4);
            mbar_init(smem_u32(&pv_done[i]), 1);
        }
        for (int i = 0; i < kKtRaw; ++i) {
            mbar_init(smem_u32(&raw_full[i]), 1);
            mbar_init(smem_u32(&raw_empty[i]), kKtUnpack);
        }
        for (int i = 0; i < kKtPowers; ++i) mbar_init(smem_u32(&power_full[i]), 1);
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
    int q0, n_q;
    kv4_rows_of(a, seq, &q0, &n_q);
    const int rows = min(n_q, a.max_q) * a.G, row0 = row_block * 256;
    if (row0 >= rows) return;
    if (warp == 8) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    const int len = (int)max(0LL, min((long long)a.lens[seq], min((long long)a.width * a.c.page, 0x7fff0000LL)));
    const int spans = (len + kKv4SpanBlocks * kKv4Block - 1) / (kKv4SpanBlocks * kKv4Block), per = (spans + a.splits - 1) / a.splits;
    constexpr int kPer = kKv4SpanBlocks / kKtBlocks;               // steps of a span
    const int step0 = min(split * per, spans) * kPer, steps = min(min(min(split * per, spans) + per, spans) * kPer, (len + kPaKeys - 1) / kPaKeys) - step0;
    const int past = len - n_q, open = past + (a.tree ? 0 : 1);    // every row sees the tokens before `open`
    const int n0 = max(steps, 0), n1 = rows - row0 > 128 ? n0 : 0, n = n0;
    const int32_t* table = a.table + seq * a.ld_table;

    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kKtRegsMany));
        const int t = warp >> 2, local = (warp & 3) * 32 + lane, row = row0 + t * 128 + local, nt = t ? n1 : n0;
        const bool live = row < rows;
        const int tok = live ? row / a.G : 0, q_head = head * a.G + row - tok * a.G;
        // The warp's 32 rows of operand A, D / 8 threads a row: scaled by a power of two, turned round where the scale is negative.
        float c = 0.f, c_b = 0.f;                              // this thread's row: from a raw score to powers of two, in two factors
        {
            constexpr int L = D / 8, kRows = 32 / L;           // threads a row, rows at a time
            const int l = lane % L, first = row0 + t * 128 + (warp & 3) * 32;
            const float sign = a.scale2 < 0.f ? -1.f : 1.f;
            uint32_t raws[8][4];
#pragma unroll 1
            for (int i0 = 0; i0 < L; i0 += 8) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int r = first + (i0 + i) * kRows + lane / L, tk = r / a.G;
#pragma unroll
                    for (int k = 0; k < 4; ++k) raws[i][k] = 0;
                    if (r < rows)
                        *reinterpret_cast<uint4*>(raws[i]) = *reinterpret_cast<const uint4*>(static_cast<const T*>(a.q) + (q0 + tk) * a.ld_q + (long long)(head * a.G + r - tk * a.G) * D + 8 * l);
                }
#pragma unroll
                for (int ii = 0; ii < 8; ++ii) {
                    const int i = i0 + ii, at = i * kRows + lane / L;
                    const uint32_t (&raw)[4] = raws[ii];
                    float f[8];
                    uint32_t big = 0;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float2 x = kv4_pair<T>(raw[k]);
                        f[2 * k] = x.x;
                        f[2 * k + 1] = x.y;
                        big = max(big, max(__float_as_uint(x.x) & 0x7fffffffu, __float_as_uint(x.y) & 0x7fffffffu));
                    }
#pragma unroll
                    for (int o = 1; o < L; o <<= 1) big = max(big, __shfl_xor_sync(0xffffffffu, big, o));
                    const int e = q4_exponent(big), mine = __shfl_sync(0xffffffffu, e, lane % kRows * L);
                    const Q4Power up(e), down(-mine);
                    if (lane / kRows == i) {
                        c = fabsf(a.scale2) * down.a;
                        c_b = down.b;
                    }
#pragma unroll
                    for (int k = 0; k < 8; ++k) f[k] = up(f[k]) * sign;
                    *reinterpret_cast<uint4*>(smem + t * kTile + kt_chunk((warp & 3) * 32 + at, l, 128)) =
                        make_uint4(half_pair(f[0], f[4]), half_pair(f[1], f[5]), half_pair(f[2], f[6]), half_pair(f[3], f[7]));
                }
            }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");           // written here, read by the MMAs
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&q_full));

        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t ts = tmem + t * 128 + lanes, to = tmem + 256 + t * 128 + lanes;
        const unsigned long long tree = a.tree && live ? __ldg(a.tree + q0 + tok) : 0ull;
        float m = kNegInf, mc = 0.f;                           // largest score that moved the reference, and the reference: 2^7 below it
        int vtop = -1000;                                      // exponent of the largest power of the values: O is in its units
        bool lost = false;
        unsigned long long sum2 = 0;
        float s[kPaKeys];
        uint32_t* sr = reinterpret_cast<uint32_t*>(s);
        for (int j = 0; j < nt; ++j) {
            const int buf = j & 1, slot = j % kKtPowers, base = (step0 + j) * kPaKeys;
            pa_wait(smem_u32(&power_full[slot]), (uint32_t)(j / kKtPowers) & 1u, &abort_flag, a.st);
            pa_wait(smem_u32(&s_full[t * 2 + buf]), (uint32_t)(j >> 1) & 1u, &abort_flag, a.st);
            __syncwarp();
            tc_fence_after();
            const uint32_t at = ts + buf * kPaKeys;
            pa_ld32(at, sr);
            pa_ld32(at + 32, sr + 32);
            const float2 power = s_power[slot];
            lost |= s_lost[slot] != 0;
            const uint32_t there = present[j % kKtPresent];
            pa_ld_wait();
            if (base + kPaKeys > open || there != (1u << kKtBlocks) - 1) {
                // which tokens of the step this row sees
                unsigned long long see = 0;
#pragma unroll
                for (int b = 0; b < kKtBlocks; ++b)
                    if (there >> b & 1u) see |= 0xffffull << (16 * b);
                const int d = past - base;                     // tokens in front of the query tokens
                const unsigned long long own = a.tree ? tree : tok >= 63 ? ~0ull : (2ull << tok) - 1;
                if (a.tree) {
                    if (d < 64) see &= d > 0 ? ((1ull << d) - 1) | own << d : d > -64 ? own >> -d : 0ull;
                } else {
                    const int upto = d + tok + 1;              // tokens from the step's first on
                    if (upto < 64) see &= upto > 0 ? (1ull << upto) - 1 : 0ull;
                }
                if (len - base < 64) see &= len > base ? (1ull << (len - base)) - 1 : 0ull;
#pragma unroll
                for (int i = 0; i < kPaKeys; ++i) s[i] = see >> i & 1ull ? s[i] : kNegInf;
            }
            float m4[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
            for (int i = 4; i < kPaKeys; i += 8)
#pragma unroll
                for (int e = 0; e < 4; ++e) m4[e] = i + 4 + e < kPaKeys ? pa_max3(m4[e], s[i + e], s[i + 4 + e]) : fmaxf(m4[e], s[i + e]);
            const float top = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
            const float cj = fmaxf(c * power.x * c_b, 0x1p-126f), peak = top * cj;      // not zero: -inf stays what it is
            const bool moves = peak > (m == kNegInf ? 0.f : m) + 8.f || (m == kNegInf && top > kNegInf);
            const int v_now = (int)(__float_as_uint(power.y) >> 23) - 127;
            if (__any_sync(0xffffffffu, moves) || v_now > vtop) {
                const float next = moves ? peak : m, next_c = (next == kNegInf ? 0.f : next) - 7.f;
                lost |= fabsf(next_c) > kPaFar || (vtop > -1000 && v_now > vtop + 10);
                const float by = m == kNegInf ? 0.f : exp2_fast(mc - next_c), f = v_now > vtop ? by * exp2_fast((float)max(vtop - v_now, -252)) : by;
                m = next;
                mc = next_c;
                vtop = max(vtop, v_now);
                sum2 = mul2(sum2, pair_of(by, by));
                if (j > 0) {                                   // O, once the step before is in it
                    pa_wait(smem_u32(&pv_done[t * 2 + (buf ^ 1)]), (uint32_t)((j - 1) >> 1) & 1u, &abort_flag, a.st);
                    __syncwarp();
                    tc_fence_after();
#pragma unroll 1
                    for (int b = 0; b < 2 * DB; ++b) {
                        uint32_t o[32];
                        pa_ld32(to + b * 32, o);
                        pa_ld_wait();
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                        pa_st32(to + b * 32, o);
                    }
                    pa_st_wait();
                }
            }
            // The weights with the step's power of the values in O's units, and their sum without it: fp16 holds weights down to 2^-25, which
            // with ten powers below the largest values still is 2^-22 of the largest weight.
            const int below = vtop - v_now, shift = max(-below, -40);
            lost |= below > 10;
            const float ref = (float)shift - mc, undo = exp2_int(-shift);
            const unsigned long long c2 = pair_of(cj, cj), m2 = pair_of(ref, ref);
            unsigned long long here = 0;
            const unsigned long long minus = pair_of(-1.f, -1.f);
            uint32_t p[kPaKeys / 2 * PARTS];
#pragma unroll
            for (int i = 0; i < kPaKeys / 2; ++i) {
                const float2 x = halves(fma2(pair_of(s[2 * i], s[2 * i + 1]), c2, m2));
                const float lo = pa_exp2(x.x), hi = pa_exp2(x.y);
                const unsigned long long both = pair_of(lo, hi);
                here = add2(here, both);
                p[i] = half_pair(lo, hi);
                if constexpr (PARTS == 2) {
                    const float2 held = kv4_pair<__half>(p[i]), rest = halves(fma2(pair_of(held.x, held.y), minus, both));
                    p[kPaKeys / 2 + i] = half_pair(rest.x, rest.y);
                }
            }
            sum2 = fma2(here, pair_of(undo, undo), sum2);
            pa_st32(at, p);
            if constexpr (PARTS == 2) pa_st32(at + 32, p + 32);
            pa_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&p_full[t * 2 + buf]));
        }
        const float2 sums = halves(sum2);
        const float sum = sums.x + sums.y;
        const bool whole = a.splits == 1;
        const float inv = sum == 0.f ? 0.f : whole ? 1.f / sum : 1.f;
        const Q4Power units(nt > 0 ? vtop : 0);
        if (nt > 0) {
            pa_wait(smem_u32(&pv_done[t * 2 + ((nt - 1) & 1)]), (uint32_t)((nt - 1) >> 1) & 1u, &abort_flag, a.st);
            __syncwarp();
            tc_fence_after();
        }
        const long long at = (long long)(q0 + tok) * a.n_q + q_head, part = (long long)split * a.n_rows * a.n_q + at;
        T* out = static_cast<T*>(a.out) + (long long)(q0 + tok) * a.ld_out + (long long)q_head * D;
        float* part_o = a.part_o + part * D;
        float odd = 0.f;                                       // NaN where a result is not finite
        // 32 places of the values: column 8 i + n stands at place n D / 8 + 8 (i / 8) + (0 2 4 6 1 3 5 7 for i % 8)
        constexpr int kPlaces = D / 8, kCols = 32 / kPlaces;   // columns n side by side in 32 places (2 or 4)
#pragma unroll
        for (int b = 0; b < 2 * DB; ++b) {
            uint32_t o[32];
            if (nt > 0) {
                pa_ld32(to + b * 32, o);
                pa_ld_wait();
            }
#pragma unroll
            for (int i = 0; i < kPlaces; ++i) {
                float x[kCols];
#pragma unroll
                for (int k = 0; k < kCols; ++k) {
                    x[k] = sum == 0.f ? 0.f : units(__uint_as_float(o[k * kPlaces + (i & ~7) + ((i & 3) * 2 + (i >> 2 & 1))])) * inv;
                    odd = fmaf(x[k], 0.f, odd);
                }
                const int col = 8 * i + b * kCols;
                if (!live) continue;
                if (!whole) {
                    if constexpr (kCols == 2) *reinterpret_cast<float2*>(part_o + col) = make_float2(x[0], x[1]);
                    else *reinterpret_cast<float4*>(part_o + col) = make_float4(x[0], x[1], x[2], x[3]);
                } else {
                    T v[kCols];
#pragma unroll
                    for (int k = 0; k < kCols; ++k) v[k] = Elem<T>::down(x[k]);
                    if constexpr (kCols == 2) *reinterpret_cast<uint32_t*>(out + col) = *reinterpret_cast<const uint32_t*>(v);
                    else *reinterpret_cast<uint2*>(out + col) = *reinterpret_cast<const uint2*>(v);
                }
            }
        }
        if (live && !whole) a.part_ml[part] = make_float2(sum == 0.f ? kKv4NoMax : mc, sum);
        if (live && whole && a.lse) a.lse[at] = sum == 0.f ? kNegInf : (mc + log2f(sum)) * 0.69314718055994531f;
        // Rows of finite weights whose result is not (values that they do not see may be the reason), and those that met tokens far apart.
        const bool again = live && (lost || (sum > 0.f && sum < __int_as_float(0x7f800000) && odd != 0.f));
        __syncwarp();
        if (__any_sync(0xffffffffu, again))
            kt_rows_again<T, D, NG>(a, __ballot_sync(0xffffffffu, again), __ballot_sync(0xffffffffu, lost), table, head, split, q0, tok, q_head, tree, step0 * kPaKeys,
                                    min(len, (step0 + n) * kPaKeys), past);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kKtRegsFew));
        if (warp == 10) {
            int place = -1;
            for (int j = 0; j < n; ++j) {
                // where the blocks of eight steps lie in the cache, one a lane (-1: none)
                if (j % 8 == 0) {
                    const int sub = (step0 + j) * kKtBlocks + lane, at = a.c.subs(sub), subs = (int)a.c.subs.d;
                    const int page = sub * kKv4Block < len ? __ldg(table + at) : -1;
                    place = page >= 0 && page < a.n_pages ? (page * a.c.n_k + head) * subs + sub - at * subs : -1;
                }
                const int at = __shfl_sync(0xffffffffu, place, (j % 8) * kKtBlocks + lane % kKtBlocks), slot = j % kKtRaw;
                const bool there = lane < kKtBlocks && at >= 0;
                const uint32_t which = __ballot_sync(0xffffffffu, there), bar = smem_u32(&raw_full[slot]);
                pa_wait(smem_u32(&raw_empty[slot]), ((uint32_t)(j / kKtRaw) & 1u) ^ 1u, &abort_flag, a.st);
                __syncwarp();
                if (lane == 0) {
                    present[j % kKtPresent] = which;
                    mbar_expect_tx(bar, __popc(which) * kBytes);
                }
                __syncwarp();
                if (there) bulk_g2s(smem_u32(s_raw + (slot * kKtBlocks + lane) * kBytes), a.c.base + (long long)at * kBytes, kBytes, bar);
            }
            // nothing is left on its way when the block ends, an expired wait elsewhere included
            for (int j = max(0, n - kKtRaw); j < n; ++j) pa_wait(smem_u32(&raw_full[j % kKtRaw]), (uint32_t)(j / kKtRaw) & 1u, &abort_flag, a.st);
        } else if (warp == 11) {
            float before = 0x1p-14f;                           // values of nothing but zeros take the power of the step before
            for (int j = 0; j < n; ++j) {
                const int slot = j % kKtRaw;
                pa_wait(smem_u32(&raw_full[slot]), (uint32_t)(j / kKtRaw) & 1u, &abort_flag, a.st);
                const uint32_t there = present[j % kKtPresent];
                float top_k[2] = {0.f, 0.f}, top_v[2] = {0.f, 0.f}, least_v = 3.4e38f;      // least_v: of groups, zeros aside
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int token = lane + 32 * i;
                    const uint32_t* pairs = reinterpret_cast<const uint32_t*>(s_raw + (slot * kKtBlocks + (token >> 4)) * kBytes + 16 * D) + (token & 15);
                    if (!(there >> (token >> 4) & 1u) || (step0 + j) * kPaKeys + token >= len) continue;
#pragma unroll
                    for (int g = 0; g < NG; ++g) {
                        top_k[i] = kt_largest<T>(top_k[i], pairs[g * 16]);
                        const float own = kt_largest<T>(0.f, pairs[(NG + g) * 16]);
                        top_v[i] = fmaxf(top_v[i], own);
                        if (own > 0.f) least_v = fminf(least_v, own);
                    }
                }
                const float all_k = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(fmaxf(top_k[0], top_k[1]))));
                const float all_v = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(fmaxf(top_v[0], top_v[1]))));
                const uint32_t lost = __ballot_sync(0xffffffffu, kt_lost(top_k[0], all_k, false) || kt_lost(top_k[1], all_k, false) ||
                                                                     kt_lost(least_v, all_v, true));
                if (all_v > 0.f) before = kt_power(all_v);
                if (lane == 0) {
                    s_power[j % kKtPowers] = make_float2(kt_power(all_k), before);
                    s_lost[j % kKtPowers] = lost;
                    mbar_arrive(smem_u32(&power_full[j % kKtPowers]));
                }
            }
        } else if (warp >= 12) {
            const int g8 = warp - 12, b = g8 >> 1, h = g8 & 1, hi = lane >> 2, lo = lane & 3;     // this warp's eight tokens of a step
            int stage = 0;
            uint32_t phase = 0;
            auto unpack = [&](int j, auto values) {
                constexpr bool V = decltype(values)::value;
                const int slot = j % kKtRaw, base = (step0 + j) * kPaKeys + g8 * 8;
                // (the warp of the powers has waited for the packed tokens)
                if (!V) pa_wait(smem_u32(&power_full[j % kKtPowers]), (uint32_t)(j / kKtPowers) & 1u, &abort_flag, a.st);
                const float2 power = s_power[j % kKtPowers];
                const float up = kt_inverse(V ? power.y : power.x);
                const int real = present[j % kKtPresent] >> b & 1u ? len - base : 0;      // tokens of the eight that there are
                unsigned char* tile = s_kv + stage * kStep;
                const unsigned char* blk = s_raw + (slot * kKtBlocks + b) * kBytes;
                const uint32_t* pairs = reinterpret_cast<const uint32_t*>(blk + 16 * D) + h * 8 + (V ? NG * 16 : 0);
                const unsigned char* at = blk + (V ? 8 * D : 0) + h * 4 * D + lane * (D / 8);
                uint32_t w[W];
                if constexpr (D == 128) *reinterpret_cast<uint4*>(w) = *reinterpret_cast<const uint4*>(at);
                else *reinterpret_cast<uint2*>(w) = *reinterpret_cast<const uint2*>(at);
                if constexpr (!V) {
                    // token hi, chunks 4 k + lo, in two tiles
                    unsigned long long step[NG], low[NG];
#pragma unroll
                    for (int i = 0; i < NG; ++i) {
                        const float2 p = kv4_pair<T>(hi < real ? pairs[i * 16 + hi] : 0u);
                        step[i] = pair_of(p.x * up, p.x * up);
                        low[i] = pair_of(p.y * up, p.y * up);
                    }
                    const int after = stage + 1 == STAGES ? 0 : stage + 1;
                    // (stages get free in their order)
                    pa_wait(smem_u32(&kv_empty[after]), after ? phase ^ 1u : phase, &abort_flag, a.st);
#pragma unroll
                    for (int k = 0; k < W; ++k) {
                        const KtTwo v = kt_values_two(w[k], step[k * NG / W], low[k * NG / W]);
                        const uint32_t at_chunk = kt_chunk(g8 * 8 + hi, 4 * k + lo, kPaKeys);
                        *reinterpret_cast<uint4*>(tile + at_chunk) = v.high;
                        *reinterpret_cast<uint4*>(s_kv + after * kStep + at_chunk) = v.rest;
                    }
                } else {
                    // place hi of tokens 2 lo and 2 lo + 1
                    uint32_t step[2][W / 2], low[2][W / 2];
#pragma unroll
                    for (int s = 0; s < 2; ++s)
#pragma unroll
                        for (int k = 0; k < W; k += 2) {
                            const bool on = 2 * lo + s < real;
                            const float2 p = kv4_pair<T>(on ? pairs[k * NG / W * 16 + 2 * lo + s] : 0u), q = kv4_pair<T>(on ? pairs[(k + 1) * NG / W * 16 + 2 * lo + s] : 0u);
                            step[s][k / 2] = half_pair(p.x * up, q.x * up);
                            low[s][k / 2] = half_pair(p.y * up, q.y * up);
                        }
                    pa_wait(smem_u32(&kv_empty[stage]), phase ^ 1u, &abort_flag, a.st);
#pragma unroll
                    for (int s = 0; s < 2; ++s)
#pragma unroll
                        for (int k = 0; k < W; k += 2)
                            *reinterpret_cast<uint4*>(tile + kt_chunk(g8 * 8 + 2 * lo + s, hi * (W / 2) + k / 2, kPaKeys)) =
                                kt_values(__byte_perm(w[k], w[k + 1], s ? 0x7632 : 0x5410), step[s][k / 2], low[s][k / 2]);
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // written here, read by the MMAs
                __syncwarp();
#pragma unroll
                for (int i = 0; i < (V ? 1 : 2); ++i) {
                    if (lane == 0) mbar_arrive(smem_u32(&kv_full[stage]));
                    if (++stage == STAGES) { stage = 0; phase ^= 1u; }
                }
                if (V && lane == 0) mbar_arrive(smem_u32(&raw_empty[slot]));
            };
            if (n > 0) unpack(0, std::false_type{});
            if (n > 1) unpack(1, std::false_type{});
            for (int j = 0; j < n; ++j) {
                unpack(j, std::true_type{});
                if (j + 2 < n) unpack(j + 2, std::false_type{});
            }
        } else if (warp == 8 || warp == 9) {
            // the MMAs of tile t, as in prompt_attention_kernel
            const int t = warp - 8, nt = t ? n1 : n0;
            constexpr uint32_t kBase = (1u << 4) | (8u << 24);
            constexpr uint32_t idesc_s = kBase | ((uint32_t)(kPaKeys / 8) << 17), idesc_o = kBase | (1u << 16) | ((uint32_t)(D / 8) << 17);
            const uint32_t q = pa_desc_k(smem_u32(smem) + t * kTile), kv = smem_u32(s_kv), ts = tmem + t * 128, to = tmem + 256 + t * 128;
            int stage = 0;
            uint32_t phase = 0;
            auto full = [&]() { pa_wait(smem_u32(&kv_full[stage]), phase, &abort_flag, a.st); };
            auto next = [&]() {
                if (++stage == STAGES) { stage = 0; phase ^= 1u; }
            };
            auto scores = [&](int j) {                             // S = Q K^T of step j, over both tiles of the keys
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    full();
                    if (j < nt) {
                        tc_fence_after();
                        if (pa_elect()) {
                            const uint32_t k = pa_desc_k(kv + stage * kStep), to_s = ts + (j & 1) * kPaKeys;
                            if (i == 0) pa_mma_ss<false>(to_s, q, k, idesc_s);
                            else pa_mma_ss<true>(to_s, q, k, idesc_s);
#pragma unroll
                            for (int kk = 1; kk < DB * 4; ++kk) pa_mma_ss<true>(to_s, q + (kk >> 2) * (kPaRows / 16) + (kk & 3) * 2, k + (kk >> 2) * (kPaBlock / 16) + (kk & 3) * 2, idesc_s);
                            if (i == 1) tc_commit(smem_u32(&s_full[t * 2 + (j & 1)]));
                            tc_commit(smem_u32(&kv_empty[stage]));
                        }
                    } else if (lane == 0) {
                        mbar_arrive(smem_u32(&kv_empty[stage]));
                    }
                    next();
                }
            };
            if (n > 0) pa_wait(smem_u32(&q_full), 0, &abort_flag, a.st);
            if (n > 0) scores(0);
            if (n > 1) scores(1);
            for (int j = 0; j < n; ++j) {
                full();
                if (j < nt) {
                    const int buf = j & 1;
                    pa_wait(smem_u32(&p_full[t * 2 + buf]), (uint32_t)(j >> 1) & 1u, &abort_flag, a.st);
                    tc_fence_after();
                    if (pa_elect()) {
                        const uint32_t v = pa_desc_n(kv + stage * kStep), p = ts + buf * kPaKeys;
                        if (j == 0) pa_mma_ts<false>(to, p, v, idesc_o);
                        else pa_mma_ts<true>(to, p, v, idesc_o);
#pragma unroll
                        for (int kk = 1; kk < PARTS * (kPaKeys / 16); ++kk) pa_mma_ts<true>(to, p + kk * 8, v + kk % (kPaKeys / 16) * 128, idesc_o);
                        tc_commit(smem_u32(&pv_done[t * 2 + buf]));
                        tc_commit(smem_u32(&kv_empty[stage]));
                    }
                } else if (lane == 0) {
                    mbar_arrive(smem_u32(&kv_empty[stage]));
                }
                next();
                if (j + 2 < n) scores(j + 2);
            }
            if (nt > 0) pa_wait(smem_u32(&pv_done[t * 2 + ((nt - 1) & 1)]), (uint32_t)((nt - 1) >> 1) & 1u, &abort_flag, a.st);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 8) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
    pdl_launch_dependents();
}

}  // namespace coral

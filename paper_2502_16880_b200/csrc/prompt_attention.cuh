// Attention over whole prompts on the 5th-generation tensor cores: packed sequences, causal, grouped heads.  For query i of a
// sequence with Lq queries and Lk keys (the queries stand at its end), and query head h with key head h / G:
//   out = sum_j softmax_j(scale q . k_j) v_j,  j <= i + Lk - Lq;   lse = log-sum-exp of scale q . k_j
// in one pass over the keys (running maximum and sum).
//
// A block takes two tiles of 128 rows: a row is a token and a query head, Gp heads (a power of two) of a group next to one another, so
// that few tokens fill a tile too.  Both tiles read the same keys and values, 64 at a time, through a ring filled by TMA.
//   S = Q K^T           operands in shared memory, sums in tensor memory (two buffers of 64 columns a tile)
//   P = exp2(S - max)   by four warps a tile, a thread a row, back into tensor memory over S as 16-bit values
//   O += P V            operand A from tensor memory, V as it lies (N-major); sums stay in tensor memory
// With two buffers a tile's warps do their exponentials while the tensor cores take the step before (its P V, then the scores
// of the step after the next into the same buffer).  Each tile has its own thread that issues MMAs.  The maximum is a
// reference that moves only when a score passes it by 2^8 (P stays below 2^8, its sum is fp32), so O is scaled in place a few times
// a row at most, by the softmax warps themselves, and nothing else touches it before the end.
// Masked scores are -inf before anything is computed of them; but a value row with an infinity or a NaN would reach every row of
// the tile through 0 * inf.  What stands behind a sequence is made zero in shared memory; for the sequence's own, rows whose result is not
// finite although their sum is are computed again by a warp each, over the keys that they see, unless that is what the values they see
// make of it; so are those of scores beyond kPaFar.  That takes as long as there are keys, so it comes when the block's turns are over and
// no warp waits any more (the waits are bounded).
// Weights are rounded to the type for their product (operand A is 16 bits wide; a second part of what is left would be half as many products
// again): outputs are off by 2.0e-3 of their norm in bf16 and 2.9e-4 in fp16, by 1.5e-3 and 2.1e-4 with fp32 weights, their own rounding.
// 8192 tokens, 32 query and 8 key heads of 128, bf16: 536 to 556 us by the power limit, 1.0 PFLOP/s or 59 to 61 % of the measured product rate
// (470 us on one box that held its clocks; there it was 626 with steps of 128 keys and one buffer, 504 with 64 and two, 470 with the longest
// pairs of tiles first on as many blocks as there are SMs and the next pair's operands loaded ahead).  What bounds it: a step of both tiles
// takes 1640 cycles, in which the products read operands from shared memory for 1300 and the exponentials issue for 1100; either alone would
// be faster.
#pragma once
#include <type_traits>

#include "element.cuh"
#include "tc_prims.cuh"

namespace coral {

constexpr int kPaThreads = 12 * 32;                // warps 0..3 and 4..7: softmax of a tile each, 8 and 9: a tile's MMAs each, 10: copies, 11: shares
constexpr int kPaShares = 4;                       // shares of a block known ahead
constexpr int kPaKeys = 64;                        // keys of a step
constexpr int kPaRows = 128 * 128;                 // bytes of 64 columns of 128 query rows
constexpr int kPaBlock = kPaKeys * 128;            // ... of a step's keys or values

struct PaArgs {
    int n_seq, T, Tk, n_q, n_k, G, gp, D;          // gp: heads side by side in a tile, gp_log2 of them
    int gp_log2, units;                            // units: places for pairs of tiles of all sequences, times groups of heads
    float c;                                       // scale log2(e)
    const int64_t *q_offsets, *k_offsets;
    const void *q, *k, *v;
    long long ld_q, ld_k, ld_v, ld_out;
    void* out;
    float* lse;
    DeviceState* st;
};

// One turn of a block: a pair of tiles of a sequence (and a group of heads, which goes by the turn's number).
struct PaShare {
    int q0, k0, Lq, Lk, pair, hg;                  // pair < 0: none
};

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x0, int x1, int x2, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(dst), "l"(map), "r"(x0), "r"(x1), "r"(x2), "r"(bar) : "memory");
}
// Shared-memory descriptors by their low words (start address / 16, leading offset); what a tile's rows of 128 bytes, eight of them 1024
// bytes, 128-byte swizzle need beside that is the same for both kinds.  N-major (the values): the next 64 columns lie kPaBlock bytes on.
constexpr uint32_t kPaDescHi = 64u | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t pa_desc_k(uint32_t saddr) { return (saddr >> 4) | (1u << 16); }
__device__ __forceinline__ uint32_t pa_desc_n(uint32_t saddr) { return (saddr >> 4) | ((uint32_t)(kPaBlock >> 4) << 16); }
// D (+)= A B, A from shared or from tensor memory.  ADD is known where the instruction is written, and the addresses are the same for
// the warp: the issuing thread has next to nothing to do beside the MMAs.
template <bool ADD>
__device__ __forceinline__ void pa_mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc) {
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 da, {%1, %4};\n\tmov.b64 db, {%2, %4};\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(kPaDescHi), "n"(ADD ? 1 : 0) : "memory");
}
template <bool ADD>
__device__ __forceinline__ void pa_mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc) {
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 db;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 db, {%2, %4};\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(kPaDescHi), "n"(ADD ? 1 : 0) : "memory");
}
__device__ __forceinline__ bool pa_elect() {
    uint32_t on;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(on));
    return on != 0;
}
// 32 columns of this thread's tensor-memory lane, not waited for.
__device__ __forceinline__ void pa_ld32(uint32_t taddr, uint32_t* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr));
}
__device__ __forceinline__ void pa_st32(uint32_t taddr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
          "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
          "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]),
          "r"(r[30]), "r"(r[31]) : "memory");
}
__device__ __forceinline__ void pa_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, DeviceState* st) {
    if (!mbar_try_wait(bar, parity)) mbar_wait(bar, parity, abort_flag, st);
}
__device__ __forceinline__ void pa_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void pa_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ float pa_exp2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float pa_max3(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }
template <typename T> __device__ __forceinline__ uint32_t pa_pack(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pa_pack<__nv_bfloat16>(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <> __device__ __forceinline__ uint32_t pa_pack<__half>(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// The turns of a block: every grid-th unit, forwards and backwards in turn.  Units come with their rows' lengths falling, so the blocks'
// sums come out alike (nine packed prompts of 1 to 2048 tokens: 113 us sequence by sequence, 97 so).
__device__ __forceinline__ int pa_unit(const PaArgs& a, int turn) {
    const long long u = (long long)turn * gridDim.x + (turn & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
    return u < a.units ? (int)u : -1;
}
__device__ __forceinline__ int pa_turns(const PaArgs& a) { return (a.units - 1) / (int)gridDim.x + 1; }

// Finds units' sequences, by a warp; the units that it is asked for must not go down.  Up to 128 sequences: pair p of every sequence that
// has one, then pair p - 1 ...; more: the sequences in turn, each from its end.
struct PaFinder {
    static constexpr int kWays = 4;
    int n[kWays];                                  // pairs of tiles of sequences 32 i + lane
    int level = 0, base = 0, before = 0;           // pair looked at, sequences passed, units in front of them
    bool by_level;

    __device__ __forceinline__ explicit PaFinder(const PaArgs& a) : by_level(a.n_seq <= 32 * kWays) {
        if (!by_level) return;
        int most = 0;
#pragma unroll
        for (int i = 0; i < kWays; ++i) {
            const int seq = i * 32 + (threadIdx.x & 31);
            int q0 = 0, Lq = 0;
            if (seq < a.n_seq) clamped_range(a.q_offsets, seq, a.T, &q0, &Lq);
            n[i] = pairs(a, Lq);
            most = max(most, n[i]);
        }
        level = __reduce_max_sync(0xffffffffu, most) - 1;
    }
    static __device__ __forceinline__ int pairs(const PaArgs& a, int Lq) {
        const int per = 256 >> a.gp_log2;
        return (Lq + per - 1) / per;
    }
    // the sequence's share, by all lanes
    static __device__ __forceinline__ PaShare share(const PaArgs& a, int seq, int pair, int hg) {
        PaShare s{0, 0, 0, 0, pair, hg};
        clamped_range(a.q_offsets, seq, a.T, &s.q0, &s.Lq);
        s.k0 = s.q0;
        s.Lk = s.Lq;
        if (a.k_offsets) clamped_range(a.k_offsets, seq, a.Tk, &s.k0, &s.Lk);
        return s;
    }
    __device__ __forceinline__ PaShare operator()(const PaArgs& a, int unit) {
        const int lane = threadIdx.x & 31, hgs = a.n_k * (a.G >> a.gp_log2), slot = unit / hgs, hg = unit - slot * hgs;
        if (by_level) {
            for (; level >= 0; --level) {
                uint32_t has[kWays];
                int all = 0;
#pragma unroll
                for (int i = 0; i < kWays; ++i) {
                    has[i] = __ballot_sync(0xffffffffu, n[i] > level);
                    all += __popc(has[i]);
                }
                if (slot >= before + all) {
                    before += all;
                    continue;
                }
                int r = slot - before, seq = -1;   // the r-th of those that have it
#pragma unroll
                for (int i = 0; i < kWays; ++i) {
                    const uint32_t at = __ballot_sync(0xffffffffu, (has[i] >> lane & 1u) && __popc(has[i] & ((1u << lane) - 1)) == r);
                    if (seq < 0 && at) seq = i * 32 + __ffs(at) - 1;
                    r = seq >= 0 ? -1 : r - __popc(has[i]);
                }
                return share(a, seq, level, hg);
            }
        } else {
            for (; base < a.n_seq; base += 32) {
                const int seq = base + lane;
                int q0 = 0, Lq = 0;
                if (seq < a.n_seq) clamped_range(a.q_offsets, seq, a.T, &q0, &Lq);
                const int mine = pairs(a, Lq);
                int sum = mine;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int v = __shfl_up_sync(0xffffffffu, sum, o);
                    if (lane >= o) sum += v;
                }
                const int all = __shfl_sync(0xffffffffu, sum, 31);
                if (slot >= before + all) {
                    before += all;
                    continue;
                }
                const int first = before + sum - mine, from = __ffs(__ballot_sync(0xffffffffu, slot >= first && slot < first + mine)) - 1;
                return share(a, base + from, __shfl_sync(0xffffffffu, mine - 1 - (slot - first), from), hg);
            }
        }
        return PaShare{0, 0, 0, 0, -1, 0};
    }
};

// What a unit's share means.
struct PaUnit {
    PaShare sh;
    int tile_tokens, kv_head, head0, past, n[2], steps;
    __device__ __forceinline__ PaUnit(const PaArgs& a, const PaShare& share) : sh(share) {
        tile_tokens = 128 >> a.gp_log2;
        const int per_head = a.G >> a.gp_log2;
        kv_head = sh.hg / per_head;
        head0 = kv_head * a.G + (sh.hg - kv_head * per_head) * a.gp;
        past = sh.Lk - sh.Lq;                      // token i sees keys up to i + past
#pragma unroll
        for (int t = 0; t < 2; ++t) {              // steps of a tile: keys that its last token sees
            const int tok0 = token0(t), last = min(tok0 + tile_tokens, sh.Lq) - 1;
            n[t] = tok0 >= sh.Lq ? 0 : (max(0, min(last + past + 1, sh.Lk)) + kPaKeys - 1) / kPaKeys;
        }
        steps = max(n[0], n[1]);
    }
    __device__ __forceinline__ int token0(int t) const { return (sh.pair * 2 + t) * tile_tokens; }
};

// References above this: S c - m in one rounding, with m = S c rounded, leaves more than half a power of two, and beyond 2^27 more than fp16 or the
// sums have room for.
constexpr float kPaFar = 0x1p22f;

// One row again, by a warp in fp32: only keys that it sees take part.  Scores: sixteen lanes a key, eight columns each; values: four columns a lane.
template <typename T>
__device__ __noinline__ void pa_row_again(const PaArgs& a, const T* q, const T* k, const T* v, int seen, T* out, float* lse) {
    const int lane = threadIdx.x & 31, part = lane & 15;
    const bool on = part * 8 < a.D;
    float x[8] = {};
    if (on) Elem<T>::load8(q + part * 8, x);
    // of key j0 + lane; eight loads on their way at a time
    auto score = [&](int j0) {
        float mine = 0.f;
        for (int i0 = 0; i0 < 16; i0 += 8) {
            float y[8][8], s[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) Elem<T>::load8(k + (long long)min(j0 + i0 + i + (lane & 16), seen - 1) * a.ld_k + (on ? part * 8 : 0), y[i]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                s[i] = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) s[i] = fmaf(x[e], y[i][e], s[i]);
                if (!on) s[i] = 0.f;
            }
#pragma unroll
            for (int o = 1; o < 16; o <<= 1)
#pragma unroll
                for (int i = 0; i < 8; ++i) s[i] += __shfl_xor_sync(0xffffffffu, s[i], o);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (part == i0 + i) mine = s[i];
        }
        return __fmul_rn(mine, a.c);                           // rounded once for the maximum and the weight, whatever its size
    };
    float top = kNegInf, sum = 0.f, acc[4] = {};
    for (int j0 = 0; j0 < seen; j0 += 32) {
        const float s = score(j0);
        if (j0 + lane < seen) top = fmaxf(top, s);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (top == kNegInf) top = 0.f;
    for (int j0 = 0; j0 < seen; j0 += 32) {
        const float s = score(j0), p = j0 + lane < seen ? pa_exp2(s - top) : 0.f;
        sum += p;
        const int n = min(32, seen - j0);
        for (int i0 = 0; i0 < n; i0 += 8) {                    // eight values on their way at a time
            uint2 r[8];
            if (lane * 4 < a.D)
#pragma unroll
                for (int i = 0; i < 8; ++i) r[i] = *reinterpret_cast<const uint2*>(v + (long long)(j0 + min(i0 + i, n - 1)) * a.ld_v + lane * 4);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float w = __shfl_sync(0xffffffffu, p, i0 + i);
                if (lane * 4 >= a.D || i0 + i >= n) continue;
                T h[4];
                *reinterpret_cast<uint2*>(h) = r[i];
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[e] = fmaf(w, Elem<T>::up(h[e]), acc[e]);
            }
        }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    if (lane * 4 < a.D) {
        T h[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] = Elem<T>::down(acc[e] * inv);
        *reinterpret_cast<uint2*>(out + lane * 4) = *reinterpret_cast<const uint2*>(h);
    }
    if (lse && lane == 0) *lse = sum == 0.f ? kNegInf : (top + log2f(sum)) * 0.69314718055994531f;
}

// What stands in the first output of a row that is to be computed again until that is done: a NaN as no conversion gives it.
constexpr uint16_t kPaAgain = 0x7fa1;
// (ordered with the outputs' other stores and loads, which have other types)
__device__ __forceinline__ void pa_mark(void* out) { asm volatile("st.global.u16 [%0], %1;" ::"l"(out), "h"(kPaAgain) : "memory"); }
__device__ __forceinline__ bool pa_marked(const void* out) {
    uint16_t w;
    asm volatile("ld.global.u16 %0, [%1];" : "=h"(w) : "l"(out) : "memory");
    return w == kPaAgain;
}

// Whether any of eight 16-bit elements is an infinity or a NaN.
template <typename T>
__device__ __forceinline__ bool pa_bad8(const uint4& w) {
    constexpr uint32_t kOnes = std::is_same_v<T, __half> ? 0x7c007c00u : 0x7f807f80u;          // two exponents
    return (__vcmpeq2(w.x & kOnes, kOnes) | __vcmpeq2(w.y & kOnes, kOnes) | __vcmpeq2(w.z & kOnes, kOnes) | __vcmpeq2(w.w & kOnes, kOnes)) != 0;
}
// The first of the rows from .. end that holds an infinity or a NaN (LAST: the last), by a warp; `end` (-1) if none does.
template <typename T, bool LAST>
__device__ __noinline__ int pa_bad_row(const T* v, long long ld, int D, int from, int end) {
    const int per = D / 8;
    int bad = LAST ? -1 : end;
    for (int j0 = from; j0 < end && (LAST || bad == end); j0 += 64) {
        const int n = min(64, end - j0);
        for (int i = threadIdx.x & 31; i < n * per; i += 32) {
            const int j = i / per;
            if (!pa_bad8<T>(*reinterpret_cast<const uint4*>(v + (long long)(j0 + j) * ld + (i - j * per) * 8))) continue;
            bad = LAST ? max(bad, j0 + j) : min(bad, j0 + j);
        }
        bad = LAST ? __reduce_max_sync(0xffffffffu, bad) : __reduce_min_sync(0xffffffffu, bad);
    }
    return bad;
}

// DB: blocks of 64 columns of a head (1 or 2).  Stages: steps' keys or values in the ring.
template <int DB> constexpr int kPaStages = DB == 2 ? 10 : 16;
template <int DB> constexpr size_t pa_smem_bytes() { return 1024 + (size_t)DB * (2 * kPaRows + kPaStages<DB> * kPaBlock); }

template <typename T, int DB>
__global__ void __launch_bounds__(kPaThreads, 1)
prompt_attention_kernel(const PaArgs a, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                        const __grid_constant__ CUtensorMap map_v) {
    constexpr int STAGES = kPaStages<DB>, kTile = DB * kPaRows, kStep = DB * kPaBlock;
    extern __shared__ unsigned char pa_smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(pa_smem_raw) + 1023) & ~(uintptr_t)1023);
    unsigned char* s_kv = smem + 2 * kTile;
    __shared__ __align__(8) uint64_t q_full, q_empty, kv_full[STAGES], kv_empty[STAGES], s_full[4], p_full[4], pv_done[4];   // [tile][buffer]
    __shared__ __align__(8) uint64_t o_free[2], share_full[kPaShares], share_empty[kPaShares];
    __shared__ PaShare shares[kPaShares];
    __shared__ uint32_t tmem_slot;
    __shared__ volatile int abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        mbar_init(smem_u32(&q_full), 1);
        mbar_init(smem_u32(&q_empty), 2);
        for (int i = 0; i < STAGES; ++i) {
            mbar_init(smem_u32(&kv_full[i]), 1);
            mbar_init(smem_u32(&kv_empty[i]), 2);
        }
        for (int i = 0; i < 4; ++i) {
            mbar_init(smem_u32(&s_full[i]), 1);
            mbar_init(smem_u32(&p_full[i]), 4);
            mbar_init(smem_u32(&pv_done[i]), 1);
        }
        for (int i = 0; i < 2; ++i) mbar_init(smem_u32(&o_free[i]), 4);
        for (int i = 0; i < kPaShares; ++i) {
            mbar_init(smem_u32(&share_full[i]), 1);
            mbar_init(smem_u32(&share_empty[i]), 11);
        }
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 8) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_wait();
    if (blockIdx.x == 0 && threadIdx.x == 0) a.st->status = 0;      // a wait would have to fail millions of polls before this
    const uint32_t tmem = tmem_slot;
    const int turns = pa_turns(a);
    // The share of a turn, by all lanes of a warp or by one thread alone (which then counts for its warp).
    auto share_of = [&](int turn, bool alone) {
        const int i = turn % kPaShares;
        pa_wait(smem_u32(&share_full[i]), (uint32_t)(turn / kPaShares) & 1u, &abort_flag, a.st);
        const PaShare sh = shares[i];
        if (!alone) __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&share_empty[i]));
        return sh;
    };

    if (warp == 11) {
        PaFinder find(a);
        for (int turn = 0; turn < turns; ++turn) {
            const int unit = pa_unit(a, turn), i = turn % kPaShares;
            PaShare sh{0, 0, 0, 0, -1, 0};
            if (unit >= 0) sh = find(a, unit);
            pa_wait(smem_u32(&share_empty[i]), ((uint32_t)(turn / kPaShares) & 1u) ^ 1u, &abort_flag, a.st);
            __syncwarp();
            if (lane == 0) {
                shares[i] = sh;
                mbar_arrive(smem_u32(&share_full[i]));
            }
        }
    } else if (warp == 10) {
        if (lane == 0) {
            int stage = 0, loads = 0, queries = 0;
            uint32_t phase = 0;
            for (int turn = 0; turn < turns; ++turn) {
                const PaShare sh = share_of(turn, true);
                if (sh.pair < 0) continue;
                const PaUnit u(a, sh);
                if (u.steps == 0) continue;
                auto load = [&](const CUtensorMap* map, int j) {
                    pa_wait(smem_u32(&kv_empty[stage]), phase ^ 1u, &abort_flag, a.st);
                    const uint32_t bar = smem_u32(&kv_full[stage]);
                    mbar_expect_tx(bar, kStep);
                    for (int b = 0; b < DB; ++b) tma_load_3d(smem_u32(s_kv + stage * kStep + b * kPaBlock), map, b * 64, u.kv_head, sh.k0 + j * kPaKeys, bar);
                    ++loads;
                    if (++stage == STAGES) { stage = 0; phase ^= 1u; }
                };
                // the order in which they are used: keys of steps 0 and 1, then a step's values and the keys of the step after the next
                load(&map_k, 0);
                pa_wait(smem_u32(&q_empty), (uint32_t)(queries & 1) ^ 1u, &abort_flag, a.st);
                mbar_expect_tx(smem_u32(&q_full), 2 * kTile);
                for (int t = 0; t < 2; ++t)
                    for (int b = 0; b < DB; ++b)
                        tma_load_3d(smem_u32(smem + t * kTile + b * kPaRows), &map_q, b * 64, u.head0, sh.q0 + u.token0(t), smem_u32(&q_full));
                ++queries;
                if (u.steps > 1) load(&map_k, 1);
                for (int j = 0; j < u.steps; ++j) {
                    load(&map_v, j);
                    if (j + 2 < u.steps) load(&map_k, j + 2);
                }
            }
            // nothing is left on its way when the block ends, an expired wait elsewhere included
            if (queries) pa_wait(smem_u32(&q_full), (uint32_t)(queries - 1) & 1u, &abort_flag, a.st);
            for (int i = max(0, loads - STAGES); i < loads; ++i) pa_wait(smem_u32(&kv_full[i % STAGES]), (uint32_t)(i / STAGES) & 1u, &abort_flag, a.st);
        }
    } else if (warp == 8 || warp == 9) {
        // The MMAs of tile t, in the ring's order; both tiles' warps free a place of it.
        const int t = warp - 8;
        constexpr uint32_t kType = std::is_same_v<T, __nv_bfloat16> ? 1u : 0u;
        constexpr uint32_t kBase = (1u << 4) | (kType << 7) | (kType << 10) | (8u << 24);
        const int d16 = (a.D + 15) / 16;
        const uint32_t idesc_s = kBase | ((uint32_t)(kPaKeys / 8) << 17), idesc_o = kBase | (1u << 16) | ((uint32_t)(2 * d16) << 17);
        const uint32_t q = pa_desc_k(smem_u32(smem) + t * kTile), kv = smem_u32(s_kv), ts = tmem + t * 128, to = tmem + 256 + t * 128;
        int stage = 0, queries = 0, outputs = 0, done = 0;     // done: steps of this tile in earlier turns
        uint32_t phase = 0;
        auto full = [&]() { pa_wait(smem_u32(&kv_full[stage]), phase, &abort_flag, a.st); };
        auto next = [&]() {
            if (++stage == STAGES) { stage = 0; phase ^= 1u; }
        };
        for (int turn = 0; turn < turns; ++turn) {
            const PaShare sh = share_of(turn, false);
            if (sh.pair < 0) continue;
            const PaUnit u(a, sh);
            const int n = u.steps, nt = u.n[t];
            if (n == 0) continue;
            auto scores = [&](int j) {                         // S = Q K^T of step j; the keys are free behind it
                full();
                if (j < nt) {
                    tc_fence_after();
                    if (pa_elect()) {
                        const int buf = (done + j) & 1;
                        const uint32_t k = pa_desc_k(kv + stage * kStep), to_s = ts + buf * kPaKeys;
                        pa_mma_ss<false>(to_s, q, k, idesc_s);
#pragma unroll
                        for (int kk = 1; kk < DB * 4; ++kk)
                            if (kk < d16) pa_mma_ss<true>(to_s, q + (kk >> 2) * (kPaRows / 16) + (kk & 3) * 2, k + (kk >> 2) * (kPaBlock / 16) + (kk & 3) * 2, idesc_s);
                        tc_commit(smem_u32(&s_full[t * 2 + buf]));
                        tc_commit(smem_u32(&kv_empty[stage]));
                        if (j == nt - 1) tc_commit(smem_u32(&q_empty));
                    }
                } else if (lane == 0) {
                    mbar_arrive(smem_u32(&kv_empty[stage]));   // the other tile's alone
                }
                next();
            };
            // the keys' place comes before the queries, as the copies do
            full();
            pa_wait(smem_u32(&q_full), (uint32_t)(queries & 1), &abort_flag, a.st);
            ++queries;
            if (nt == 0 && lane == 0) mbar_arrive(smem_u32(&q_empty));
            scores(0);
            if (n > 1) scores(1);
            for (int j = 0; j < n; ++j) {
                full();
                if (j < nt) {
                    const int buf = (done + j) & 1, left = sh.Lk - j * kPaKeys;
                    // Rows behind the sequence's values get zero (by both tiles' warps alike): what lies there may be anything, and a
                    // weight of zero times it not zero.
                    if (left < kPaKeys) {
                        for (int i = left * 8 + lane; i < kPaKeys * 8; i += 32)
#pragma unroll
                            for (int d = 0; d < DB; ++d) *reinterpret_cast<uint4*>(s_kv + stage * kStep + d * kPaBlock + i * 16) = make_uint4(0, 0, 0, 0);
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                    }
                    if (j == 0) pa_wait(smem_u32(&o_free[t]), (uint32_t)(outputs & 1) ^ 1u, &abort_flag, a.st);
                    pa_wait(smem_u32(&p_full[t * 2 + buf]), (uint32_t)((done + j) >> 1) & 1u, &abort_flag, a.st);
                    tc_fence_after();
                    if (pa_elect()) {
                        const uint32_t v = pa_desc_n(kv + stage * kStep), p = ts + buf * kPaKeys;
                        if (j == 0) pa_mma_ts<false>(to, p, v, idesc_o);
                        else pa_mma_ts<true>(to, p, v, idesc_o);
#pragma unroll
                        for (int kk = 1; kk < kPaKeys / 16; ++kk) pa_mma_ts<true>(to, p + kk * 8, v + kk * 128, idesc_o);
                        tc_commit(smem_u32(&pv_done[t * 2 + buf]));
                        tc_commit(smem_u32(&kv_empty[stage]));
                    }
                } else if (lane == 0) {
                    mbar_arrive(smem_u32(&kv_empty[stage]));
                }
                next();
                if (j + 2 < n) scores(j + 2);
            }
            done += nt;
            if (nt > 0) ++outputs;
        }
        // the last products are done before the block ends
        if (done > 0) pa_wait(smem_u32(&pv_done[t * 2 + ((done - 1) & 1)]), (uint32_t)((done - 1) >> 1) & 1u, &abort_flag, a.st);
    } else {
        const int t = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t ts = tmem + t * 128 + lanes, to = tmem + 256 + t * 128 + lanes;
        int done = 0, first_again = turns;                     // steps of this tile in earlier turns; the first with a row to be computed again
        for (int turn = 0; turn < turns; ++turn) {
            const PaShare sh = share_of(turn, false);
            if (sh.pair < 0) continue;
            const PaUnit u(a, sh);
            const int nt = u.n[t], tok0 = u.token0(t), past = u.past;
            if (tok0 >= sh.Lq) continue;
            const int tok = tok0 + (row >> a.gp_log2), head = u.head0 + (row & (a.gp - 1));
            const int seen = max(0, min(tok + past + 1, sh.Lk));   // keys that this row sees
            const int all_see = max(0, min(tok0 + past + 1, sh.Lk));
            float m = kNegInf, mc = 0.f;                           // reference, raw and in powers of two
            bool far = false;
            unsigned long long sum2 = 0;
            float s[kPaKeys];
            uint32_t* sr = reinterpret_cast<uint32_t*>(s);
            for (int j = 0; j < nt; ++j) {
                const int at_step = done + j, buf = at_step & 1;
                pa_wait(smem_u32(&s_full[t * 2 + buf]), (uint32_t)(at_step >> 1) & 1u, &abort_flag, a.st);
                __syncwarp();
                tc_fence_after();
                const uint32_t at = ts + buf * kPaKeys;
                pa_ld32(at, sr);
                pa_ld32(at + 32, sr + 32);
                pa_ld_wait();
                if ((j + 1) * kPaKeys > all_see) {
                    const int left = seen - j * kPaKeys;
#pragma unroll
                    for (int i = 0; i < kPaKeys; ++i) s[i] = i < left ? s[i] : kNegInf;
                }
                float m4[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
                for (int i = 4; i < kPaKeys; i += 8)
#pragma unroll
                    for (int e = 0; e < 4; ++e) m4[e] = i + 4 + e < kPaKeys ? pa_max3(m4[e], s[i + e], s[i + 4 + e]) : fmaxf(m4[e], s[i + e]);
                const float top = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
                const bool moves = top * a.c > mc + 8.f || (m == kNegInf && top > kNegInf);
                if (__any_sync(0xffffffffu, moves)) {
                    const float next = moves ? top : m, next_c = next == kNegInf ? 0.f : next * a.c;
                    const float f = !moves ? 1.f : m == kNegInf ? 0.f : pa_exp2(mc - next_c);
                    far |= fabsf(next_c) > kPaFar;
                    m = next;
                    mc = next_c;
                    sum2 = mul2(sum2, pair_of(f, f));
                    if (j > 0) {                                   // O, once the step before is in it
                        pa_wait(smem_u32(&pv_done[t * 2 + (buf ^ 1)]), (uint32_t)((at_step - 1) >> 1) & 1u, &abort_flag, a.st);
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
                const unsigned long long c2 = pair_of(a.c, a.c), m2 = pair_of(-mc, -mc);
                uint32_t p[kPaKeys / 2];
#pragma unroll
                for (int i = 0; i < kPaKeys / 2; ++i) {
                    const float2 x = halves(fma2(pair_of(s[2 * i], s[2 * i + 1]), c2, m2));
                    const float lo = pa_exp2(x.x), hi = pa_exp2(x.y);
                    sum2 = add2(sum2, pair_of(lo, hi));
                    p[i] = pa_pack<T>(lo, hi);
                }
                pa_st32(at, p);
                pa_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&p_full[t * 2 + buf]));
            }
            const float2 sums = halves(sum2);
            const float sum = sums.x + sums.y, inv = sum == 0.f ? 0.f : 1.f / sum;
            if (nt > 0) {
                done += nt;
                pa_wait(smem_u32(&pv_done[t * 2 + ((done - 1) & 1)]), (uint32_t)((done - 1) >> 1) & 1u, &abort_flag, a.st);
                __syncwarp();
                tc_fence_after();
            }
            const bool live = tok < sh.Lq;
            T* out = static_cast<T*>(a.out) + (long long)(sh.q0 + tok) * a.ld_out + (long long)head * a.D;
            float odd = 0.f;                                       // NaN where a result is not finite
#pragma unroll
            for (int b = 0; b < 2 * DB; ++b) {
                if (b * 32 >= a.D) break;
                uint32_t o[32];
                if (nt > 0) {
                    pa_ld32(to + b * 32, o);
                    pa_ld_wait();
                }
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int col = b * 32 + g * 8;
                    float x[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        x[e] = sum == 0.f ? 0.f : __uint_as_float(o[g * 8 + e]) * inv;
                        if (col < a.D) odd = fmaf(x[e], 0.f, odd);
                    }
                    if (live && col < a.D) Elem<T>::store8(out + col, x);
                }
            }
            if (nt > 0) {                                          // the next turn's sums may go there
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&o_free[t]));
            }
            if (live && a.lse) a.lse[(long long)(sh.q0 + tok) * a.n_q + head] = sum == 0.f ? kNegInf : (mc + log2f(sum)) * 0.69314718055994531f;
            // Rows of finite weights whose result is not (values that they do not see may be the reason), and those of scores too large.
            far = far && live;
            if (far) pa_mark(out);
            if (__any_sync(0xffffffffu, far || (live && sum > 0.f && sum < __int_as_float(0x7f800000) && odd != 0.f))) first_again = min(first_again, turn);
        }
        if (first_again < turns) {
            PaFinder find(a);
            for (int turn = first_again; turn < turns; ++turn) {
                const int unit = pa_unit(a, turn);
                if (unit < 0) continue;
                const PaShare sh = find(a, unit);
                if (sh.pair < 0) continue;
                const PaUnit u(a, sh);
                const int tok = u.token0(t) + (row >> a.gp_log2), head = u.head0 + (row & (a.gp - 1)), seen = max(0, min(tok + u.past + 1, sh.Lk));
                const T* v = static_cast<const T*>(a.v) + (long long)sh.k0 * a.ld_v + (long long)u.kv_head * a.D;
                T* out = static_cast<T*>(a.out) + (long long)(sh.q0 + tok) * a.ld_out + (long long)head * a.D;
                bool odd = false, far = false;                     // by what this thread wrote
                if (tok < sh.Lq) {
                    far = pa_marked(out);
                    for (int c = 0; c < a.D; c += 8) odd |= pa_bad8<T>(*reinterpret_cast<const uint4*>(out + c));
                }
                // Not finite, and rightly so: the row sees a value of that kind, and its last step held none that it does not see.  (fp16 has no
                // weights below 2^-25, and zero times an infinity is a NaN where the sum is infinite: there all are computed again.)
                if (std::is_same_v<T, __nv_bfloat16> && __any_sync(0xffffffffu, odd && !far)) {
                    const int end = min(u.n[t] * kPaKeys, sh.Lk), least = __reduce_min_sync(0xffffffffu, odd ? seen : end);
                    const int last = pa_bad_row<T, true>(v, a.ld_v, a.D, least, end);
                    const int first = pa_bad_row<T, false>(v, a.ld_v, a.D, 0, __reduce_max_sync(0xffffffffu, odd ? seen : 0));
                    odd = odd && (last >= seen || first >= seen);
                }
                for (uint32_t todo = __ballot_sync(0xffffffffu, odd || far); todo; todo &= todo - 1) {
                    const int r = __ffs(todo) - 1, tok_r = __shfl_sync(0xffffffffu, tok, r), head_r = __shfl_sync(0xffffffffu, head, r);
                    const bool lse_r = __shfl_sync(0xffffffffu, far, r) && a.lse;
                    pa_row_again<T>(a, static_cast<const T*>(a.q) + (long long)(sh.q0 + tok_r) * a.ld_q + (long long)head_r * a.D,
                                    static_cast<const T*>(a.k) + (long long)sh.k0 * a.ld_k + (long long)u.kv_head * a.D, v, __shfl_sync(0xffffffffu, seen, r),
                                    static_cast<T*>(a.out) + (long long)(sh.q0 + tok_r) * a.ld_out + (long long)head_r * a.D,
                                    lse_r ? a.lse + (long long)(sh.q0 + tok_r) * a.n_q + head_r : nullptr);
                }
            }
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

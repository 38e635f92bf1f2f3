// Products of 17 and more rows with 4-bit weights on the 5th-generation tensor cores.  One MMA takes 128 output rows of weights
// as its operand A, straight from tensor memory, and up to 64 rows of activations as operand B from shared memory:
//   * eight warps, one thread an output row (two tiles of 128 rows a block), turn packed words into exact fp16 operands
//     (q - z, as subnormals: two operations a pair) and store them to tensor memory; no weight goes through shared memory,
//     whose bandwidth would bound the kernel otherwise,
//   * one thread issues the MMAs of a group of columns, accumulating from zero,
//   * the same eight warps read a finished group's sums back, scale them in fp32 and add them up in registers.
// Operands and sums of two groups are in flight, so a group is unpacked while the tensor cores work on the one before.
// Each tile has its own barriers and its own issuing thread: one thread alone issues an MMA every 45 cycles, two of them keep the
// 32 that one takes (152064 x 3584, 60 rows: 181 -> 157 us with groups of 128, 226 -> 218 with groups of 64).
// The activations (laid out by q4_stage_kernel, swizzled) come through a ring of 64-column slabs, one bulk copy each, shared by
// the block's 256 output rows.
#pragma once
#include "q4.cuh"
#include "tc_prims.cuh"

namespace coral {

constexpr int kQ4TcWarps = 8;                      // unpacking warps; warps 8 and 9 issue the MMAs of a tile each, warp 10 the copies
constexpr int kQ4TcThreads = (kQ4TcWarps + 3) * 32;
constexpr int kQ4TcTiles = 16;                     // 16-row weight tiles of a pass: two MMA tiles of 128 rows
constexpr int kQ4TcSlabs = 8;                      // slabs of activations in flight
constexpr int kQ4TcMaxRows = 64;                   // activation rows of a launch
constexpr int kQ4TcMaxSplit = 16, kQ4TcMaxParts = 160;

// Who computes what: block i takes the passes (256 output rows each) i, i + full_step, ... of the first `full` a block, and then
// one of the `tail` passes left over, or a part of its columns: they are split into `split` parts where that keeps more SMs busy.
struct Q4Share {
    int full, tail, split;
    float* part;                                   // [tail * split][activation row][256] sums of the parts, as yet scaled
};

template <int MP>
constexpr size_t q4_tc_smem_bytes() { return 1024 + (size_t)kQ4TcSlabs * MP * 128 + MP * sizeof(Q4Power) + 256; }

__device__ __forceinline__ uint32_t q4_sub_f16x2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}

// Stores this thread's next 32-bit columns of its tensor-memory lane.
__device__ __forceinline__ void tc_st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
          "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
// D (128 x n) += A (128 x 16, tensor memory) * B (n x 16, shared memory)
__device__ __forceinline__ void tc_mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}

// grid: the SMs, or tail * split blocks if there are no full passes.  K columns are PER groups a block of 128; `st` holds the
// slabs of MP rows.
template <int MP, int PER, bool ZEROS>
__global__ void __launch_bounds__(kQ4TcThreads, 1) q4_tc_kernel(Q4View q, Q4Staged st, Q4Share share, int M, void* __restrict__ out, int out_type, DeviceState* state) {
    extern __shared__ unsigned char q4_smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(q4_smem_raw) + 1023) & ~(uintptr_t)1023);
    constexpr int kSlabBytes = MP * 128;
    constexpr uint32_t kIdesc = (1u << 4) | ((uint32_t)(MP >> 3) << 17) | (8u << 24);      // D fp32, A and B fp16, 128 x MP
    Q4Power* s_back = reinterpret_cast<Q4Power*>(smem + (size_t)kQ4TcSlabs * kSlabBytes);
    uint64_t* x_full = reinterpret_cast<uint64_t*>(s_back + MP);
    uint64_t* x_empty = x_full + kQ4TcSlabs;
    uint64_t* a_full = x_empty + kQ4TcSlabs;       // [tile][2] a group's operands are in tensor memory (and the buffer's old sums out)
    uint64_t* d_full = a_full + 4;                 // [2][2] its sums are
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(d_full + 4);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kQ4TcSlabs; ++i) {
            mbar_init(smem_u32(&x_full[i]), 1);
            mbar_init(smem_u32(&x_empty[i]), 2);
        }
        for (int i = 0; i < 4; ++i) {
            mbar_init(smem_u32(&a_full[i]), kQ4TcWarps / 2);
            mbar_init(smem_u32(&d_full[i]), 1);
        }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == kQ4TcWarps) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    // tensor memory: sums of (tile, buffer) at (2 tile + buffer) MP, operands behind them, 64 columns each
    auto d_at = [&](int tile, int buf) { return tmem + (uint32_t)((tile * 2 + buf) * MP); };
    auto a_at = [&](int tile, int buf) { return tmem + (uint32_t)(4 * MP + (tile * 2 + buf) * 64); };

    const int passes = share.full + ((int)blockIdx.x < share.tail * share.split ? 1 : 0);
    constexpr int kGroupCols = 128 / PER;
    const int groups = q.K / kGroupCols, slabs = (q.K + 63) / 64;
    // a pass of this block: its first 16-row weight tile and its blocks of 128 columns
    auto tile_of = [&](int pass) {
        return (pass < share.full ? pass * (int)gridDim.x + (int)blockIdx.x : share.full * (int)gridDim.x + (int)blockIdx.x / share.split) * kQ4TcTiles;
    };
    auto from_block = [&](int pass) { return pass < share.full ? 0 : (int)(blockIdx.x % share.split) * q.KB / share.split; };
    auto to_block = [&](int pass) { return pass < share.full ? q.KB : ((int)(blockIdx.x % share.split) + 1) * q.KB / share.split; };

    if (warp == kQ4TcWarps + 2) {
        if (lane == 0) {
            pdl_wait();
            int stage = 0;
            uint32_t phase = 0;
            int copies = 0;
            for (int pass = 0; pass < passes; ++pass)
                for (int i = from_block(pass) * 2; i < min(to_block(pass) * 2, slabs); ++i, ++copies) {
                    tc_wait(smem_u32(&x_empty[stage]), phase ^ 1u, abort_flag, state);
                    const uint32_t bar = smem_u32(&x_full[stage]);
                    mbar_expect_tx(bar, kSlabBytes);
                    bulk_g2s(smem_u32(smem + (size_t)stage * kSlabBytes), st.x + (size_t)i * MP * 8, kSlabBytes, bar);
                    if (++stage == kQ4TcSlabs) { stage = 0; phase ^= 1u; }
                }
            // nothing is left on its way when the block ends, an expired wait elsewhere included
            for (int i = 0; i < kQ4TcSlabs && i < copies; ++i)
                tc_wait(smem_u32(&x_full[i]), (uint32_t)((copies - 1 - i) / kQ4TcSlabs) & 1u, abort_flag, state);
        }
    } else if (warp >= kQ4TcWarps) {
        if (lane == 0) {
            const int tile = warp - kQ4TcWarps;
            int stage = 0, unit = 0;
            uint32_t phase = 0;
            for (int pass = 0; pass < passes; ++pass)
                for (int g = from_block(pass) * PER, to = min(to_block(pass) * PER, groups); g < to; ++g, ++unit) {
                    const int buf = unit & 1;
                    tc_wait(smem_u32(&a_full[tile * 2 + buf]), (uint32_t)(unit >> 1) & 1u, abort_flag, state);
                    constexpr int kSteps = kGroupCols / 16;            // MMAs of a group and tile; 4 a slab
#pragma unroll
                    for (int k0 = 0; k0 < kSteps; k0 += 4) {
                        const int half = PER == 4 ? (g & 1) * 2 : 0;   // 32-column groups: half a slab each
                        if (half == 0) tc_wait(smem_u32(&x_full[stage]), phase, abort_flag, state);
                        tc_fence_after();
                        const uint32_t sb = smem_u32(smem + (size_t)stage * kSlabBytes);
#pragma unroll
                        for (int kk = 0; kk < (kSteps < 4 ? kSteps : 4); ++kk) {
                            const uint64_t bdesc = tc_smem_desc(sb + (half + kk) * 32);
                            tc_mma_ts(d_at(tile, buf), a_at(tile, buf) + (uint32_t)((k0 + kk) * 8), bdesc, kIdesc, k0 + kk > 0 ? 1u : 0u);
                        }
                        if (PER != 4 || half == 2 || g + 1 == to) {
                            tc_commit(smem_u32(&x_empty[stage]));
                            if (++stage == kQ4TcSlabs) { stage = 0; phase ^= 1u; }
                        }
                    }
                    tc_commit(smem_u32(&d_full[tile * 2 + buf]));
                }
            if (unit > 0) tc_wait(smem_u32(&d_full[tile * 2 + ((unit - 1) & 1)]), (uint32_t)((unit - 1) >> 1) & 1u, abort_flag, state);
        }
    } else {
        const int tile = warp >> 2, row = (warp & 3) * 32 + lane;          // this thread's row of its 128-row tile
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        constexpr int kSz = Q4Scales<PER, ZEROS>::kBytes;
        if (threadIdx.x < MP) {
            pdl_wait();
            s_back[threadIdx.x] = Q4Power(st.back[threadIdx.x]);
        }
        asm volatile("bar.sync 1, 256;" ::: "memory");
        int unit = 0;
        for (int pass = 0; pass < passes; ++pass) {
            const int first = tile_of(pass) + tile * 8, t16 = first + (row >> 4), kb0 = from_block(pass), kb1 = to_block(pass);
            const bool live = t16 < q.T;
            const size_t blk0 = live ? (size_t)t16 * q.KB : 0;
            const uint4* wp = q.w + blk0 * 64 + ((row >> 3) & 1) * 32 + (row & 7) * 4;
            const unsigned char* sp = q.sz + (blk0 * 16 + (row & 15)) * kSz;
            uint4 w[2][4];                                             // two blocks of 128 columns ahead
            Q4Scales<PER, ZEROS> sc[2];
            auto fetch = [&](int d, int b) {
                if (!live || b >= kb1) return;
#pragma unroll
                for (int c = 0; c < 4; ++c) w[d][c] = __ldg(wp + (size_t)b * 64 + c);
                sc[d].load(sp + (size_t)b * 16 * kSz);
                if (b + 8 < kb1) asm volatile("prefetch.global.L2 [%0];" ::"l"(wp + (size_t)(b + 8) * 64));
            };
            fetch(0, kb0);
            fetch(1, kb0 + 1);
            unsigned long long acc[MP / 2];
#pragma unroll
            for (int i = 0; i < MP / 2; ++i) acc[i] = 0;
            float s_old = 0.f, s_new = 0.f;                            // scales of the two groups in flight
            // the sums of the group two before: out of tensor memory, scaled, added
            auto drain = [&](int u) {
                const int buf = u & 1;
                tc_wait(smem_u32(&d_full[tile * 2 + buf]), (uint32_t)(u >> 1) & 1u, abort_flag, state);
                tc_fence_after();
                const unsigned long long s2 = pair_of(s_old, s_old);
#pragma unroll
                for (int c = 0; c < MP; c += 32) {
                    float v[32];
                    tc_ld32(d_at(tile, buf) + lanes + (uint32_t)c, v);
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[c / 2 + i] = fma2(s2, pair_of(v[2 * i], v[2 * i + 1]), acc[c / 2 + i]);
                }
            };
#pragma unroll 1
            for (int b0 = kb0; b0 < kb1; b0 += 2) {
#pragma unroll
                for (int d = 0; d < 2; ++d) {
                    const int b = b0 + d;
                    if (b >= kb1) break;
#pragma unroll
                    for (int gi = 0; gi < PER; ++gi) {
                        const int g = b * PER + gi;
                        if (g >= groups) break;
                        if (g >= kb0 * PER + 2) drain(unit - 2);
                        s_old = s_new;
                        s_new = live ? sc[d].scale(gi, q.scale_half) : 0.f;
                        // zero points as subnormals, once as they are and once times 16
                        const uint32_t z = (uint32_t)sc[d].zero(gi), z1 = z | z << 16, z16 = z1 << 4;
                        constexpr int kChunks = 4 / PER;
#pragma unroll
                        for (int i = 0; i < kChunks; ++i) {
                            uint32_t r[16];
#pragma unroll
                            for (int c = 0; c < 4; ++c) {
                                const int j = gi * kChunks + i;
                                const uint4 u = w[d][c];
                                uint32_t v[4];
                                q4_spread(j == 0 ? u.x : j == 1 ? u.y : j == 2 ? u.z : u.w, v);
                                r[c * 4] = q4_sub_f16x2(v[0], z1);
                                r[c * 4 + 1] = q4_sub_f16x2(v[1], z16);
                                r[c * 4 + 2] = q4_sub_f16x2(v[2], z1);
                                r[c * 4 + 3] = q4_sub_f16x2(v[3], z16);
                            }
                            tc_st16(a_at(tile, unit & 1) + lanes + (uint32_t)(i * 16), r);
                        }
                        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(&a_full[tile * 2 + (unit & 1)]));
                        ++unit;
                    }
                    fetch(d, b + 2);
                }
            }
            if (min(kb1 * PER, groups) >= kb0 * PER + 2) drain(unit - 2);
            s_old = s_new;
            drain(unit - 1);
            const long long n_row = (long long)t16 * 16 + (row & 15);
            if (pass >= share.full && share.split > 1) {
                float* to = share.part + (size_t)blockIdx.x * MP * 256 + tile * 128 + row;
#pragma unroll
                for (int i = 0; i < MP / 2; ++i) {
                    const float2 f = halves(acc[i]);
                    if (2 * i < M) to[(size_t)(2 * i) * 256] = f.x;
                    if (2 * i + 1 < M) to[(size_t)(2 * i + 1) * 256] = f.y;
                }
            } else if (live && n_row < q.N) {
#pragma unroll
                for (int i = 0; i < MP / 2; ++i) {
                    const float2 f = halves(acc[i]);
                    if (2 * i < M) store_as(out, (size_t)(2 * i) * q.N + n_row, s_back[2 * i](f.x), out_type);
                    if (2 * i + 1 < M) store_as(out, (size_t)(2 * i + 1) * q.N + n_row, s_back[2 * i + 1](f.y), out_type);
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kQ4TcWarps) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
    pdl_launch_dependents();
}

// Adds up the parts of the tail passes, in order.  grid: tail passes x activation rows; 256 threads, one an output row.
__global__ void __launch_bounds__(256) q4_join_kernel(Q4Share share, const int* back, int first_row, int MP, int N, void* __restrict__ out, int out_type) {
    const long long n = first_row + (long long)blockIdx.x * 256 + threadIdx.x;
    pdl_wait();
    if (n >= N) return;
    const float* from = share.part + ((size_t)blockIdx.x * share.split * MP + blockIdx.y) * 256 + threadIdx.x;
    float sum = 0.f;
#pragma unroll 4
    for (int i = 0; i < share.split; ++i) sum += __ldcg(from + (size_t)i * MP * 256);
    store_as(out, (size_t)blockIdx.y * N + n, Q4Power(__ldcg(back + blockIdx.y))(sum), out_type);
}

}  // namespace coral

// Products of few rows with 4-bit weights and group scales (the dense head and the drafter's projections):
//   out[m][n] = sum_g s[n][g] * sum_{k in group g} (q[n][k] - z[n][g]) * x[m][k]
// The sums inside a group run over exact operands on the warp's fp16 MMA with fp32 accumulation, no weight is ever rounded:
// four bits under a mask are a subnormal fp16 number, q 2^-24, so a word becomes operands with five instructions (q under the
// upper mask is 16 times that, which the activations of those columns make good).  What the group's sum then has too much,
// zero point times the sum of the activations, is taken off in fp32 before the scale multiplies it.  Activations come as fp16
// numbers too: a row is scaled by a power of two that brings its largest value to 2^14..2^15, so bf16 rows fit as well.  A value of
// 2^-24 of the row's largest is at least 2^-10, 2^-14 where it is divided by 16, and exact; a smaller one is off by half a
// subnormal step, 2^-25, times 16 at most: 2^-35 of the largest.
// Few rows are bound by the weight bytes, so a weight is read once, straight into registers in the order the MMA wants
// (the packed layout below), with several kilobytes a warp in flight.  One row of 128256 x 4096 takes 56 us (4.8 TB/s, 73% of
// what a copy reaches), 8 rows of 32000 x 4096 with zero points 20.5: a block of columns is a chain of unpacking, MMAs and one
// scaling a group, and 111 registers leave 16 warps a SM to hide it.
//
// Packed layout: [tile of 16 output rows][block of 128 columns][row half][lane][4 words].  Word i of lane (r, c) = (lane / 4,
// lane % 4) holds the 8 columns 32 i + 8 c .. + 7 of row r (first half) or r + 8 (second half), low nibble first.  The MMA's
// k order inside 32 columns is free as long as both operands agree: one word gives the pairs (0,4) (1,5) | (2,6) (3,7) by
// shift and mask, and the activations are staged in that order.  A group of 32 columns is one word a lane, so every group
// size that is a multiple of 32 ends on a word.  Scales (and zero points) follow: [tile][block][16 rows][128 / group].
#pragma once
#include "cp_async.cuh"
#include "element.cuh"

namespace coral {

constexpr int kQ4Warps = 16;                       // largest block: 16 warps
constexpr int kQ4Threads = kQ4Warps * 32;
constexpr int kQ4Depth = 4;                        // column blocks a warp has in flight
constexpr int kQ4PassRows = 16;                    // activation rows of one launch

struct Q4View {
    const uint4* w;                                // packed weights
    const unsigned char* sz;                       // scales (2 bytes) or scale and zero point (4 bytes)
    int N, K, KB, T;                               // T = tiles of 16 rows, KB = blocks of 128 columns
    int scale_half;                                // scales are fp16 (else bf16)
};

// One rounding, to the type the caller asked for (CORAL_TYPE_*).
__device__ __forceinline__ void store_as(void* out, size_t i, float v, int type) {
    if (type == 0) reinterpret_cast<float*>(out)[i] = v;
    else if (type == 1) reinterpret_cast<__nv_bfloat16*>(out)[i] = __float2bfloat16_rn(v);
    else reinterpret_cast<__half*>(out)[i] = __float2half_rn(v);
}

// One thread per 16-byte piece of the packed weights; the first threads of a tile's block also place its scales.
__global__ void q4_pack_kernel(const unsigned char* __restrict__ Wq, const uint16_t* __restrict__ scales,
                               const unsigned char* __restrict__ zeros, int N, int K, int KB, int group, uint4* __restrict__ w,
                               unsigned char* __restrict__ sz, size_t pieces) {
    const size_t piece = (size_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (piece >= pieces) return;
    const int lane = (int)(piece & 31), half = (int)(piece >> 5) & 1;
    const size_t blk = piece >> 6;                 // tile * KB + block
    const int b = (int)(blk % KB);
    const long long row = (long long)(blk / KB) * 16 + half * 8 + (lane >> 2);
    uint32_t word[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int col = b * 128 + 32 * i + 8 * (lane & 3);
        word[i] = row < N && col < K ? *reinterpret_cast<const uint32_t*>(Wq + (size_t)row * (K / 2) + col / 2) : 0x88888888u;
    }
    w[piece] = make_uint4(word[0], word[1], word[2], word[3]);
    const int per = 128 / group, G = K / group;
    const int e = (int)(piece & 63);               // 64 threads a block place its 16 * per entries
    for (int i = e; i < 16 * per; i += 64) {
        const long long r = (long long)(blk / KB) * 16 + i / per;
        const int g = b * per + i % per;
        const bool in = r < N && g < G;
        const uint32_t s = in ? scales[(size_t)r * G + g] : 0;
        const size_t at = blk * 16 * per + i;
        if (zeros) reinterpret_cast<uint32_t*>(sz)[at] = s | (in ? (uint32_t)(zeros[(size_t)r * G + g] & 0x7f) << 16 : 0x80000u);
        else reinterpret_cast<uint16_t*>(sz)[at] = (uint16_t)s;
    }
}

__device__ __forceinline__ void q4_mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// A word's eight weights as four MMA operands: (0,4), 16 (1,5), (2,6), 16 (3,7), in units of 2^-24.
__device__ __forceinline__ void q4_spread(uint32_t w, uint32_t (&v)[4]) {
    v[0] = w & 0x000f000fu;
    v[1] = w & 0x00f000f0u;
    w >>= 8;
    v[2] = w & 0x000f000fu;
    v[3] = w & 0x00f000f0u;
}

// The power of two that brings the largest absolute value (as bits) to 2^14..2^15 (below that, subnormal bf16 numbers: at least
// to 2^8, all of them whole); 1 for a row that is not finite.
__device__ __forceinline__ int q4_exponent(uint32_t max_bits) { return max_bits >= 0x7f800000u ? 0 : 141 - (int)(max_bits >> 23); }
__device__ __forceinline__ float exp2_int(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
// v 2^e for e from -252 to 254: as two factors, since rows of bf16 want exponents from -113 to 141 and those that undo them.
// Neither product leaves the range of fp32 unless the result does.
struct Q4Power {
    float a, b;
    Q4Power() = default;
    __device__ __forceinline__ explicit Q4Power(int e) : a(exp2_int(e / 2)), b(exp2_int(e - e / 2)) {}
    __device__ __forceinline__ float operator()(float v) const { return v * a * b; }
};

// Eight scaled activations in the order of q4_spread.
__device__ __forceinline__ uint4 q4_operand(const float (&f)[8]) {
    uint4 v;
    const __half2 h[4] = {__floats2half2_rn(f[0], f[4]), __floats2half2_rn(f[1] * 0.0625f, f[5] * 0.0625f),
                          __floats2half2_rn(f[2], f[6]), __floats2half2_rn(f[3] * 0.0625f, f[7] * 0.0625f)};
    v.x = *reinterpret_cast<const uint32_t*>(&h[0]);
    v.y = *reinterpret_cast<const uint32_t*>(&h[1]);
    v.z = *reinterpret_cast<const uint32_t*>(&h[2]);
    v.w = *reinterpret_cast<const uint32_t*>(&h[3]);
    return v;
}

// Raw scale entries of one row's block: PER = 128 / group of them, 2 or 4 bytes each, one load.
template <int PER, bool ZEROS> struct Q4Scales {
    static constexpr int kBytes = PER * (ZEROS ? 4 : 2);
    static constexpr int kWords = kBytes < 4 ? 1 : kBytes / 4;
    uint32_t v[kWords];
    __device__ __forceinline__ void load(const unsigned char* p) {
        if constexpr (kBytes == 2) v[0] = __ldg(reinterpret_cast<const uint16_t*>(p));
        else if constexpr (kBytes == 4) v[0] = __ldg(reinterpret_cast<const uint32_t*>(p));
        else if constexpr (kBytes == 8) {
            const uint2 a = __ldg(reinterpret_cast<const uint2*>(p));
            v[0] = a.x; v[1] = a.y;
        } else {
            const uint4 a = __ldg(reinterpret_cast<const uint4*>(p));
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        }
    }
    __device__ __forceinline__ float scale(int g, int half) const {
        const uint32_t u = ZEROS ? v[g] & 0xffffu : (v[g >> 1] >> (16 * (g & 1))) & 0xffffu;
        return half ? __half2float(__ushort_as_half((unsigned short)u)) : __uint_as_float(u << 16);
    }
    __device__ __forceinline__ float zero(int g) const { return ZEROS ? (float)(v[g] >> 16) : 8.f; }
};

// ---- activations ---------------------------------------------------------------------------------------------
// More than a few rows are scaled and laid out once, by a kernel of their own (a block a row), instead of by every block of the
// product.  Two layouts: rows (for q4_rows_kernel, with the group sums) and slabs (for the tensor-core kernel: 64 columns of
// `slab_rows` rows, 128 bytes a row, 16-byte chunks of row r swapped by r % 8 as the 128-byte swizzle has them).
struct Q4Staged {
    int* status;                                   // the call's status word, cleared here, or null
    uint4* x;                                      // rows: [M][KB * 16]; slabs: [ceil(K / 64)][slab_rows][8]
    float* sums;                                   // rows: [M][KB * PER]
    int* back;                                     // the power of two that undoes a row's scale and the weights' 2^-24
};

template <typename TX, int PER>
__global__ void __launch_bounds__(256) q4_stage_kernel(const TX* __restrict__ x, int M, int K, int KB, int slab_rows, Q4Staged st) {
    __shared__ uint32_t s_max[8];
    pdl_launch_dependents();
    const int m = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (st.status && m == 0 && threadIdx.x == 0) *st.status = 0;
    const int chunks = slab_rows ? (K + 63) / 64 * 8 : KB * 16;
    const TX* row = x + (size_t)m * K;             // rows from M on are zeros
    uint32_t top = 0;
    for (int ch = threadIdx.x; ch * 8 < K && m < M; ch += 256) {
        float f[8];
        Elem<TX>::load8(row + ch * 8, f);
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(f[e]) & 0x7fffffffu);
    }
    top = __reduce_max_sync(0xffffffffu, top);
    if (lane == 0) s_max[warp] = top;
    __syncthreads();
    top = s_max[0];
#pragma unroll
    for (int w = 1; w < 8; ++w) top = max(top, s_max[w]);
    const int e2 = q4_exponent(top);
    const Q4Power scale(e2);
    if (threadIdx.x == 0) st.back[m] = 24 - e2;
    for (int c0 = 0; c0 < chunks; c0 += 256) {
        const int ch = c0 + threadIdx.x;
        float f[8] = {}, sum = 0.f;
        if (ch * 8 < K && m < M) Elem<TX>::load8(row + ch * 8, f);
#pragma unroll
        for (int e = 0; e < 8; ++e) { f[e] = scale(f[e]); sum += f[e]; }
        if (slab_rows) {
            if (ch < chunks) st.x[((size_t)(ch >> 3) * slab_rows + m) * 8 + ((ch & 7) ^ (m & 7))] = q4_operand(f);
            continue;
        }
        if (ch < chunks) st.x[(size_t)m * chunks + ch] = q4_operand(f);
#pragma unroll
        for (int o = 1; o < 16 / PER; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (ch < chunks && (ch & (16 / PER - 1)) == 0) st.sums[(size_t)m * KB * PER + ch / (16 / PER)] = sum * 0x1p-24f;
    }
}

// grid: any number of blocks of `warps` warps; `split` warps (a power of two dividing warps) share a tile's columns.
// dynamic shared memory: M rows of x (KB * 256 + 64 bytes each), group sums [KB * PER][8 NT], then 2 * warps * 16 * 8 NT floats.
// Rows of x are padded to 64 bytes past a multiple of 128, so the eight rows of a quarter warp's 16-byte loads fall on
// different banks.  x is read from `st` if it has been laid out there, else each block scales and lays out the few rows itself.
template <typename TX, int NT, int PER, bool ZEROS>
__global__ void __launch_bounds__(kQ4Threads, 1) q4_rows_kernel(Q4View q, const TX* __restrict__ x, Q4Staged st, int M, void* __restrict__ out, int out_type, int split) {
    extern __shared__ __align__(16) unsigned char smem_raw[];
    constexpr int kCols = 8 * NT;
    __shared__ uint32_t s_max[kCols];
    __shared__ Q4Power s_back[kCols];              // what undoes the row's scale and the weights' 2^-24
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int xrow = q.KB * 256 + 64, groups = q.KB * PER;
    unsigned char* xs = smem_raw;
    float* xsum = reinterpret_cast<float*>(smem_raw + (size_t)M * xrow);
    float* red = xsum + (size_t)groups * kCols;
    const int lane_in = warp % split, team = warp / split, teams = warps / split;

    // this warp's stream of (tile, block): tiles tile0, tile0 + step, ..., blocks lane_in, lane_in + split, ...
    const int nb = (q.KB + split - 1) / split;
    const int tile0 = blockIdx.x * teams + team, step = gridDim.x * teams;
    const int tiles = tile0 < q.T ? (q.T - 1 - tile0) / step + 1 : 0;
    const long long total = (long long)tiles * nb;
    constexpr int kSz = Q4Scales<PER, ZEROS>::kBytes;

    uint4 w[kQ4Depth][2];
    Q4Scales<PER, ZEROS> sc[kQ4Depth][2];
    int f_b = lane_in, f_tiles = tiles;
    size_t f_blk = (size_t)tile0 * q.KB + lane_in;             // block of the next fetch, counted over all tiles
    const size_t f_wrap = (size_t)step * q.KB - (size_t)(nb - 1) * split;
    const uint4* const w_lane = q.w + lane;
    const unsigned char* const sz_lane = q.sz + (lane >> 2) * kSz;
    auto fetch = [&](int d) {
        if (f_tiles > 0 && f_b < q.KB) {
            const uint4* p = w_lane + f_blk * 64;
            w[d][0] = __ldcs(p);
            w[d][1] = __ldcs(p + 32);
            const unsigned char* s = sz_lane + f_blk * (16 * kSz);
            sc[d][0].load(s);
            sc[d][1].load(s + 8 * kSz);
        }
        if (f_b + split < nb * split) { f_b += split; f_blk += split; }
        else { f_b = lane_in; f_blk += f_wrap; --f_tiles; }
    };
    // With x laid out by a kernel of this call, that kernel began behind all that came before the call, so the weights may be
    // fetched before its end.  Else the kernel before is the caller's: it may still be writing x or the weights, or reading out.
    if (!st.x) pdl_wait();
#pragma unroll
    for (int d = 0; d < kQ4Depth; ++d) fetch(d);

    const int units = q.KB * 16, all = M * units;
    if (st.x) {
        pdl_wait();                                // the kernel that lays x out
        for (int m = 0; m < M; ++m)
            for (int ch = threadIdx.x; ch < units; ch += blockDim.x)
                cp_async16(xs + (size_t)m * xrow + ch * 16, st.x + (size_t)m * units + ch);
        cp_async_commit();
        for (int i = threadIdx.x; i < groups * kCols; i += blockDim.x) {
            const int m = i % kCols;
            xsum[i] = m < M ? st.sums[(size_t)m * groups + i / kCols] : 0.f;
        }
        if (threadIdx.x < M) s_back[threadIdx.x] = Q4Power(st.back[threadIdx.x]);
        cp_async_wait<0>();
    } else {
        // x, scaled, in the MMA's order, and its sums over the groups (16 neighbouring lanes hold 128 columns)
        if (threadIdx.x < kCols) s_max[threadIdx.x] = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < all; i += blockDim.x) {
            const int m = i / units, ch = i - m * units;
            if (ch * 8 >= q.K) continue;
            float f[8];
            Elem<TX>::load8(x + (size_t)m * q.K + ch * 8, f);
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(f[e]) & 0x7fffffffu);
            if (top > s_max[m]) atomicMax(&s_max[m], top);
        }
        __syncthreads();
        if (threadIdx.x < M) s_back[threadIdx.x] = Q4Power(24 - q4_exponent(s_max[threadIdx.x]));
        for (int i0 = 0; i0 < all; i0 += blockDim.x) {
            const int i = i0 + threadIdx.x, m = i < all ? i / units : 0, ch = i - m * units;
            float f[8] = {}, sum = 0.f;
            if (i < all) {
                if (ch * 8 < q.K) Elem<TX>::load8(x + (size_t)m * q.K + ch * 8, f);
                const Q4Power scale(q4_exponent(s_max[m]));
#pragma unroll
                for (int e = 0; e < 8; ++e) { f[e] = scale(f[e]); sum += f[e]; }
                *reinterpret_cast<uint4*>(xs + (size_t)m * xrow + ch * 16) = q4_operand(f);
            }
#pragma unroll
            for (int o = 1; o < 16 / PER; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if (i < all && (ch & (16 / PER - 1)) == 0) xsum[ch / (16 / PER) * kCols + m] = sum * 0x1p-24f;
        }
    }
    __syncthreads();

    // columns of the result past M are never written: their lanes read row M - 1 (and sums nobody set)
    const unsigned char* xl[NT];
    const float2* const sl = reinterpret_cast<const float2*>(xsum) + (lane & 3);
#pragma unroll
    for (int j = 0; j < NT; ++j) xl[j] = xs + (size_t)min(8 * j + (lane >> 2), M - 1) * xrow + (lane & 3) * 16;
    float acc[NT][4] = {};
    int b = lane_in, at = 0, turn = 0, tile = tile0;
    for (long long base = 0; base < total; base += kQ4Depth) {
#pragma unroll
        for (int d = 0; d < kQ4Depth; ++d) {
            if (base + d >= total) break;
            if (b < q.KB) {
                float part[NT][4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    constexpr int kChunks = 4 / PER;               // 32-column chunks a group has in this block
                    const int g = i / kChunks;
                    if (i % kChunks == 0) {
#pragma unroll
                        for (int j = 0; j < NT; ++j)
#pragma unroll
                            for (int e = 0; e < 4; ++e) part[j][e] = 0.f;
                    }
                    const uint32_t lo = i == 0 ? w[d][0].x : i == 1 ? w[d][0].y : i == 2 ? w[d][0].z : w[d][0].w;
                    const uint32_t hi = i == 0 ? w[d][1].x : i == 1 ? w[d][1].y : i == 2 ? w[d][1].z : w[d][1].w;
                    uint32_t l[4], h[4];
                    q4_spread(lo, l);
                    q4_spread(hi, h);
                    const uint32_t a0[4] = {l[0], h[0], l[1], h[1]}, a1[4] = {l[2], h[2], l[3], h[3]};
#pragma unroll
                    for (int j = 0; j < NT; ++j) {
                        const uint4 v = *reinterpret_cast<const uint4*>(xl[j] + b * 256 + i * 64);
                        q4_mma(part[j], a0, v.x, v.y);
                        q4_mma(part[j], a1, v.z, v.w);
                    }
                    if (i % kChunks == kChunks - 1) {
                        const float s0 = sc[d][0].scale(g, q.scale_half), s1 = sc[d][1].scale(g, q.scale_half);
                        const float z0 = -sc[d][0].zero(g), z1 = -sc[d][1].zero(g);
#pragma unroll
                        for (int j = 0; j < NT; ++j) {
                            const float2 u = sl[(b * PER + g) * (kCols / 2) + 4 * j];
                            acc[j][0] = fmaf(s0, fmaf(z0, u.x, part[j][0]), acc[j][0]);
                            acc[j][1] = fmaf(s0, fmaf(z0, u.y, part[j][1]), acc[j][1]);
                            acc[j][2] = fmaf(s1, fmaf(z1, u.x, part[j][2]), acc[j][2]);
                            acc[j][3] = fmaf(s1, fmaf(z1, u.y, part[j][3]), acc[j][3]);
                        }
                    }
                }
            }
            fetch(d);
            b += split;
            if (++at < nb) continue;
            // the tile is complete: join the team's parts and write 16 outputs of each row
            at = 0;
            b = lane_in;
            float* mine = red + ((size_t)turn * warps + warp) * 16 * kCols;
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const int r = lane >> 2, c = 8 * j + (lane & 3) * 2;
                mine[c * 16 + r] = acc[j][0];
                mine[(c + 1) * 16 + r] = acc[j][1];
                mine[c * 16 + r + 8] = acc[j][2];
                mine[(c + 1) * 16 + r + 8] = acc[j][3];
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[j][e] = 0.f;
            }
            if (split == 1) __syncwarp();
            else asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(split * 32) : "memory");
            const float* first = red + ((size_t)turn * warps + team * split) * 16 * kCols;
            for (int e = lane_in * 32 + lane; e < 16 * M; e += split * 32) {
                float s = 0.f;
                for (int p = 0; p < split; ++p) s += first[(size_t)p * 16 * kCols + e];
                const long long n = (long long)tile * 16 + (e & 15);
                if (n < q.N) store_as(out, (size_t)(e >> 4) * q.N + n, s_back[e >> 4](s), out_type);
            }
            turn ^= 1;
            tile += step;
        }
    }
}

}  // namespace coral

// Products of few rows with 4-bit weights and group scales (the dense head and the drafter's projections):
//   out[m][n] = sum_g s[n][g] * sum_{k in group g} (q[n][k] - z[n][g]) * x[m][k]
// The sums inside a group run over exact operands: q - z is a small integer, exact in bf16 and fp16, so a warp MMA of
// integers and activations accumulates in fp32 with no rounded weight, and the scale multiplies the group's fp32 sum.
// Few rows are bound by the weight bytes, so a weight is read once, straight into registers in the order the MMA wants
// (the packed layout below), with several kilobytes a warp in flight.
//
// Packed layout: [tile of 16 output rows][block of 128 columns][row half][lane][4 words].  Word i of lane (r, c) = (lane / 4,
// lane % 4) holds the 8 columns 32 i + 8 c .. + 7 of row r (first half) or r + 8 (second half), low nibble first.  The MMA's
// k order inside 32 columns is free as long as both operands agree: one word gives the pairs (0,4) (1,5) | (2,6) (3,7) by
// shift and mask, and the activations are staged in that order.  A group of 32 columns is one word a lane, so every group
// size that is a multiple of 32 ends on a word.  Scales (and zero points) follow: [tile][block][16 rows][128 / group].
#pragma once
#include "element.cuh"

namespace coral {

constexpr int kQ4Warps = 16;                       // largest block: 16 warps
constexpr int kQ4Threads = kQ4Warps * 32;
constexpr int kQ4Depth = 4;                        // column blocks a warp has in flight
constexpr int kQ4PassRows = 16;                    // activation rows of one launch

__host__ __device__ __forceinline__ size_t q4_tile_bytes(int KB) { return (size_t)KB * 1024; }

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

template <typename T> struct Q4Num;
template <> struct Q4Num<__nv_bfloat16> {
    static constexpr uint32_t kMagic = 0x43004300u;     // 128 + q, q < 128, is exact
    static __device__ __forceinline__ uint32_t sub(uint32_t a, uint32_t z) {
        uint32_t d;
        asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(z));
        return d;
    }
    static __device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
};
template <> struct Q4Num<__half> {
    static constexpr uint32_t kMagic = 0x64006400u;     // 1024 + q
    static __device__ __forceinline__ uint32_t sub(uint32_t a, uint32_t z) {
        uint32_t d;
        asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(z));
        return d;
    }
    static __device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
};

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
    __device__ __forceinline__ uint32_t zero(int g) const {            // the zero point in both halves
        if (!ZEROS) return 0x00080008u;
        return __byte_perm(v[g], 0, 0x3232);
    }
};

// grid: any number of blocks of `warps` warps; `split` warps (a power of two dividing warps) share a tile's columns.
// dynamic shared memory: M rows of x (KB * 256 + 64 bytes each), then 2 * warps * 16 * 8 NT floats.
// Rows of x are padded to 64 bytes past a multiple of 128, so the eight rows of a quarter warp's 16-byte loads fall on
// different banks.
template <typename TX, int NT, int PER, bool ZEROS>
__global__ void __launch_bounds__(kQ4Threads, 1) q4_rows_kernel(Q4View q, const TX* __restrict__ x, int M, void* __restrict__ out, int out_type, int split) {
    extern __shared__ __align__(16) unsigned char smem_raw[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int xrow = q.KB * 256 + 64;
    unsigned char* xs = smem_raw;
    float* red = reinterpret_cast<float*>(smem_raw + (size_t)M * xrow);
    const int lane_in = warp % split, team = warp / split, teams = warps / split;

    // this warp's stream of (tile, block): tiles tile0, tile0 + step, ..., blocks lane_in, lane_in + split, ...
    const int nb = (q.KB + split - 1) / split;
    const int tile0 = blockIdx.x * teams + team, step = gridDim.x * teams;
    const int tiles = tile0 < q.T ? (q.T - 1 - tile0) / step + 1 : 0;
    const long long total = (long long)tiles * nb;
    constexpr int kSz = Q4Scales<PER, ZEROS>::kBytes;

    uint4 w[kQ4Depth][2];
    Q4Scales<PER, ZEROS> sc[kQ4Depth][2];
    int f_tile = tile0, f_b = lane_in, f_i = 0;
    long long f_at = 0;
    auto fetch = [&](int d) {
        if (f_at < total && f_b < q.KB) {
            const size_t blk = (size_t)f_tile * q.KB + f_b;
            const uint4* p = q.w + blk * 64 + lane;
            w[d][0] = __ldcs(p);
            w[d][1] = __ldcs(p + 32);
            const unsigned char* s = q.sz + (blk * 16 + (lane >> 2)) * kSz;
            sc[d][0].load(s);
            sc[d][1].load(s + 8 * kSz);
        }
        ++f_at;
        f_b += split;
        if (++f_i == nb) { f_i = 0; f_b = lane_in; f_tile += step; }
    };
#pragma unroll
    for (int d = 0; d < kQ4Depth; ++d) fetch(d);

    // x in the MMA's order, 8 columns (16 bytes) at a time: 0 4 1 5 2 6 3 7; zero past K
    for (int i = threadIdx.x; i < M * q.KB * 16; i += blockDim.x) {
        const int m = i / (q.KB * 16), ch = i - m * (q.KB * 16);
        uint4 v = make_uint4(0, 0, 0, 0);
        if (ch * 8 < q.K) v = __ldg(reinterpret_cast<const uint4*>(x + (size_t)m * q.K) + ch);
        *reinterpret_cast<uint4*>(xs + (size_t)m * xrow + ch * 16) =
            make_uint4(__byte_perm(v.x, v.z, 0x5410), __byte_perm(v.x, v.z, 0x7632), __byte_perm(v.y, v.w, 0x5410),
                       __byte_perm(v.y, v.w, 0x7632));
    }
    __syncthreads();

    const int n_row = lane >> 2;
    const unsigned char* xl[NT];
    bool live[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        live[j] = 8 * j + n_row < M;
        xl[j] = xs + (size_t)(live[j] ? 8 * j + n_row : 0) * xrow + (lane & 3) * 16;
    }
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
                    const uint32_t zl = Q4Num<TX>::kMagic | sc[d][0].zero(g), zh = Q4Num<TX>::kMagic | sc[d][1].zero(g);
                    uint32_t a[2][4];
#pragma unroll
                    for (int p = 0; p < 4; ++p) {
                        a[p >> 1][(p & 1) * 2] = Q4Num<TX>::sub(((lo >> (4 * p)) & 0x000f000fu) | Q4Num<TX>::kMagic, zl);
                        a[p >> 1][(p & 1) * 2 + 1] = Q4Num<TX>::sub(((hi >> (4 * p)) & 0x000f000fu) | Q4Num<TX>::kMagic, zh);
                    }
#pragma unroll
                    for (int j = 0; j < NT; ++j) {
                        uint4 v = make_uint4(0, 0, 0, 0);
                        if (live[j]) v = *reinterpret_cast<const uint4*>(xl[j] + b * 256 + i * 64);
                        Q4Num<TX>::mma(part[j], a[0], v.x, v.y);
                        Q4Num<TX>::mma(part[j], a[1], v.z, v.w);
                    }
                    if (i % kChunks == kChunks - 1) {
                        const float s0 = sc[d][0].scale(g, q.scale_half), s1 = sc[d][1].scale(g, q.scale_half);
#pragma unroll
                        for (int j = 0; j < NT; ++j) {
                            acc[j][0] = fmaf(s0, part[j][0], acc[j][0]);
                            acc[j][1] = fmaf(s0, part[j][1], acc[j][1]);
                            acc[j][2] = fmaf(s1, part[j][2], acc[j][2]);
                            acc[j][3] = fmaf(s1, part[j][3], acc[j][3]);
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
            constexpr int kCols = 8 * NT;
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
                if (n < q.N) store_as(out, (size_t)(e >> 4) * q.N + n, s, out_type);
            }
            turn ^= 1;
            tile += step;
        }
    }
}

}  // namespace coral

// Norms before and after a block, fused with its gate and residual scale, and their gradient: the step that makes the
// hidden rows the draft head reads (row m, columns c, all sums in fp32):
//   b = w_post ? x / sqrt(mean x^2 + eps) * w_post : x       norm behind the block
//   y = alpha r + gate b                                      residual stream
//   h = y / sqrt(mean y^2 + eps) * w_pre                      norm in front of the next block or of the head
// y feeds the second norm unrounded.  Both directions are bound by the bytes of the rows (4 resp. 6 tensors), so a row
// is read once: a block owns a row, a thread owns the same 8-column chunks of every row, and the weights stay in its
// registers.  A thread copies its own chunks of the next rows into its own shared-memory slots with cp.async, so the
// loads run ahead of the reductions without registers and without a barrier (only the row sums need one).
// bf16 with both norms and a gate a column: 16384 x 4096 forward 108-113 us (4.95 TB/s; bound by issue slots, 67% of them used,
// and by the two row sums; 64 registers a thread, 64 bytes more spilled), gradient of 8192 x 4096 124 us (3.2 TB/s; three column
// sums of 16 columns a thread take the registers, 16 warps a SM are left to hide three row sums in turn.  All three are kept
// even where two of them are one: with S = sum dY xh, a gate a column has dgate = w_post S and dw_post = gate S).  fp32: forward
// of 8192 x 4096 117 us, gradient of 4096 x 4096 110.  Rows of more than 8192 columns in 16 bits take four chunks a thread, and
// their gradient spills 490 bytes: 2048 x 16384 bf16 210 us (forward of 4096 rows 124).
#pragma once
#include "cp_async.cuh"
#include "element.cuh"

namespace coral {

constexpr int kNormMaxThreads = 512;
constexpr int kNormMaxRowBytes = 32768;             // H * element size: five staged rows fit shared memory
constexpr int kNormWarps = kNormMaxThreads / 32;

// Gate modes: 0 none, 1 one value a column, 2 one value a row, 3 one value an element.
struct NormArgs {
    int M, H, gate_mode;
    float alpha, eps;
    const void *x, *r, *gate, *w_post, *w_pre;      // r, gate, w_post, w_pre may be null
    void *y, *h;                                    // forward outputs (h null when w_pre is)
    const void *dy, *dh;                            // backward: either may be null
    void *dx, *dr, *dgate;                          // dr null when r is; dgate: modes 2 (fp32) and 3 (element type)
    float* part;                                    // [grid][3][H] column sums: w_pre, w_post, gate (backward)
    int want;                                       // ... bits 0 to 2: which of them
};

// All but the newest `left` groups have arrived (left is uniform and at most 3).
__device__ __forceinline__ void cp_async_wait_left(int left) {
    if (left == 0) cp_async_wait<0>();
    else if (left == 1) cp_async_wait<1>();
    else if (left == 2) cp_async_wait<2>();
    else cp_async_wait<3>();
}

// Sums over the block, the same bits in every thread and on every run: a shuffle tree a warp, then the warps' sums in order.
// `turn` alternates between two buffers, so one barrier a sum is enough: a buffer is written again only behind the barrier of
// the sum in between.  The buffers start as zeros, and warps that do not exist stay zero.
struct NormSums {
    float4 a[2][kNormWarps / 4], b[2][kNormWarps / 4];
};
__device__ __forceinline__ float sum_warps(const float4 (&v)[kNormWarps / 4]) {
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < kNormWarps / 4; ++i) t += (v[i].x + v[i].y) + (v[i].z + v[i].w);
    return t;
}
__device__ __forceinline__ float block_sum(float a, NormSums& s, int& turn) {
    a = warp_sum(a);
    if ((threadIdx.x & 31) == 0) reinterpret_cast<float*>(s.a[turn])[threadIdx.x >> 5] = a;
    __syncthreads();
    a = sum_warps(s.a[turn]);
    turn ^= 1;
    return a;
}
__device__ __forceinline__ void block_sum2(float& a, float& b, NormSums& s, int& turn) {
    a = warp_sum(a);
    b = warp_sum(b);
    if ((threadIdx.x & 31) == 0) {
        reinterpret_cast<float*>(s.a[turn])[threadIdx.x >> 5] = a;
        reinterpret_cast<float*>(s.b[turn])[threadIdx.x >> 5] = b;
    }
    __syncthreads();
    a = sum_warps(s.a[turn]);
    b = sum_warps(s.b[turn]);
    turn ^= 1;
}
__device__ __forceinline__ void clear_sums(NormSums& s) {
    for (int i = threadIdx.x; i < (int)(sizeof(s) / 4); i += blockDim.x) reinterpret_cast<float*>(&s)[i] = 0.f;
    __syncthreads();
}

// Eight elements as they lie in memory, widened where they are used (weights wait in registers this way).
template <typename T> struct Raw8 {
    uint4 v[sizeof(T) / 2];
    __device__ __forceinline__ void load(const void* p, int ch) {
        const uint4* q = reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(p) + (size_t)ch * 8);
#pragma unroll
        for (int i = 0; i < (int)(sizeof(T) / 2); ++i) v[i] = __ldg(q + i);
    }
    __device__ __forceinline__ V8 get() const { return load8v(reinterpret_cast<const T*>(v)); }
};

// Staged tensors of one row: x, then r, then (backward) dy, dh, then a full gate; absent ones are not staged.
template <typename T, int NV>
struct NormStage {
    static constexpr int kChunkBytes = 8 * (int)sizeof(T);
    unsigned char* base;                            // [stage][tensor][NV][threads] chunks
    int tensors, chunks;

    __device__ __forceinline__ T* slot(int stage, int tensor, int i) const {
        return reinterpret_cast<T*>(base + ((((size_t)stage * tensors + tensor) * NV + i) * blockDim.x + threadIdx.x) * kChunkBytes);
    }
    __device__ __forceinline__ void copy(int stage, int tensor, const void* src, size_t row, int H) const {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int ch = threadIdx.x + i * blockDim.x;
            if (ch < chunks) {
                const T* p = reinterpret_cast<const T*>(src) + row * H + (size_t)ch * 8;
                T* d = slot(stage, tensor, i);
#pragma unroll
                for (int o = 0; o < kChunkBytes; o += 16)
                    cp_async16(reinterpret_cast<unsigned char*>(d) + o, reinterpret_cast<const unsigned char*>(p) + o);
            }
        }
    }
};

// grid: any; dynamic shared memory: stages * tensors * NV * blockDim * 8 elements.
template <typename T, int NV>
__global__ void __launch_bounds__(kNormMaxThreads, NV < 4 ? 2 : 1) block_norm_kernel(NormArgs a, int stages) {
    extern __shared__ __align__(16) unsigned char smem_raw[];
    __shared__ NormSums s_sum;
    const int H = a.H, chunks = H >> 3;
    const int t_r = a.r ? 1 : -1, t_g = a.gate_mode == 3 ? 1 + (a.r ? 1 : 0) : -1;
    const NormStage<T, NV> st{smem_raw, 1 + (a.r ? 1 : 0) + (a.gate_mode == 3 ? 1 : 0), chunks};
    auto fetch = [&](int stage, size_t row) {
        st.copy(stage, 0, a.x, row, H);
        if (t_r >= 0) st.copy(stage, t_r, a.r, row, H);
        if (t_g >= 0) st.copy(stage, t_g, a.gate, row, H);
    };
    for (int s = 0; s < stages; ++s) {              // one group a stage, empty past the last row
        const size_t row = blockIdx.x + (size_t)s * gridDim.x;
        if (row < (size_t)a.M) fetch(s, row);
        cp_async_commit();
    }
    Raw8<T> w_post[NV], w_pre[NV], w_gate[NV];      // the weights of this thread's columns
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int ch = threadIdx.x + i * blockDim.x;
        if (ch >= chunks) continue;
        if (a.w_post) w_post[i].load(a.w_post, ch);
        if (a.w_pre) w_pre[i].load(a.w_pre, ch);
        if (a.gate_mode == 1) w_gate[i].load(a.gate, ch);
    }
    clear_sums(s_sum);
    int turn = 0, stage = 0;
    const float inv_h = 1.f / (float)H;
    for (size_t row = blockIdx.x; row < (size_t)a.M; row += gridDim.x) {
        cp_async_wait_left(stages - 1);
        V8 y[NV];                                   // first x, then y
        float scale = a.gate_mode == 2 ? Elem<T>::up(reinterpret_cast<const T*>(a.gate)[row]) : 1.f;
        unsigned long long sx = 0, sy = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (threadIdx.x + i * blockDim.x >= chunks) continue;
            y[i] = load8v(st.slot(stage, 0, i));
            sx = dot8v(y[i], y[i], sx);
        }
        if (a.w_post) {
            const float2 s = halves(sx);
            scale *= rsqrtf(fmaf(block_sum(s.x + s.y, s_sum, turn), inv_h, a.eps));
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int ch = threadIdx.x + i * blockDim.x;
            if (ch >= chunks) continue;
            if (a.w_post || a.gate_mode == 2) y[i] = y[i] * splat8(scale);
            if (a.w_post) y[i] = y[i] * w_post[i].get();
            if (a.gate_mode == 1) y[i] = y[i] * w_gate[i].get();
            if (a.gate_mode == 3) y[i] = y[i] * load8v(st.slot(stage, t_g, i));
            if (t_r >= 0) y[i] = fma8(splat8(a.alpha), load8v(st.slot(stage, t_r, i)), y[i]);
            sy = dot8v(y[i], y[i], sy);
            if (a.y) store8v(reinterpret_cast<T*>(a.y) + row * H + (size_t)ch * 8, y[i]);
        }
        // this thread's slots of the stage have been read: the row `stages` turns ahead may come in
        const size_t next = row + (size_t)stages * gridDim.x;
        if (next < (size_t)a.M) fetch(stage, next);
        cp_async_commit();
        stage = stage + 1 == stages ? 0 : stage + 1;
        if (!a.h) continue;
        const float2 s = halves(sy);
        const V8 ry = splat8(rsqrtf(fmaf(block_sum(s.x + s.y, s_sum, turn), inv_h, a.eps)));
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int ch = threadIdx.x + i * blockDim.x;
            if (ch >= chunks) continue;
            store8v(reinterpret_cast<T*>(a.h) + row * H + (size_t)ch * 8, y[i] * ry * w_pre[i].get());
        }
    }
}

// Backward, with xh = x / sqrt(mean x^2 + eps), yh likewise, b = w_post ? xh w_post : x, y recomputed as above:
//   dY = dy + ry (dh w_pre - yh mean(dh w_pre yh));  dr = alpha dY;  db = gate dY;  dgate = dY b (summed as the gate is shared)
//   dx = w_post ? rx (db w_post - xh mean(db w_post xh)) : db;  dw_pre = sum_m dh yh;  dw_post = sum_m db xh
// The sums over rows go through a fixed order: each block adds its rows in turn in registers and writes one partial row,
// block_norm_columns_kernel adds the partial rows; no atomics, so the same call gives the same bits.
template <typename T, int NV>
__global__ void __launch_bounds__(kNormMaxThreads) block_norm_backward_kernel(NormArgs a, int stages) {
    extern __shared__ __align__(16) unsigned char smem_raw[];
    __shared__ NormSums s_sum;
    const int H = a.H, chunks = H >> 3;
    int n_t = 1;
    const int t_r = a.r ? n_t++ : -1, t_dy = a.dy ? n_t++ : -1, t_dh = a.dh ? n_t++ : -1, t_g = a.gate_mode == 3 ? n_t++ : -1;
    const NormStage<T, NV> st{smem_raw, n_t, chunks};
    auto fetch = [&](int stage, size_t row) {
        st.copy(stage, 0, a.x, row, H);
        if (t_r >= 0) st.copy(stage, t_r, a.r, row, H);
        if (t_dy >= 0) st.copy(stage, t_dy, a.dy, row, H);
        if (t_dh >= 0) st.copy(stage, t_dh, a.dh, row, H);
        if (t_g >= 0) st.copy(stage, t_g, a.gate, row, H);
    };
    for (int s = 0; s < stages; ++s) {
        const size_t row = blockIdx.x + (size_t)s * gridDim.x;
        if (row < (size_t)a.M) fetch(s, row);
        cp_async_commit();
    }
    V8 acc_pre[NV] = {}, acc_post[NV] = {}, acc_gate[NV] = {};
    // weights come from L1 wherever they are used: the column sums take the registers
    auto weights = [&](const void* w, int i) {
        Raw8<T> r;
        r.load(w, threadIdx.x + i * blockDim.x);
        return r.get();
    };
    clear_sums(s_sum);
    int turn = 0, stage = 0;
    const float inv_h = 1.f / (float)H;
    for (size_t row = blockIdx.x; row < (size_t)a.M; row += gridDim.x) {
        cp_async_wait_left(stages - 1);
        float rx = 1.f;
        if (a.w_post) {
            unsigned long long sx = 0;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (threadIdx.x + i * blockDim.x >= chunks) continue;
                const V8 x = load8v(st.slot(stage, 0, i));
                sx = dot8v(x, x, sx);
            }
            const float2 s = halves(sx);
            rx = rsqrtf(fmaf(block_sum(s.x + s.y, s_sum, turn), inv_h, a.eps));
        }
        const float g_row = a.gate_mode == 2 ? Elem<T>::up(reinterpret_cast<const T*>(a.gate)[row]) : 1.f;
        // v times the gate
        auto gated = [&](const V8& v, int i) {
            if (a.gate_mode == 1) return v * weights(a.gate, i);
            if (a.gate_mode == 2) return v * splat8(g_row);
            if (a.gate_mode == 3) return v * load8v(st.slot(stage, t_g, i));
            return v;
        };
        V8 y[NV], b[NV];
        unsigned long long sy = 0, sd = 0;          // sum y^2, sum dh w_pre y
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (threadIdx.x + i * blockDim.x >= chunks) continue;
            b[i] = load8v(st.slot(stage, 0, i));
            if (a.w_post) b[i] = b[i] * splat8(rx) * weights(a.w_post, i);
            y[i] = gated(b[i], i);
            if (t_r >= 0) y[i] = fma8(splat8(a.alpha), load8v(st.slot(stage, t_r, i)), y[i]);
            if (t_dh >= 0) {
                sy = dot8v(y[i], y[i], sy);
                sd = dot8v(load8v(st.slot(stage, t_dh, i)) * weights(a.w_pre, i), y[i], sd);
            }
        }
        float ry = 0.f, mean = 0.f;                 // mean of dh w_pre yh, times ry
        if (t_dh >= 0) {
            const float2 u = halves(sy), v = halves(sd);
            float s0 = u.x + u.y, s1 = v.x + v.y;
            block_sum2(s0, s1, s_sum, turn);
            ry = rsqrtf(fmaf(s0, inv_h, a.eps));
            mean = s1 * ry * inv_h;
        }
        unsigned long long sb = 0, sg = 0;          // sum db w_post x, sum dY b
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int ch = threadIdx.x + i * blockDim.x;
            if (ch >= chunks) continue;
            V8 d = {};
            if (t_dy >= 0) d = load8v(st.slot(stage, t_dy, i));
            if (t_dh >= 0) {
                const V8 dh = load8v(st.slot(stage, t_dh, i)), yh = y[i] * splat8(ry);
                acc_pre[i] = fma8(dh, yh, acc_pre[i]);
                d = fma8(splat8(ry), fma8(yh, splat8(-mean), dh * weights(a.w_pre, i)), d);
            }
            if (a.dr) store8v(reinterpret_cast<T*>(a.dr) + row * H + (size_t)ch * 8, d * splat8(a.alpha));
            if (a.gate_mode == 1) acc_gate[i] = fma8(d, b[i], acc_gate[i]);
            else if (a.gate_mode == 2) sg = dot8v(d, b[i], sg);
            else if (a.gate_mode == 3 && a.dgate) store8v(reinterpret_cast<T*>(a.dgate) + row * H + (size_t)ch * 8, d * b[i]);
            y[i] = gated(d, i);                     // from here on: db, times w_post if there is one
            if (a.w_post) {
                const V8 x = load8v(st.slot(stage, 0, i));
                acc_post[i] = fma8(y[i], x * splat8(rx), acc_post[i]);
                y[i] = y[i] * weights(a.w_post, i);
                sb = dot8v(y[i], x, sb);
                b[i] = x;                           // ... and x
            } else store8v(reinterpret_cast<T*>(a.dx) + row * H + (size_t)ch * 8, y[i]);
        }
        const size_t next = row + (size_t)stages * gridDim.x;
        if (next < (size_t)a.M) fetch(stage, next);
        cp_async_commit();
        stage = stage + 1 == stages ? 0 : stage + 1;
        if (!a.w_post && a.gate_mode != 2) continue;
        const float2 u = halves(sb), v = halves(sg);
        float s0 = u.x + u.y, s1 = v.x + v.y;
        block_sum2(s0, s1, s_sum, turn);
        if (a.gate_mode == 2 && a.dgate && threadIdx.x == 0) reinterpret_cast<float*>(a.dgate)[row] = s1;
        if (!a.w_post) continue;
        const V8 back = splat8(-s0 * rx * rx * inv_h);          // minus the mean of db w_post xh, times rx
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int ch = threadIdx.x + i * blockDim.x;
            if (ch >= chunks) continue;
            store8v(reinterpret_cast<T*>(a.dx) + row * H + (size_t)ch * 8, splat8(rx) * fma8(b[i], back, y[i]));
        }
    }
    float* part = a.part + (size_t)blockIdx.x * 3 * H;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int ch = threadIdx.x + i * blockDim.x;
        if (ch >= chunks) continue;
        if (a.want & 1) store8v(part + (size_t)ch * 8, acc_pre[i]);
        if (a.want & 2) store8v(part + H + (size_t)ch * 8, acc_post[i]);
        if (a.want & 4) store8v(part + 2 * H + (size_t)ch * 8, acc_gate[i]);
    }
    pdl_launch_dependents();
}

// Column sums of the partial rows [n][3][H]: a block takes 32 columns, its warps every sixteenth partial row.
constexpr int kNormColWarps = 16;
__global__ void __launch_bounds__(kNormColWarps * 32) block_norm_columns_kernel(const float* __restrict__ part, int n, int H,
                                                                               float* d_w_pre, float* d_w_post, float* d_gate) {
    __shared__ float s[kNormColWarps][32];
    float* out = blockIdx.y == 0 ? d_w_pre : blockIdx.y == 1 ? d_w_post : d_gate;
    if (!out) return;
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int col = blockIdx.x * 32 + lane;
    float acc = 0.f;
    if (col < H) {
        const float* p = part + (size_t)blockIdx.y * H + col;
#pragma unroll 8
        for (int i = warp; i < n; i += kNormColWarps) acc += p[(size_t)i * 3 * H];
    }
    s[warp][lane] = acc;
    __syncthreads();
    if (warp == 0 && col < H) {
#pragma unroll
        for (int w = 1; w < kNormColWarps; ++w) acc += s[w][lane];
        out[col] = acc;
    }
}

}  // namespace coral

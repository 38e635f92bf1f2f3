// Norms before and after a block, fused with its gate and residual scale, and their gradient: the step that makes the
// hidden rows the draft head reads (row m, columns c, all sums in fp32):
//   b = w_post ? x / sqrt(mean x^2 + eps) * w_post : x       norm behind the block
//   y = alpha r + gate b                                      residual stream
//   h = y / sqrt(mean y^2 + eps) * w_pre                      norm in front of the next block or of the head
// y feeds the second norm unrounded.  Both directions are bound by the bytes of the rows (4 resp. 6 tensors), so a row
// is read once: a block owns a row, a thread owns the same 8-column chunks of every row, and the weights stay in its
// registers.  A thread copies its own chunks of the next rows into its own shared-memory slots with cp.async, so the
// loads run ahead of the reductions without registers and without a barrier (only the row sums need one).
#pragma once
#include "element.cuh"

namespace coral {

constexpr int kNormMaxThreads = 512;
constexpr int kNormMaxNV = 4;                       // chunks of 8 columns per thread: H <= 512 * 4 * 8
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

__device__ __forceinline__ void cp_async16(void* dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
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
    __device__ __forceinline__ void get(float (&f)[8]) const { Elem<T>::load8(reinterpret_cast<const T*>(v), f); }
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

template <typename T>
__device__ __forceinline__ void load_weights8(const void* w, int ch, float (&v)[8]) {
    if (w) Elem<T>::load8(reinterpret_cast<const T*>(w) + (size_t)ch * 8, v);
    else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = 1.f;
    }
}

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
        float y[NV][8];                             // first x, then y
        float sx = 0.f, sy = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (threadIdx.x + i * blockDim.x >= chunks) continue;
            Elem<T>::load8(st.slot(stage, 0, i), y[i]);
#pragma unroll
            for (int j = 0; j < 8; ++j) sx = fmaf(y[i][j], y[i][j], sx);
        }
        float scale = a.gate_mode == 2 ? Elem<T>::up(reinterpret_cast<const T*>(a.gate)[row]) : 1.f;
        if (a.w_post) scale *= rsqrtf(fmaf(block_sum(sx, s_sum, turn), inv_h, a.eps));
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int ch = threadIdx.x + i * blockDim.x;
            if (ch >= chunks) continue;
            float f[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) y[i][j] *= scale;
            if (a.w_post) {
                w_post[i].get(f);
#pragma unroll
                for (int j = 0; j < 8; ++j) y[i][j] *= f[j];
            }
            if (a.gate_mode == 1 || a.gate_mode == 3) {
                if (a.gate_mode == 1) w_gate[i].get(f);
                else Elem<T>::load8(st.slot(stage, t_g, i), f);
#pragma unroll
                for (int j = 0; j < 8; ++j) y[i][j] *= f[j];
            }
            if (t_r >= 0) {
                Elem<T>::load8(st.slot(stage, t_r, i), f);
#pragma unroll
                for (int j = 0; j < 8; ++j) y[i][j] = fmaf(a.alpha, f[j], y[i][j]);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) sy = fmaf(y[i][j], y[i][j], sy);
            if (a.y) Elem<T>::store8(reinterpret_cast<T*>(a.y) + row * H + (size_t)ch * 8, y[i]);
        }
        // this thread's slots of the stage have been read: the row `stages` turns ahead may come in
        const size_t next = row + (size_t)stages * gridDim.x;
        if (next < (size_t)a.M) fetch(stage, next);
        cp_async_commit();
        stage = stage + 1 == stages ? 0 : stage + 1;
        if (!a.h) continue;
        const float ry = rsqrtf(fmaf(block_sum(sy, s_sum, turn), inv_h, a.eps));
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int ch = threadIdx.x + i * blockDim.x;
            if (ch >= chunks) continue;
            float f[8];
            w_pre[i].get(f);
#pragma unroll
            for (int j = 0; j < 8; ++j) y[i][j] = y[i][j] * ry * f[j];
            Elem<T>::store8(reinterpret_cast<T*>(a.h) + row * H + (size_t)ch * 8, y[i]);
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
    float acc_pre[NV][8] = {}, acc_post[NV][8] = {}, acc_gate[NV][8] = {};
    clear_sums(s_sum);
    int turn = 0, stage = 0;
    const float inv_h = 1.f / (float)H;
    for (size_t row = blockIdx.x; row < (size_t)a.M; row += gridDim.x) {
        cp_async_wait_left(stages - 1);
        float sx = 0.f;
        float rx = 1.f;
        if (a.w_post) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (threadIdx.x + i * blockDim.x >= chunks) continue;
                float x[8];
                Elem<T>::load8(st.slot(stage, 0, i), x);
#pragma unroll
                for (int j = 0; j < 8; ++j) sx = fmaf(x[j], x[j], sx);
            }
            rx = rsqrtf(fmaf(block_sum(sx, s_sum, turn), inv_h, a.eps));
        }
        const float g_row = a.gate_mode == 2 ? Elem<T>::up(reinterpret_cast<const T*>(a.gate)[row]) : 1.f;
        auto gate8 = [&](int i, int ch, float (&g)[8]) {
            if (a.gate_mode == 3) Elem<T>::load8(st.slot(stage, t_g, i), g);
            else if (a.gate_mode == 1) load_weights8<T>(a.gate, ch, g);
            else {
#pragma unroll
                for (int j = 0; j < 8; ++j) g[j] = g_row;
            }
        };
        float y[NV][8], b[NV][8];
        float sy = 0.f, sd = 0.f;                   // sum y^2, sum dh w_pre y
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int ch = threadIdx.x + i * blockDim.x;
            if (ch >= chunks) continue;
            float x[8], r[8], g[8], w[8], dh[8];
            Elem<T>::load8(st.slot(stage, 0, i), x);
            if (t_r >= 0) Elem<T>::load8(st.slot(stage, t_r, i), r);
            gate8(i, ch, g);
            load_weights8<T>(a.w_post, ch, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                b[i][j] = x[j] * rx * w[j];
                y[i][j] = t_r >= 0 ? fmaf(a.alpha, r[j], g[j] * b[i][j]) : g[j] * b[i][j];
            }
            if (t_dh >= 0) {
                Elem<T>::load8(st.slot(stage, t_dh, i), dh);
                load_weights8<T>(a.w_pre, ch, w);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    sy = fmaf(y[i][j], y[i][j], sy);
                    sd = fmaf(dh[j] * w[j], y[i][j], sd);
                }
            }
        }
        float ry = 0.f, mean = 0.f;                 // mean of dh w_pre yh, times ry
        if (t_dh >= 0) {
            block_sum2(sy, sd, s_sum, turn);
            ry = rsqrtf(fmaf(sy, inv_h, a.eps));
            mean = sd * ry * inv_h;
        }
        float sb = 0.f, sg = 0.f;                   // sum db w_post x, sum dY b
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int ch = threadIdx.x + i * blockDim.x;
            if (ch >= chunks) continue;
            float d[8] = {}, w[8], g[8];
            if (t_dy >= 0) Elem<T>::load8(st.slot(stage, t_dy, i), d);
            if (t_dh >= 0) {
                float dh[8];
                Elem<T>::load8(st.slot(stage, t_dh, i), dh);
                load_weights8<T>(a.w_pre, ch, w);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float yh = y[i][j] * ry;
                    acc_pre[i][j] = fmaf(dh[j], yh, acc_pre[i][j]);
                    d[j] = fmaf(ry, fmaf(-yh, mean, dh[j] * w[j]), d[j]);
                }
            }
            if (a.dr) {
                float o[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = a.alpha * d[j];
                Elem<T>::store8(reinterpret_cast<T*>(a.dr) + row * H + (size_t)ch * 8, o);
            }
            gate8(i, ch, g);
            if (a.gate_mode == 3 && a.dgate) {
                float o[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = d[j] * b[i][j];
                Elem<T>::store8(reinterpret_cast<T*>(a.dgate) + row * H + (size_t)ch * 8, o);
            }
            float x[8];
            Elem<T>::load8(st.slot(stage, 0, i), x);
            load_weights8<T>(a.w_post, ch, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float db = g[j] * d[j];
                sg = fmaf(d[j], b[i][j], sg);
                acc_gate[i][j] = fmaf(d[j], b[i][j], acc_gate[i][j]);
                acc_post[i][j] = fmaf(db, x[j] * rx, acc_post[i][j]);
                y[i][j] = db * w[j];                // from here on: db w_post
                sb = fmaf(y[i][j], x[j], sb);
                b[i][j] = x[j];                     // ... and x
            }
        }
        const size_t next = row + (size_t)stages * gridDim.x;
        if (next < (size_t)a.M) fetch(stage, next);
        cp_async_commit();
        stage = stage + 1 == stages ? 0 : stage + 1;
        float back = 0.f;                           // mean of db w_post xh, times rx
        if (a.w_post || a.gate_mode == 2) {
            block_sum2(sb, sg, s_sum, turn);
            if (a.w_post) back = sb * rx * rx * inv_h;
            if (a.gate_mode == 2 && a.dgate && threadIdx.x == 0) reinterpret_cast<float*>(a.dgate)[row] = sg;
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int ch = threadIdx.x + i * blockDim.x;
            if (ch >= chunks) continue;
            float o[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = rx * fmaf(-b[i][j], back, y[i][j]);
            Elem<T>::store8(reinterpret_cast<T*>(a.dx) + row * H + (size_t)ch * 8, o);
        }
    }
    float* part = a.part + (size_t)blockIdx.x * 3 * H;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int ch = threadIdx.x + i * blockDim.x;
        if (ch >= chunks) continue;
        if (a.want & 1) Elem<float>::store8(part + (size_t)ch * 8, acc_pre[i]);
        if (a.want & 2) Elem<float>::store8(part + H + (size_t)ch * 8, acc_post[i]);
        if (a.want & 4) Elem<float>::store8(part + 2 * H + (size_t)ch * 8, acc_gate[i]);
    }
    pdl_launch_dependents();
}

// Column sums of the partial rows [n][3][H]: a block takes 32 columns, its warps every eighth partial row.
constexpr int kNormColWarps = 8;
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
#pragma unroll 4
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

// Norms of queries and keys for each head with the position rotation in the same pass, and their gradient.  For every token t
// and head, all sums in fp32, one rounding per output:
//   n = w ? x / sqrt(mean(x^2) + eps) * w : x
//   y = n, but each of the rot / 2 pairs (a, b) of its first rot columns turned by the angle position[t] freq[i]:
//       (a cos - b sin, b cos + a sin)
// Backward, with d = dy turned back, r = 1 / sqrt(mean(x^2) + eps), xh = r x:
//   dx = w ? r (d w - xh mean(d w xh)) : d,   dw = sum over tokens and heads of d xh
// Bound by the bytes of the rows (2 resp. 3 tensors).  A thread takes an item of 16 (or 8) columns of a head that holds both
// members of its pairs, so nothing but the row sums crosses threads, and those stay inside a part of a warp.  The angles of a
// token serve all of its heads: a block of several tokens computes them once into shared memory, the product position * freq
// and what is left of it after whole turns in 64 bits (in 32, a position of a million is off by a tenth of a turn).
#pragma once
#include "element.cuh"

namespace coral {

constexpr int kQkThreads = 256;
constexpr int kQkTokens = 8;                        // most tokens of a block's turn
constexpr int kQkMaxD = 256;

struct QkArgs {
    int T, n_q, n_k, D, rot, items, lanes, tokens;   // items of a head, threads a head (a power of two), tokens a turn
    float eps;
    const int32_t* pos;
    const float* freq;
    const void *x[2], *w[2], *dy[2];                 // queries, keys
    void* y[2];                                      // outputs: y forward, dx backward
    long long ld_x[2], ld_dy[2], ld_y[2];            // elements from a token to the next; heads are D apart
    float* part;                                     // backward: [grid][2][D] column sums, or null
};

// N (4 or 8) consecutive elements, widened, and back.
template <typename T, int N>
__device__ __forceinline__ void load_cols(const T* p, float (&v)[N]) {
    if constexpr (N == 8) {
        Elem<T>::load8(p, v);
    } else if constexpr (sizeof(T) == 4) {
        const float4 a = *reinterpret_cast<const float4*>(p);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    } else {
        const uint2 a = *reinterpret_cast<const uint2*>(p);
        T h[4];
        *reinterpret_cast<uint2*>(h) = a;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = Elem<T>::up(h[i]);
    }
}
template <typename T, int N>
__device__ __forceinline__ void store_cols(T* p, const float (&v)[N]) {
    if constexpr (N == 8) {
        Elem<T>::store8(p, v);
    } else if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    } else {
        T h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = Elem<T>::down(v[i]);
        *reinterpret_cast<uint2*>(p) = *reinterpret_cast<uint2*>(h);
    }
}

// What this thread's item covers: columns at c0 and at c1 (N each, c1 < 0: none), the first of its pairs, and whether its
// granules are rotated.  HALVES: pair i is columns i and rot / 2 + i, an item is N pairs; behind the rotated columns come items of
// two neighbouring granules.  Otherwise pair i is columns 2 i and 2 i + 1, and all items are two neighbouring granules.
template <bool HALVES, int N>
struct QkItem {
    int c0 = -1, c1 = -1, pair = 0;
    bool turn0 = false, turn1 = false;
    __device__ __forceinline__ QkItem(int i, const QkArgs& a) {
        if (i >= a.items) return;
        const int turned = HALVES ? a.rot / 2 / N : 0;
        if (i < turned) {
            c0 = i * N;
            c1 = a.rot / 2 + c0;
            pair = c0;
            turn0 = turn1 = true;
        } else {
            c0 = (HALVES ? a.rot : 0) + (i - turned) * 2 * N;
            c1 = c0 + N < a.D ? c0 + N : -1;
            pair = c0 / 2;
            turn0 = !HALVES && c0 < a.rot;
            turn1 = !HALVES && c1 >= 0 && c1 < a.rot;
        }
    }
    // Turns the item's pairs (back: by the opposite angle).
    __device__ __forceinline__ void turn(float (&u)[N], float (&v)[N], const float* cs, const float* sn, float back) const {
        if (HALVES) {
            if (!turn0) return;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float c = cs[pair + i], s = sn[pair + i] * back, a = u[i], b = v[i];
                u[i] = a * c - b * s;
                v[i] = b * c + a * s;
            }
        } else {
            half(u, turn0, cs + pair, sn + pair, back);
            half(v, turn1, cs + pair + N / 2, sn + pair + N / 2, back);
        }
    }
    static __device__ __forceinline__ void half(float (&u)[N], bool on, const float* cs, const float* sn, float back) {
        if (!on) return;
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const float c = cs[i], s = sn[i] * back, a = u[2 * i], b = u[2 * i + 1];
            u[2 * i] = a * c - b * s;
            u[2 * i + 1] = b * c + a * s;
        }
    }
};

// Cosines and sines of a turn's tokens: the product in 64 bits is exact to 2^-53, and so are the turns taken off it.
__device__ __forceinline__ void qk_angles(const QkArgs& a, int t0, int n, float* cs, float* sn) {
    const int half = a.rot >> 1;
    for (int i = threadIdx.x; i < n * half; i += blockDim.x) {
        const int t = i / half;
        const double turns = (double)a.pos[t0 + t] * (double)a.freq[i - t * half] * 0.15915494309189533577;
        sincospif((float)(2.0 * (turns - rint(turns))), &sn[i], &cs[i]);
    }
}

__device__ __forceinline__ float lanes_sum(float v, int lanes) {
    for (int o = lanes >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// The heads of one tensor in a turn, `lanes` threads each: f(token of the turn, head, whether there is one), the same number of
// times in all threads of a warp.
template <typename F>
__device__ __forceinline__ void qk_rows(const QkArgs& a, int heads, int n, F f) {
    const int per = kQkThreads / a.lanes, mine = threadIdx.x / a.lanes, first = (threadIdx.x & ~31) / a.lanes;
    int t = mine / heads, h = mine - t * heads;
    const int step_t = per / heads, step_h = per - step_t * heads;
    for (int r = first; r < n * heads; r += per) {
        f(t, h, t < n);
        t += step_t;
        h += step_h;
        if (h >= heads) {
            h -= heads;
            ++t;
        }
    }
}

template <typename T, bool HALVES, int N>
__global__ void __launch_bounds__(kQkThreads) qk_rotate_kernel(QkArgs a) {
    extern __shared__ float qk_smem[];
    float *cs = qk_smem, *sn = qk_smem + a.tokens * (a.rot >> 1);
    const int lane = threadIdx.x & (a.lanes - 1), half = a.rot >> 1;
    const QkItem<HALVES, N> it(lane, a);
    const float inv_d = 1.f / (float)a.D;
    pdl_wait();
    const int t0 = blockIdx.x * a.tokens, n = min(a.tokens, a.T - t0);
    qk_angles(a, t0, n, cs, sn);
    __syncthreads();
#pragma unroll
    for (int part = 0; part < 2; ++part) {
        const int heads = part ? a.n_k : a.n_q;
        if (heads == 0) continue;
        const T* x = static_cast<const T*>(a.x[part]);
        const T* w = static_cast<const T*>(a.w[part]);
        T* y = static_cast<T*>(a.y[part]);
        qk_rows(a, heads, n, [&](int t, int h, bool on) {
            const T* from = x + (size_t)(t0 + t) * a.ld_x[part] + (size_t)h * a.D;
            float u[N] = {}, v[N] = {};
            if (on && it.c0 >= 0) load_cols<T, N>(from + it.c0, u);
            if (on && it.c1 >= 0) load_cols<T, N>(from + it.c1, v);
            if (w) {
                float ss = 0.f;
#pragma unroll
                for (int i = 0; i < N; ++i) ss += u[i] * u[i] + v[i] * v[i];
                const float r = 1.f / sqrtf(lanes_sum(ss, a.lanes) * inv_d + a.eps);
                float wu[N] = {}, wv[N] = {};
                if (it.c0 >= 0) load_cols<T, N>(w + it.c0, wu);
                if (it.c1 >= 0) load_cols<T, N>(w + it.c1, wv);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    u[i] *= r * wu[i];
                    v[i] *= r * wv[i];
                }
            }
            if (!on) return;
            it.turn(u, v, cs + t * half, sn + t * half, 1.f);
            T* to = y + (size_t)(t0 + t) * a.ld_y[part] + (size_t)h * a.D;
            if (it.c0 >= 0) store_cols<T, N>(to + it.c0, u);
            if (it.c1 >= 0) store_cols<T, N>(to + it.c1, v);
        });
    }
    pdl_launch_dependents();
}

// Blocks take turns of tokens, grid apart, and keep the column sums of all their rows in registers; the sums go through a fixed
// order (a thread's rows, the block's threads, the blocks' partial rows), so the same call gives the same bits.
template <typename T, bool HALVES, int N>
__global__ void __launch_bounds__(kQkThreads) qk_rotate_backward_kernel(QkArgs a) {
    extern __shared__ float qk_smem[];
    float *cs = qk_smem, *sn = qk_smem + a.tokens * (a.rot >> 1);
    const int lane = threadIdx.x & (a.lanes - 1), half = a.rot >> 1;
    const QkItem<HALVES, N> it(lane, a);
    const float inv_d = 1.f / (float)a.D;
    float acc[2][2 * N] = {};
    pdl_wait();
    for (int t0 = blockIdx.x * a.tokens; t0 < a.T; t0 += gridDim.x * a.tokens) {
        const int n = min(a.tokens, a.T - t0);
        __syncthreads();
        qk_angles(a, t0, n, cs, sn);
        __syncthreads();
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            const int heads = part ? a.n_k : a.n_q;
            if (heads == 0) continue;
            const T* x = static_cast<const T*>(a.x[part]);
            const T* w = static_cast<const T*>(a.w[part]);
            const T* dy = static_cast<const T*>(a.dy[part]);
            T* dx = static_cast<T*>(a.y[part]);
            qk_rows(a, heads, n, [&](int t, int h, bool on) {
                const size_t tok = (size_t)(t0 + t), head = (size_t)h * a.D;
                float u[N] = {}, v[N] = {}, du[N] = {}, dv[N] = {};
                if (on && it.c0 >= 0) load_cols<T, N>(dy + tok * a.ld_dy[part] + head + it.c0, du);
                if (on && it.c1 >= 0) load_cols<T, N>(dy + tok * a.ld_dy[part] + head + it.c1, dv);
                if (w) {
                    if (on && it.c0 >= 0) load_cols<T, N>(x + tok * a.ld_x[part] + head + it.c0, u);
                    if (on && it.c1 >= 0) load_cols<T, N>(x + tok * a.ld_x[part] + head + it.c1, v);
                }
                if (on) it.turn(du, dv, cs + t * half, sn + t * half, -1.f);
                if (w) {
                    float ss = 0.f, dot = 0.f;
                    float wu[N] = {}, wv[N] = {};
                    if (it.c0 >= 0) load_cols<T, N>(w + it.c0, wu);
                    if (it.c1 >= 0) load_cols<T, N>(w + it.c1, wv);
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        ss += u[i] * u[i] + v[i] * v[i];
                        dot += du[i] * wu[i] * u[i] + dv[i] * wv[i] * v[i];
                    }
                    for (int o = a.lanes >> 1; o > 0; o >>= 1) {
                        ss += __shfl_xor_sync(0xffffffffu, ss, o);
                        dot += __shfl_xor_sync(0xffffffffu, dot, o);
                    }
                    const float r = 1.f / sqrtf(ss * inv_d + a.eps);
                    const float m = dot * r * inv_d;                        // mean(d w xh)
                    if (on) {
#pragma unroll
                        for (int i = 0; i < N; ++i) {
                            const float xu = r * u[i], xv = r * v[i];
                            acc[part][i] += du[i] * xu;
                            acc[part][N + i] += dv[i] * xv;
                            du[i] = r * (du[i] * wu[i] - xu * m);
                            dv[i] = r * (dv[i] * wv[i] - xv * m);
                        }
                    }
                }
                if (!on) return;
                T* to = dx + tok * a.ld_y[part] + head;
                if (it.c0 >= 0) store_cols<T, N>(to + it.c0, du);
                if (it.c1 >= 0) store_cols<T, N>(to + it.c1, dv);
            });
        }
    }
    if (a.part) {
        float* s = qk_smem;                                                 // [threads a column][columns of an item]
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 2 * N; ++i) s[i * kQkThreads + threadIdx.x] = acc[part][i];
            __syncthreads();
            // one thread a column of an item: its sum over the block's heads
            for (int c = threadIdx.x; c < 2 * N * a.lanes; c += kQkThreads) {
                const int i = c / a.lanes, l = c - i * a.lanes;
                float sum = 0.f;
                for (int j = l; j < kQkThreads; j += a.lanes) sum += s[i * kQkThreads + j];
                const QkItem<HALVES, N> of(l, a);
                const int col = i < N ? of.c0 : of.c1;
                if (col >= 0) a.part[((size_t)blockIdx.x * 2 + part) * a.D + col + (i < N ? i : i - N)] = sum;
            }
        }
    }
    pdl_launch_dependents();
}

// Column sums of the partial rows [n][2][D].  grid: (column blocks of 32, 2).
constexpr int kQkColWarps = 16;
__global__ void __launch_bounds__(kQkColWarps * 32) qk_columns_kernel(const float* __restrict__ part, int n, int D, float* dw_q, float* dw_k) {
    __shared__ float s[kQkColWarps][32];
    float* out = blockIdx.y ? dw_k : dw_q;
    if (!out) return;
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    float acc = 0.f;
    if (col < D) {
        const float* p = part + (size_t)blockIdx.y * D + col;
#pragma unroll 8
        for (int i = warp; i < n; i += kQkColWarps) acc += p[(size_t)i * 2 * D];
    }
    s[warp][lane] = acc;
    __syncthreads();
    if (warp == 0 && col < D) {
#pragma unroll
        for (int i = 1; i < kQkColWarps; ++i) acc += s[i][lane];
        out[col] = acc;
    }
}

}  // namespace coral

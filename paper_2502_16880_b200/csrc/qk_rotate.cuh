// Norms of queries and keys for each head with the position rotation in the same pass, and their gradient.  For every token t
// and head, all sums in fp32, one rounding per output:
//   n = w ? x / sqrt(mean(x^2) + eps) * w : x
//   y = n, but each of the rot / 2 pairs (a, b) of its first rot columns turned by the angle position[t] freq[i]:
//       (a cos - b sin, b cos + a sin)
// Backward, with d = dy turned back, r = 1 / sqrt(mean(x^2) + eps), xh = r x:
//   dx = w ? r (d w - xh mean(d w xh)) : d,   dw = sum over tokens and heads of d xh
// Bound by the bytes of the rows (2 resp. 3 tensors).  A thread takes an item of 16 (or 8) columns of a head that holds both
// members of its pairs, so nothing but the row sums crosses threads, and those stay inside a part of a warp.  A warp takes a token
// and some of its heads at a time: it computes the token's angles once, the product position * freq and what is left of it after
// whole turns in 64 bits (in 32, a position of a million is off by a tenth of a turn), and its threads keep what their item
// needs of them, times the weights, in registers over all of those heads.  No block-wide barrier but for the column sums.
// 16384 tokens of 32 + 8 heads of 128, bf16: 58.7 us, 87 % of the copy bandwidth measured (75 before a warp kept a token's factors over its
// heads and loaded rows ahead, 60 with each position read where it is needed).  Gradient of 8192 tokens: 58 us, 66 % (136 before; 62 with one
// row ahead in registers): 126 registers leave 16 warps a SM, each token's angles are computed for the queries and again for the keys, and the
// column sums' second kernel takes 4 of it.
#pragma once
#include <type_traits>

#include "cp_async.cuh"
#include "element.cuh"

namespace coral {

constexpr int kQkThreads = 256;
constexpr int kQkWarps = kQkThreads / 32;
constexpr int kQkMaxD = 256;

struct QkArgs {
    int T, n_q, n_k, D, rot, items, lanes;           // items of a head, threads a head (a power of two)
    int shares, span[2];                             // warps that share a token, query and key heads of each
    float eps;
    const int32_t* pos;
    const float* freq;
    const void *x[2], *w[2], *dy[2];                 // queries, keys
    void* y[2];                                      // outputs: y forward, dx backward
    long long ld_x[2], ld_dy[2], ld_y[2];            // elements from a token to the next; heads are D apart
    float* part;                                     // backward: [grid][2][D] column sums, or null
};

// N (4 or 8) consecutive elements as N / 2 pairs of fp32 (the two-wide instructions do the arithmetic), and back.
template <int N> struct QkCols {
    unsigned long long p[N / 2];
};
template <typename T, int N> struct QkRaw {
    static constexpr int kWords = N * (int)sizeof(T) / 4;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const T* p) {
        if constexpr (kWords == 2) {
            *reinterpret_cast<uint2*>(w) = *reinterpret_cast<const uint2*>(p);
        } else {
#pragma unroll
            for (int i = 0; i < kWords; i += 4) *reinterpret_cast<uint4*>(w + i) = reinterpret_cast<const uint4*>(p)[i / 4];
        }
    }
    __device__ __forceinline__ QkCols<N> cols() const {
        QkCols<N> r;
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            if constexpr (sizeof(T) == 4) {
                r.p[i] = pair_of(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
            } else if constexpr (std::is_same_v<T, __half>) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
                r.p[i] = pair_of(f.x, f.y);
            } else {
                r.p[i] = pair_of(bf16_lo(w[i]), bf16_hi(w[i]));
            }
        }
        return r;
    }
};
template <typename T, int N>
__device__ __forceinline__ void store_cols(T* p, const QkCols<N>& v) {
    if constexpr (N == 8) {
        store8v<T>(p, V8{{v.p[0], v.p[1], v.p[2], v.p[3]}});
    } else {
        const float2 a = halves(v.p[0]), b = halves(v.p[1]);
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<float4*>(p) = make_float4(a.x, a.y, b.x, b.y);
        } else {
            const T h[4] = {Elem<T>::down(a.x), Elem<T>::down(a.y), Elem<T>::down(b.x), Elem<T>::down(b.y)};
            *reinterpret_cast<uint2*>(p) = *reinterpret_cast<const uint2*>(h);
        }
    }
}

// What this thread's item covers: columns at c0 and at c1 (N each, < 0: none), the first of its pairs, and whether its granules are
// turned.  HALVES: pair i is columns i and rot / 2 + i, an item is N pairs; behind the turned columns come items of two neighbouring
// granules.  Otherwise pair i is columns 2 i and 2 i + 1, and all items are two neighbouring granules.  ALL: every thread has both.
template <typename T, bool HALVES, int N, bool ALL>
struct QkItem {
    int c0 = -1, c1 = -1, pair = 0;
    bool turn0 = false, turn1 = false;
    __device__ __forceinline__ QkItem(int i, const QkArgs& a) {
        if (!ALL && i >= a.items) return;
        const int turned = HALVES ? a.rot / 2 / N : 0;
        if (i < turned) {
            c0 = i * N;
            c1 = a.rot / 2 + c0;
            pair = c0;
            turn0 = turn1 = true;
        } else {
            c0 = (HALVES ? a.rot : 0) + (i - turned) * 2 * N;
            c1 = ALL || c0 + N < a.D ? c0 + N : -1;
            pair = c0 / 2;
            turn0 = !HALVES && c0 < a.rot;
            turn1 = !HALVES && c1 >= 0 && c1 < a.rot;
        }
    }
    __device__ __forceinline__ void load(const T* row, bool on, QkRaw<T, N>& u, QkRaw<T, N>& v) const {
        u = v = QkRaw<T, N>{};
        if (on && (ALL || c0 >= 0)) u.load(row + c0);
        if (on && (ALL || c1 >= 0)) v.load(row + c1);
    }
    __device__ __forceinline__ void store(T* row, const QkCols<N>& u, const QkCols<N>& v) const {
        if (ALL || c0 >= 0) store_cols<T, N>(row + c0, u);
        if (ALL || c1 >= 0) store_cols<T, N>(row + c1, v);
    }
};

// The turn of an item as factors, times weights: u' = u uc + v~ us, v' = v vc + u~ vs, where v~ is the other granule (HALVES) or the
// granule itself with the members of its pairs exchanged.  A granule that is not turned has the weight for a factor and no second term (zero
// times an infinity in a column that is none of its business would be a NaN).
template <int N> struct QkTurn {
    QkCols<N> uc, us, vc, vs;
    template <bool HALVES>
    __device__ __forceinline__ void operator()(QkCols<N>& u, QkCols<N>& v, bool turn_u, bool turn_v) const {
        if (turn_u && turn_v) {                      // (in one piece: granule by granule it is 2 % slower)
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                const unsigned long long a = u.p[i], b = v.p[i];
                u.p[i] = fma2(HALVES ? b : exchanged(a), us.p[i], mul2(a, uc.p[i]));
                v.p[i] = fma2(HALVES ? a : exchanged(b), vs.p[i], mul2(b, vc.p[i]));
            }
        } else {                                     // (of two halves none is turned alone)
#pragma unroll
            for (int i = 0; i < N / 2; ++i) {
                const unsigned long long a = u.p[i], b = v.p[i];
                u.p[i] = mul2(a, uc.p[i]);
                v.p[i] = mul2(b, vc.p[i]);
                if (!HALVES && turn_u) u.p[i] = fma2(exchanged(a), us.p[i], u.p[i]);
                if (!HALVES && turn_v) v.p[i] = fma2(exchanged(b), vs.p[i], v.p[i]);
            }
        }
    }
    static __device__ __forceinline__ unsigned long long exchanged(unsigned long long a) {
        const float2 x = halves(a);
        return pair_of(x.y, x.x);
    }
};
// wu, wv: the weights of the item's own columns.  BACK: the opposite angle.
template <bool HALVES, bool BACK, int N, typename Item>
__device__ __forceinline__ QkTurn<N> qk_turn(const Item& it, const float* cs, const float* sn, const QkCols<N>& wu, const QkCols<N>& wv) {
    QkTurn<N> r;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        const float2 x = halves(wu.p[i]), y = halves(wv.p[i]);
        if (HALVES) {
            const int j = it.pair + 2 * i;
            const float c0 = it.turn0 ? cs[j] : 1.f, c1 = it.turn0 ? cs[j + 1] : 1.f;
            const float s0 = it.turn0 ? (BACK ? -sn[j] : sn[j]) : 0.f, s1 = it.turn0 ? (BACK ? -sn[j + 1] : sn[j + 1]) : 0.f;
            r.uc.p[i] = pair_of(c0 * x.x, c1 * x.y);
            r.us.p[i] = pair_of(-s0 * y.x, -s1 * y.y);
            r.vc.p[i] = pair_of(c0 * y.x, c1 * y.y);
            r.vs.p[i] = pair_of(s0 * x.x, s1 * x.y);
        } else {
            const int j = it.pair + i, k = j + N / 2;
            const float c0 = it.turn0 ? cs[j] : 1.f, s0 = it.turn0 ? (BACK ? -sn[j] : sn[j]) : 0.f;
            const float c1 = it.turn1 ? cs[k] : 1.f, s1 = it.turn1 ? (BACK ? -sn[k] : sn[k]) : 0.f;
            r.uc.p[i] = pair_of(c0 * x.x, c0 * x.y);
            r.us.p[i] = pair_of(-s0 * x.y, s0 * x.x);
            r.vc.p[i] = pair_of(c1 * y.x, c1 * y.y);
            r.vs.p[i] = pair_of(-s1 * y.y, s1 * y.x);
        }
    }
    return r;
}

template <int N>
__device__ __forceinline__ QkCols<N> mul_cols(const QkCols<N>& a, const QkCols<N>& b) {
    QkCols<N> r;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) r.p[i] = mul2(a.p[i], b.p[i]);
    return r;
}
template <int N>
__device__ __forceinline__ QkCols<N> scale_cols(const QkCols<N>& a, float f) {
    QkCols<N> r;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) r.p[i] = mul2(a.p[i], pair_of(f, f));
    return r;
}
// sum over both granules of a b
template <int N>
__device__ __forceinline__ float dot_cols(const QkCols<N>& a0, const QkCols<N>& b0, const QkCols<N>& a1, const QkCols<N>& b1) {
    unsigned long long x = 0, y = 0;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        x = fma2(a0.p[i], b0.p[i], x);
        y = fma2(a1.p[i], b1.p[i], y);
    }
    const float2 s = halves(x), t = halves(y);
    return (s.x + s.y) + (t.x + t.y);
}
template <int N>
__device__ __forceinline__ void add_products(QkCols<N>& acc, const QkCols<N>& a, const QkCols<N>& b) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) acc.p[i] = fma2(a.p[i], b.p[i], acc.p[i]);
}

// Cosines and sines of a token's position, by a warp: the product in 64 bits is exact to 2^-53, and so are the turns taken off it.
__device__ __forceinline__ void qk_angles(const QkArgs& a, int pos, float* cs, float* sn) {
    const double p = (double)pos * 0.15915494309189533577;
    __syncwarp();
    for (int i = threadIdx.x & 31; i < a.rot >> 1; i += 32) {
        const double turns = p * (double)a.freq[i];
        sincospif((float)(2.0 * (turns - rint(turns))), &sn[i], &cs[i]);
    }
    __syncwarp();
}

template <int L>
__device__ __forceinline__ float lanes_sum(float v, int lanes) {
#pragma unroll
    for (int o = (L ? L : 32) / 2; o > 0; o >>= 1)
        if (L || o < lanes) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// L: threads a head where every item is whole (0: any number, at run time).  A warp's turn is a token with a share of its query heads and
// one of its key heads; two rows of heads are worked on while the next two are on their way.
template <typename T, bool HALVES, int N, int L>
__global__ void __launch_bounds__(kQkThreads, 2) qk_rotate_kernel(const __grid_constant__ QkArgs a) {
    __shared__ __align__(16) float s_cs[kQkWarps][kQkMaxD / 2], s_sn[kQkWarps][kQkMaxD / 2];
    float *cs = s_cs[threadIdx.x >> 5], *sn = s_sn[threadIdx.x >> 5];
    const int lanes = L ? L : a.lanes, lane = threadIdx.x & 31, row = lane / lanes, rows = 32 / lanes;
    const QkItem<T, HALVES, N, L != 0> it(lane & (lanes - 1), a);
    const float inv_d = 1.f / (float)a.D;
    const int warps = gridDim.x * kQkWarps, step = rows * a.D;
    const long long units = (long long)a.T * a.shares;
    auto token = [&](long long unit) { return a.shares == 1 ? (int)unit : (int)(unit / a.shares); };
    const long long first = blockIdx.x * kQkWarps + (threadIdx.x >> 5);
    pdl_wait();
    int pos_ahead = first < units ? a.pos[token(first)] : 0;
    for (long long unit = first; unit < units; unit += warps) {
        const int t = token(unit), share = (int)(unit - (long long)t * a.shares), pos = pos_ahead;
        if (unit + warps < units) pos_ahead = a.pos[token(unit + warps)];
        bool known = false;                                    // the token's angles
#pragma unroll 1
        for (int part = 0; part < 2; ++part) {
            const int h0 = share * a.span[part], heads = min(a.span[part], (part ? a.n_k : a.n_q) - h0);
            if (heads <= 0) continue;
            const T *w = static_cast<const T*>(a.w[part]), *from = static_cast<const T*>(a.x[part]) + t * a.ld_x[part] + (h0 + row) * a.D;
            T* to = static_cast<T*>(a.y[part]) + t * a.ld_y[part] + (h0 + row) * a.D;
            QkRaw<T, N> u0[2], v0[2], u1[2], v1[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) it.load(from + i * step, row + i * rows < heads, u0[i], v0[i]);
            if (!known) qk_angles(a, pos, cs, sn);
            known = true;
            it.load(w, w != nullptr, u1[0], v1[0]);            // from L1: kept in the turn's factors only
            QkCols<N> wu = u1[0].cols(), wv = v1[0].cols();
            if (!w)
#pragma unroll
                for (int i = 0; i < N / 2; ++i) wu.p[i] = wv.p[i] = pair_of(1.f, 1.f);
            const QkTurn<N> f = qk_turn<HALVES, false>(it, cs, sn, wu, wv);
            for (int h = row; h - row < heads; h += 2 * rows) {
                from += 2 * step;
#pragma unroll
                for (int i = 0; i < 2; ++i) it.load(from + i * step, h + (2 + i) * rows < heads, u1[i], v1[i]);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    QkCols<N> u = u0[i].cols(), v = v0[i].cols();
                    if (w) {
                        const float r = rsqrtf(fmaf(lanes_sum<L>(dot_cols(u, u, v, v), lanes), inv_d, a.eps));
                        u = scale_cols(u, r);
                        v = scale_cols(v, r);
                    }
                    f.template operator()<HALVES>(u, v, it.turn0, it.turn1);
                    if (h + i * rows < heads) it.store(to + i * step, u, v);
                    u0[i] = u1[i];
                    v0[i] = v1[i];
                }
                to += 2 * step;
            }
        }
    }
    pdl_launch_dependents();
}

// The column sums of a warp's rows stay in registers; they go through a fixed order (a thread's rows, the block's threads, the blocks'
// partial rows), so the same call gives the same bits.  What a thread reads of dy and x comes through a ring in shared memory of its own,
// several rows ahead and across tokens: registers have room for one row ahead only.
template <typename T, int N> constexpr int kQkStep = 4 * N * (int)sizeof(T) * kQkThreads;          // a row of each thread: two granules of dy and of x
template <typename T, int N> constexpr int kQkSlots = 80 * 1024 / kQkStep<T, N>;
// Static shared memory of the kernel: angles of its warps, sums of its threads.
template <int N> constexpr size_t kQkStatic = 2 * kQkWarps * (kQkMaxD / 2) * sizeof(float) + 2 * N * kQkThreads * sizeof(float);
template <typename T, int N>
struct QkRing {
    static constexpr int kBytes = N * (int)sizeof(T);
    unsigned char* base;
    __device__ __forceinline__ unsigned char* at(int slot, int granule) const { return base + ((slot * 4 + granule) * kQkThreads + (int)threadIdx.x) * kBytes; }
    __device__ __forceinline__ void fill(int slot, int granule, const T* from) const {
        if constexpr (kBytes == 8) {
            cp_async8(at(slot, granule), from);
        } else {
#pragma unroll
            for (int i = 0; i < kBytes; i += 16) cp_async16(at(slot, granule) + i, reinterpret_cast<const unsigned char*>(from) + i);
        }
    }
    __device__ __forceinline__ QkRaw<T, N> row(int slot, int granule, bool on) const {
        QkRaw<T, N> r{};
        if (on) r.load(reinterpret_cast<const T*>(at(slot, granule)));
        return r;
    }
};

template <typename T, bool HALVES, int N, int L>
__global__ void __launch_bounds__(kQkThreads, 2) qk_rotate_backward_kernel(const __grid_constant__ QkArgs a) {
    __shared__ __align__(16) float s_cs[kQkWarps][kQkMaxD / 2], s_sn[kQkWarps][kQkMaxD / 2];
    __shared__ float s_sum[2 * N * kQkThreads];               // [column of an item][thread]
    extern __shared__ __align__(16) unsigned char qk_ring[];
    constexpr int SLOTS = kQkSlots<T, N>;
    static_assert(SLOTS >= 2, "a row is read while the next is on its way");
    const QkRing<T, N> ring{qk_ring};
    float *cs = s_cs[threadIdx.x >> 5], *sn = s_sn[threadIdx.x >> 5];
    const int lanes = L ? L : a.lanes, lane = threadIdx.x & 31, row = lane / lanes, rows = 32 / lanes;
    const QkItem<T, HALVES, N, L != 0> it(lane & (lanes - 1), a);
    const float inv_d = 1.f / (float)a.D;
    const int warps = gridDim.x * kQkWarps;
    const long long units = (long long)a.T * a.shares;
    QkCols<N> one;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) one.p[i] = pair_of(1.f, 1.f);
    pdl_wait();
#pragma unroll 1
    for (int part = 0; part < 2; ++part) {
        const int all_heads = part ? a.n_k : a.n_q;
        if (all_heads == 0) continue;
        const T *x = static_cast<const T*>(a.x[part]), *dy = static_cast<const T*>(a.dy[part]), *w = static_cast<const T*>(a.w[part]);
        T* dx = static_cast<T*>(a.y[part]);
        const long long ld_x = a.ld_x[part], ld_dy = a.ld_dy[part], ld_dx = a.ld_y[part];
        QkCols<N> acc_u{}, acc_v{}, wu, wv;
        {
            QkRaw<T, N> ru, rv;
            it.load(w, w != nullptr, ru, rv);
            wu = ru.cols();
            wv = rv.cols();
        }
        const long long first = blockIdx.x * kQkWarps + (threadIdx.x >> 5);
        auto token = [&](long long unit, int* h0, int* heads) {     // of a unit, with its heads
            const int t = a.shares == 1 ? (int)unit : (int)(unit / a.shares);
            *h0 = (int)(unit - (long long)t * a.shares) * a.span[part];
            *heads = min(a.span[part], all_heads - *h0);
            return t;
        };
        // the next row to be fetched
        long long next = first;
        int next_h = row, next_heads = 0;
        const T *next_x = nullptr, *next_dy = nullptr;
        auto open = [&]() {
            for (; next < units; next += warps) {
                int h0;
                const int t = token(next, &h0, &next_heads);
                if (next_heads <= 0) continue;
                next_h = row;
                next_x = x + t * ld_x + (h0 + row) * a.D;
                next_dy = dy + t * ld_dy + (h0 + row) * a.D;
                return;
            }
        };
        auto fetch = [&](int slot) {
            if (next < units) {
                if (next_h < next_heads) {
                    if (L || it.c0 >= 0) {
                        ring.fill(slot, 0, next_dy + it.c0);
                        if (w) ring.fill(slot, 2, next_x + it.c0);
                    }
                    if (L || it.c1 >= 0) {
                        ring.fill(slot, 1, next_dy + it.c1);
                        if (w) ring.fill(slot, 3, next_x + it.c1);
                    }
                }
                next_h += rows;
                next_x += rows * a.D;
                next_dy += rows * a.D;
                if (next_h - row >= next_heads) {
                    next += warps;
                    open();
                }
            }
            cp_async_commit();
        };
        open();
#pragma unroll 1
        for (int i = 0; i < SLOTS - 1; ++i) fetch(i);
        int slot = 0;
        for (long long unit = first; unit < units; unit += warps) {
            int h0, heads;
            const int t = token(unit, &h0, &heads);
            if (heads <= 0) continue;
            T* to = dx + t * ld_dx + (h0 + row) * a.D;
            qk_angles(a, a.pos[t], cs, sn);
            const QkTurn<N> f = qk_turn<HALVES, true>(it, cs, sn, one, one);
            for (int h = row; h - row < heads; h += rows) {
                cp_async_wait<SLOTS - 2>();
                const bool on = h < heads, on0 = on && (L || it.c0 >= 0), on1 = on && (L || it.c1 >= 0);
                const QkRaw<T, N> p0 = ring.row(slot, 0, on0), q0 = ring.row(slot, 1, on1), u0 = ring.row(slot, 2, on0 && w), v0 = ring.row(slot, 3, on1 && w);
                fetch(slot == 0 ? SLOTS - 1 : slot - 1);           // the row before: its values are in use
                slot = slot + 1 == SLOTS ? 0 : slot + 1;
                QkCols<N> du = p0.cols(), dv = q0.cols();
                f.template operator()<HALVES>(du, dv, it.turn0, it.turn1);
                if (w) {
                    QkCols<N> u = u0.cols(), v = v0.cols();
                    const QkCols<N> dwu = mul_cols(du, wu), dwv = mul_cols(dv, wv);
                    const float ss = lanes_sum<L>(dot_cols(u, u, v, v), lanes), dot = lanes_sum<L>(dot_cols(dwu, u, dwv, v), lanes);
                    const float r = rsqrtf(fmaf(ss, inv_d, a.eps));
                    u = scale_cols(u, r);                                       // xh
                    v = scale_cols(v, r);
                    if (h < heads) {
                        add_products(acc_u, du, u);
                        add_products(acc_v, dv, v);
                    }
                    // r d w - xh r mean(d w xh)
                    const float m = -dot * r * inv_d * r;
#pragma unroll
                    for (int i = 0; i < N / 2; ++i) {
                        du.p[i] = fma2(u.p[i], pair_of(m, m), mul2(dwu.p[i], pair_of(r, r)));
                        dv.p[i] = fma2(v.p[i], pair_of(m, m), mul2(dwv.p[i], pair_of(r, r)));
                    }
                }
                if (h < heads) it.store(to, du, dv);
                to += rows * a.D;
            }
        }
        if (!a.part) continue;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const float2 p = halves(acc_u.p[i]), q = halves(acc_v.p[i]);
            s_sum[(2 * i) * kQkThreads + threadIdx.x] = p.x;
            s_sum[(2 * i + 1) * kQkThreads + threadIdx.x] = p.y;
            s_sum[(N + 2 * i) * kQkThreads + threadIdx.x] = q.x;
            s_sum[(N + 2 * i + 1) * kQkThreads + threadIdx.x] = q.y;
        }
        __syncthreads();
        // one thread a column of an item: its sum over the block's heads
        for (int c = threadIdx.x; c < 2 * N * lanes; c += kQkThreads) {
            const int i = c / lanes, l = c - i * lanes;
            float sum = 0.f;
            for (int j = l; j < kQkThreads; j += lanes) sum += s_sum[i * kQkThreads + j];
            const QkItem<T, HALVES, N, L != 0> of(l, a);
            const int col = i < N ? of.c0 : of.c1;
            if (col >= 0) a.part[((size_t)blockIdx.x * 2 + part) * a.D + col + (i < N ? i : i - N)] = sum;
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

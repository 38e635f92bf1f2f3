// Penalties for repeated tokens, biases and grammar masks on dense logits, with the candidates of the result in the same
// pass (the dense counterpart of the draft step's merge; the candidates feed the tree expansion).  Per token x of a row:
//   l1 = x seen ? (l > 0 ? l / rep : l * rep) : l      l2 = l1 - freq * count(x)      l3 = l2 - (count(x) > 0 ? pres : 0)
//   l4 = l3 + bias(x)      out = x allowed ? l4 : -inf            (each step one fp32 operation, in this order)
// Bound by the logits' bytes, so a row is streamed once, by a kernel with no more in it than that needs, and what is rare or
// needs a whole row is done by two small kernels around it:
//   logits_lists_kernel   per sequence: counts its token lists into tables in shared memory (whole numbers: the order of the
//                         atomics does not matter), writes the listed tokens with their counts and biases, in a fixed order,
//                         and a bitmap of them;
//   logits_stream_kernel  reads the logits, leaves out listed tokens (bitmap) and those of the row's path, applies the mask,
//                         writes the result, and keeps the maximum of every 512 bytes and a (maximum, sum of exponentials)
//                         of every warp's part;
//   logits_finish_kernel  per row: the listed and path tokens one a thread (their logits are read again, a few bytes each), the
//                         log-sum-exp, and the candidates: only the k pieces of 512 bytes with the largest maxima can hold
//                         one of the k best of the streamed tokens, so only they are read again.
// (Everything in one kernel, a cluster of blocks a row, took 850 us for 960 x 128256 fp32: candidates and lists cost each block
// a chain of barriers a row, and their code pushed the streaming loop out of the instruction cache.)
#pragma once
#include <cooperative_groups.h>

#include <type_traits>

#include "element.cuh"

namespace coral {

constexpr int kLogitsThreads = 256;
constexpr int kLogitsWarps = kLogitsThreads / 32;
constexpr int kLogitsCap = 2048;                 // keys ranked by counting
constexpr int kLogitsMaxPath = 64;
constexpr int kListThreads = 512;
constexpr int kListWindow = 16384;               // tokens of a block's table
constexpr int kListCluster = 8;

constexpr uint32_t kSeenBit = 0x80000000u, kBiasBit = 0x40000000u;      // table word: flags, count
constexpr uint32_t kCountMask = kBiasBit - 1;

struct LogitsArgs {
    const void* logits;
    void* out;                                   // or null
    long long ld_in, ld_out;
    int M, V, n_seq, path_len, n_masks, mask_words, k;
    const int32_t* row_seq;                      // null: row m is sequence m
    const int32_t *prompt, *output, *path, *bias_tokens;
    const long long *prompt_off, *output_off, *bias_off;
    long long prompt_total, output_total, bias_total;
    const float *rep, *freq, *pres, *bias_values;
    const uint32_t* mask;
    const int32_t* mask_rows;                    // null: row m uses mask m
    int32_t* out_ids;
    float *out_logprobs, *out_lse;
};

// Scratch of a call (the caller's workspace).
struct LogitsWork {
    uint32_t* bitmap;                            // [n_seq][mask_words] listed tokens of a sequence
    uint4* entry;                                // token, table word, bias; a sequence's from its lists' offsets on
    int2* range;                                 // [n_seq] first entry and number
    uint32_t* piece;                             // [M][pieces] largest value (logit_order) of 512 bytes of logits
    float2* part;                                // [M][parts] maximum and sum of a warp's vectors
    int pieces, parts;
};

// Monotone map of a float to an unsigned integer; NaN and -inf (no candidate) become 0.  -0 counts as +0.
__device__ __forceinline__ uint32_t logit_order(float v) {
    if (!(v > kNegInf)) return 0;
    const uint32_t b = __float_as_uint(v + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_unorder(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u); }
__device__ __forceinline__ unsigned long long logit_key(uint32_t order, int token) {
    return order ? ((unsigned long long)order << 32) | (0xffffffffu - (uint32_t)token) : 0ull;
}

__device__ __forceinline__ void list_range(const long long* off, int seq, long long total, long long& a, long long& b) {
    a = off[seq];
    b = off[seq + 1];
    a = a < 0 ? 0 : a > total ? total : a;
    b = b < a ? a : b > total ? total : b;
}

// e^t for t <= 0: one product, one rounding, ex2 (2 ulp)
__device__ __forceinline__ float exp_fast(float t) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(t * 1.4426950408889634f));
    return r;
}

// Sum of e^(v - base) over a vector's values, two at a time where there is an instruction for it.
template <int N>
__device__ __forceinline__ float exp_sum(const float (&val)[N], float base) {
    const unsigned long long nb = pair_of(-base, -base), c = pair_of(1.4426950408889634f, 1.4426950408889634f);
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < N; e += 2) {
        unsigned long long t = pair_of(val[e], val[e + 1]);
        asm("add.rn.f32x2 %0, %1, %2;" : "=l"(t) : "l"(t), "l"(nb));
        float2 f = halves(mul2(t, c));
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(f.x) : "f"(f.x));
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(f.y) : "f"(f.y));
        sum += f.x + f.y;
    }
    return sum;
}

// The k-th largest of the first n lanes' values, in every lane; 0 if there are fewer.
__device__ __forceinline__ uint32_t kth_largest(uint32_t v, int n, int k) {
    if (k > n) return 0;
    const int lane = threadIdx.x & 31;
    if (2 * k > n) {                             // the (n + 1 - k)-th smallest
        if (lane >= n) v = 0xffffffffu;
        for (int i = n - k; i > 0; --i) {
            const uint32_t low = __reduce_min_sync(0xffffffffu, v), who = __ballot_sync(0xffffffffu, v == low);
            if (lane == __ffs(who) - 1) v = 0xffffffffu;
        }
        return __reduce_min_sync(0xffffffffu, v);
    }
    if (lane >= n) v = 0;
    for (int i = k; i > 1; --i) {
        const uint32_t best = __reduce_max_sync(0xffffffffu, v), who = __ballot_sync(0xffffffffu, v == best);
        if (lane == __ffs(who) - 1) v = 0;
    }
    return __reduce_max_sync(0xffffffffu, v);
}

// l / rep for l > 0, correctly rounded: with inv the correctly rounded 1 / rep, q = l inv and the exact remainder l - q rep,
// q + remainder * inv is the correctly rounded quotient (Markstein's theorem), as long as nothing leaves the normal range;
// else the division itself.
__device__ __noinline__ float divide_any(float l, float rep) { return __fdiv_rn(l, rep); }
__device__ __forceinline__ float divide(float l, float rep, float inv) {
    if (!(l > 0x1p-64f && l < 0x1p64f && rep > 0x1p-32f && rep < 0x1p32f)) return divide_any(l, rep);
    const float q = __fmul_rn(l, inv);
    return __fmaf_rn(__fmaf_rn(-q, rep, l), inv, q);
}

// ---- token lists of a sequence -----------------------------------------------------------------------------
// grid: n_seq clusters of kListCluster blocks; a block counts the tokens of windows rank, rank + kListCluster, ...
// dynamic shared memory: the table, and a second one (1 + place of a token's last bias) if there are biases.
__global__ void __launch_bounds__(kListThreads, 1) logits_lists_kernel(const __grid_constant__ LogitsArgs a, LogitsWork w) {
    namespace cg = cooperative_groups;
    extern __shared__ __align__(16) uint32_t tables[];
    __shared__ int s_warp[kListThreads / 32], s_total;
    auto cluster = cg::this_cluster();
    const int seq = blockIdx.x / kListCluster, rank = blockIdx.x % kListCluster, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t* places = tables + kListWindow;
    pdl_launch_dependents();
    long long p0 = 0, p1 = 0, o0 = 0, o1 = 0, b0 = 0, b1 = 0;
    if (a.prompt) list_range(a.prompt_off, seq, a.prompt_total, p0, p1);
    if (a.output) list_range(a.output_off, seq, a.output_total, o0, o1);
    if (a.bias_tokens) list_range(a.bias_off, seq, a.bias_total, b0, b1);
    long long at = p0 + o0 + b0;                 // a sequence has room for as many entries as its lists are long
    const long long first = at;
    for (int base = 0; base < a.V; base += kListCluster * kListWindow) {
        const int lo = base + rank * kListWindow, n = min(kListWindow, a.V - lo);
        const int words = (a.bias_tokens ? 2 : 1) * kListWindow;
        for (int i = threadIdx.x * 4; i < words; i += kListThreads * 4) *reinterpret_cast<uint4*>(tables + i) = make_uint4(0, 0, 0, 0);
        __syncthreads();
        auto each = [&](const int32_t* tokens, long long from, long long to, auto put) {
            for (long long i = from + threadIdx.x; i < to; i += 4 * kListThreads) {
                int32_t t[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) t[u] = i + u * kListThreads < to ? tokens[i + u * kListThreads] : -1;
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (t[u] >= lo && t[u] - lo < n) put(t[u] - lo, (uint32_t)(i + u * kListThreads - from) + 1u);
            }
        };
        if (a.prompt) each(a.prompt, p0, p1, [&](int t, uint32_t) { atomicOr(tables + t, kSeenBit); });
        if (a.output) each(a.output, o0, o1, [&](int t, uint32_t) { atomicAdd(tables + t, 1u); });
        if (a.bias_tokens)
            each(a.bias_tokens, b0, b1, [&](int t, uint32_t place) {
                atomicOr(tables + t, kBiasBit);
                atomicMax(places + t, place);
            });
        __syncthreads();
        // the bitmap, and the number of entries: a warp takes 1024 neighbouring tokens at a time, a lane 32 of them by ballots
        int mine = 0;
        for (int i = warp * 32; i < n; i += kListThreads) {
            const uint32_t bits = __ballot_sync(0xffffffffu, i + lane < n && tables[i + lane] != 0);
            if (lane == 0) w.bitmap[(size_t)seq * a.mask_words + (lo + i) / 32] = bits;
            mine += __popc(bits);                // the same in every lane
        }
        if (lane == 0) s_warp[warp] = mine;
        __syncthreads();
        int before = 0, total = 0;
        for (int i = 0; i < kListThreads / 32; ++i) {
            before += i < warp ? s_warp[i] : 0;
            total += s_warp[i];
        }
        if (threadIdx.x == 0) s_total = total;
        cluster.sync();
        long long next = at;
        for (int c = 0; c < kListCluster; ++c) {
            const int t = *cluster.map_shared_rank(&s_total, c);
            if (c < rank) before += t;
            next += t;
        }
        cluster.sync();                          // s_total has been read
        uint4* out = w.entry + at + before;
        for (int i = warp * 32; i < n; i += kListThreads) {
            const uint32_t word = i + lane < n ? tables[i + lane] : 0, bits = __ballot_sync(0xffffffffu, word != 0);
            if (word) {
                const float bias = word & kBiasBit ? a.bias_values[b0 + places[i + lane] - 1] : 0.f;
                out[__popc(bits & ((1u << lane) - 1))] = make_uint4((uint32_t)(lo + i + lane), word, __float_as_uint(bias), 0);
            }
            out += __popc(bits);
        }
        at = next;
        __syncthreads();
    }
    if (rank == 0 && threadIdx.x == 0) w.range[seq] = make_int2((int)first, (int)(at - first));
}

// ---- the pass over the logits ------------------------------------------------------------------------------
// Positions p = token + shift of a row start on 16 bytes: a vector is loaded whole unless it holds an end of the row.  A piece is
// what a warp loads at once, 32 vectors.
template <typename T>
struct LogitsVec {
    static constexpr int kVec = 16 / (int)sizeof(T), kPiece = 32 * kVec;
};

// A vector that holds an end of its row (or lies behind it): what is outside is -inf.
template <typename T>
__device__ __noinline__ uint4 load_edge(const T* in, int p, int shift, int end) {
    __align__(16) T v[16 / sizeof(T)];
    for (int e = 0; e < (int)(16 / sizeof(T)); ++e)
        v[e] = p + e >= shift && p + e < end ? in[p + e - shift] : Elem<T>::down(kNegInf);
    return *reinterpret_cast<const uint4*>(v);
}
// A vector that cannot be stored whole: leaves out what is outside the row and the tokens in `listed`.
template <typename T, int N>
__device__ __noinline__ void store_edge(T* to, const float (&val)[N], int p, int shift, int end, uint32_t listed) {
    for (int e = 0; e < N; ++e)
        if (p + e >= shift && p + e < end && !((listed >> e) & 1u)) to[e] = Elem<T>::down(val[e]);
}
// Bits of a row's bitmap for the n tokens from j0 on, which need not be a multiple of n.
__device__ __noinline__ uint32_t mask_bits(const uint32_t* mask, int j0, int n, int V) {
    if (j0 >= V) return 0;
    const uint32_t w0 = mask[max(j0, 0) / 32], w1 = mask[min(j0 + n - 1, V - 1) / 32];
    return j0 < 0 ? w0 << -j0 : __funnelshift_r(w0, w1, j0 & 31);
}


// grid: M * ceil(pieces / (8 NV)) blocks of 8 warps; a warp takes NV pieces, 8 apart.
template <typename T, int NV>
__global__ void __launch_bounds__(kLogitsThreads) logits_stream_kernel(const __grid_constant__ LogitsArgs a, const __grid_constant__ LogitsWork w) {
    constexpr int kVec = LogitsVec<T>::kVec, kPiece = LogitsVec<T>::kPiece, kSpan = kLogitsWarps * NV * kPiece;
    __shared__ uint32_t s_path[kSpan / 32];      // path tokens among the block's positions
    const int per_row = (w.pieces + kLogitsWarps * NV - 1) / (kLogitsWarps * NV);
    const int row = blockIdx.x / per_row, block = blockIdx.x - row * per_row, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const T* in = reinterpret_cast<const T*>(a.logits) + (size_t)row * a.ld_in;
    T* out = reinterpret_cast<T*>(a.out) + (a.out ? (size_t)row * a.ld_out : 0);
    const int shift = (int)((reinterpret_cast<uintptr_t>(in) & 15) / sizeof(T)), end = a.V + shift;
    const int p_block = block * kSpan, p0 = p_block + warp * kPiece + lane * kVec;
    uint4 raw[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int p = p0 + i * kLogitsWarps * kPiece;
        raw[i] = p >= shift && p + kVec <= end ? __ldcs(reinterpret_cast<const uint4*>(in - shift + p)) : load_edge(in, p, shift, end);
    }
    const uint32_t* mask = nullptr;
    bool nothing = false;
    if (a.mask) {
        const int mr = a.mask_rows ? a.mask_rows[row] : row;
        nothing = mr >= a.n_masks;               // no such mask: allow nothing
        if (mr >= 0 && !nothing) mask = a.mask + (size_t)mr * a.mask_words;
    }
    const uint32_t* listed = nullptr;
    bool path = false;
    if (w.bitmap) {
        const int seq = a.row_seq ? a.row_seq[row] : row;
        if (seq >= 0 && seq < a.n_seq) {         // a row of no sequence has no lists and no penalties
            listed = w.bitmap + (size_t)seq * a.mask_words;
            path = a.path != nullptr;
        }
    }
    if (path) {
        for (int i = threadIdx.x; i < kSpan / 32; i += kLogitsThreads) s_path[i] = 0;
        __syncthreads();
        if (threadIdx.x < a.path_len) {
            const int token = a.path[(size_t)row * a.path_len + threadIdx.x], at = token + shift - p_block;
            if (token >= 0 && token < a.V && at >= 0 && at < kSpan) atomicOr(&s_path[at >> 5], 1u << (at & 31));
        }
        __syncthreads();
    }
    if (w.bitmap) pdl_wait();                    // the bitmap comes from the kernel before
    const bool vec_out = a.out && (int)((reinterpret_cast<uintptr_t>(out) & 15) / sizeof(T)) == shift;
    auto bits_of = [&](const uint32_t* words, int p) {
        const int j0 = p - shift;
        return shift == 0 && p < end ? __ldg(words + (j0 >> 5)) >> (j0 & 31) : mask_bits(words, j0, kVec, a.V);
    };
    float val[NV][kVec];
    uint32_t top[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int p = p0 + i * kLogitsWarps * kPiece;
        const T* r = reinterpret_cast<const T*>(&raw[i]);
#pragma unroll
        for (int e = 0; e < kVec; ++e) val[i][e] = Elem<T>::up(r[e]);
        uint32_t keep = nothing ? 0u : ~0u, skip = 0;          // bit e: token p + e - shift is allowed; is listed or on the path
        if (mask) keep = bits_of(mask, p);
        if (listed) skip = bits_of(listed, p);
        if (path) skip |= s_path[(p - p_block) >> 5] >> ((p - p_block) & 31);
        skip &= (1u << kVec) - 1;
        if (mask || nothing || skip) {
            const uint32_t bits = keep & ~skip;
#pragma unroll
            for (int e = 0; e < kVec; ++e)
                if (!(bits & (1u << e))) val[i][e] = kNegInf;
        }
        if (a.out) {
            T* to = out - shift + p;
            if (vec_out && p >= shift && p + kVec <= end && !skip) {
                uint4 o;
                T* t = reinterpret_cast<T*>(&o);
#pragma unroll
                for (int e = 0; e < kVec; ++e) t[e] = Elem<T>::down(val[i][e]);
                __stcs(reinterpret_cast<uint4*>(to), o);
            } else store_edge(to, val[i], p, shift, end, skip);
        }
        float m = val[i][0];
#pragma unroll
        for (int e = 1; e < kVec; ++e) m = fmaxf(m, val[i][e]);
        top[i] = __reduce_max_sync(0xffffffffu, logit_order(m));
    }
    uint32_t all = top[0];
#pragma unroll
    for (int i = 1; i < NV; ++i) all = max(all, top[i]);
    const float base = all ? logit_unorder(all) : 0.f;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) sum += exp_sum(val[i], base);
    sum = warp_sum(sum);
    const int piece = block * kLogitsWarps * NV + warp;
    if (lane < NV && piece + lane * kLogitsWarps < w.pieces) {
        uint32_t t = top[0];
#pragma unroll
        for (int i = 1; i < NV; ++i) t = lane == i ? top[i] : t;
        w.piece[(size_t)row * w.pieces + piece + lane * kLogitsWarps] = t;
    }
    if (lane == 0) w.part[(size_t)row * w.parts + block * kLogitsWarps + warp] = make_float2(all ? base : kNegInf, sum);
    pdl_launch_dependents();
}

// ---- the end of a row ----------------------------------------------------------------------------------------
struct LogitsShared {
    unsigned long long buf[kLogitsCap];
    unsigned long long best[32];
    unsigned long long warp_key[kLogitsWarps];
    uint32_t warp_u[32];
    float warp_m[kLogitsWarps], warp_s[kLogitsWarps];
    int n;
    int path[kLogitsMaxPath];
    uint32_t path_bits[64];                      // hashed path tokens, to pass most entries over
};

// Largest key of the block, in every thread.
__device__ __forceinline__ unsigned long long block_max_key(unsigned long long key, LogitsShared& s) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const unsigned long long other = __shfl_xor_sync(0xffffffffu, key, o);
        key = other > key ? other : key;
    }
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s.warp_key[threadIdx.x >> 5] = key;
    __syncthreads();
    unsigned long long best = 0;
#pragma unroll
    for (int w = 0; w < kLogitsWarps; ++w) best = s.warp_key[w] > best ? s.warp_key[w] : best;
    return best;
}

// Ranks the n distinct keys of s.buf by counting the larger ones and leaves the best k in s.best, descending (0 behind the
// last).  Up to 16 neighbouring lanes share the counting for one key.  Begins and ends with a barrier.
__device__ __noinline__ void rank_keys(int n, int k, LogitsShared& s) {
    __syncthreads();
    if (threadIdx.x < 32) s.best[threadIdx.x] = 0;
    __syncthreads();
    const int log2s = n <= kLogitsThreads / 16 ? 4 : n <= kLogitsThreads / 8 ? 3 : n <= kLogitsThreads / 4 ? 2 : n <= kLogitsThreads / 2 ? 1 : 0;
    const int share = 1 << log2s;
    for (int i = 0; (i >> log2s) < n; i += kLogitsThreads) {
        const int at = (i + threadIdx.x) >> log2s;
        const unsigned long long mine = at < n ? s.buf[at] : ~0ull;
        int r = 0;
        for (int j = threadIdx.x & (share - 1); j < n; j += share) r += s.buf[j] > mine ? 1 : 0;
        for (int o = share >> 1; o > 0; o >>= 1) r += __shfl_xor_sync(0xffffffffu, r, o);
        if (at < n && (threadIdx.x & (share - 1)) == 0 && r < k) s.best[r] = mine;
    }
    __syncthreads();
}

// grid: M blocks.
template <typename T>
__global__ void __launch_bounds__(kLogitsThreads) logits_finish_kernel(const __grid_constant__ LogitsArgs a, const __grid_constant__ LogitsWork w) {
    constexpr int kVec = LogitsVec<T>::kVec, kPiece = LogitsVec<T>::kPiece;
    __shared__ LogitsShared s;
    const int row = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const T* in = reinterpret_cast<const T*>(a.logits) + (size_t)row * a.ld_in;
    T* out = reinterpret_cast<T*>(a.out) + (a.out ? (size_t)row * a.ld_out : 0);
    const int shift = (int)((reinterpret_cast<uintptr_t>(in) & 15) / sizeof(T)), end = a.V + shift;
    const uint32_t* mask = nullptr;
    bool nothing = false;
    if (a.mask) {
        const int mr = a.mask_rows ? a.mask_rows[row] : row;
        nothing = mr >= a.n_masks;
        if (mr >= 0 && !nothing) mask = a.mask + (size_t)mr * a.mask_words;
    }
    const int seq = !w.bitmap ? -1 : a.row_seq ? a.row_seq[row] : row;
    const bool known = seq >= 0 && seq < a.n_seq, path = known && a.path;
    const uint32_t* listed = known ? w.bitmap + (size_t)seq * a.mask_words : nullptr;
    if (threadIdx.x == 0) s.n = 0;
    if (threadIdx.x < 64) s.path_bits[threadIdx.x] = 0;
    if (path && threadIdx.x < a.path_len) s.path[threadIdx.x] = a.path[(size_t)row * a.path_len + threadIdx.x];
    __syncthreads();
    auto on_path = [&](int token) { return path && (s.path_bits[(token >> 5) & 63] >> (token & 31)) & 1u; };
    if (path && threadIdx.x < a.path_len && s.path[threadIdx.x] >= 0)
        atomicOr(&s.path_bits[(s.path[threadIdx.x] >> 5) & 63], 1u << (s.path[threadIdx.x] & 31));
    pdl_wait();
    __syncthreads();

    // the k pieces with the largest maxima (equal ones: the lower), in s.best
    const uint32_t* piece = w.piece + (size_t)row * w.pieces;
    uint32_t tau = 0;                            // order of the last one's maximum: no streamed candidate is below it
    int n_pieces = 0;
    if (a.k) {
        uint32_t top = 0;
        for (int i = threadIdx.x; i < w.pieces; i += kLogitsThreads) top = max(top, piece[i]);
        // at least k pieces reach the k-th largest of the warps' four largest threads
        uint32_t best = top;
        for (int i = 0; i < 4; ++i) {
            const uint32_t t = __reduce_max_sync(0xffffffffu, best);
            if (lane == 0) s.warp_u[warp * 4 + i] = t;
            if (lane == __ffs(__ballot_sync(0xffffffffu, best == t)) - 1) best = 0;
        }
        __syncthreads();
        const uint32_t floor = max(kth_largest(s.warp_u[lane], 32, a.k), 1u);
        if (top >= floor)
            for (int i = threadIdx.x; i < w.pieces; i += kLogitsThreads)
                if (piece[i] >= floor) {
                    const int at = atomicAdd(&s.n, 1);
                    if (at < kLogitsCap) s.buf[at] = logit_key(piece[i], i);
                }
        __syncthreads();
        const int n = s.n;
        if (n <= kLogitsCap) rank_keys(n, a.k, s);
        else {                                   // very many pieces with one maximum: k rounds over them
            unsigned long long last = ~0ull;
            for (int i = 0; i < a.k; ++i) {
                unsigned long long key = 0;
                for (int j = threadIdx.x; j < w.pieces; j += kLogitsThreads) {
                    const unsigned long long mine = logit_key(piece[j], j);
                    if (mine < last && mine > key) key = mine;
                }
                last = block_max_key(key, s);
                if (threadIdx.x == 0) s.best[i] = last;
            }
            __syncthreads();
        }
        n_pieces = min(n, a.k);
        if (n_pieces == a.k) tau = (uint32_t)(s.best[a.k - 1] >> 32);
        __syncthreads();
        if (threadIdx.x == 0) s.n = 0;
        __syncthreads();
        // their tokens from tau on; of a piece with more than k of them the best k
        for (int i = warp; i < n_pieces; i += kLogitsWarps) {
            const int p = (int)(0xffffffffu - (uint32_t)s.best[i]) * kPiece + lane * kVec, j0 = p - shift;
            const uint4 raw = p >= shift && p + kVec <= end ? *reinterpret_cast<const uint4*>(in - shift + p) : load_edge(in, p, shift, end);
            const T* r = reinterpret_cast<const T*>(&raw);
            uint32_t keep = ~0u;
            if (mask) keep = mask_bits(mask, j0, kVec, a.V);
            if (listed) keep &= ~mask_bits(listed, j0, kVec, a.V);
            unsigned long long key[kVec];
            int found = 0;
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                bool use = (keep >> e) & 1u;
                if (use && on_path(j0 + e))
                    for (int q = 0; q < a.path_len; ++q) use &= s.path[q] != j0 + e;
                const uint32_t order = use ? logit_order(Elem<T>::up(r[e])) : 0;
                key[e] = order >= max(tau, 1u) ? logit_key(order, j0 + e) : 0;
                found += key[e] != 0;
            }
            const int total = __reduce_add_sync(0xffffffffu, found);
            if (total <= a.k) {
#pragma unroll
                for (int e = 0; e < kVec; ++e)
                    if (key[e]) s.buf[atomicAdd(&s.n, 1)] = key[e];
            } else {
                for (int t = 0; t < a.k; ++t) {
                    unsigned long long best = 0;
#pragma unroll
                    for (int e = 0; e < kVec; ++e) best = key[e] > best ? key[e] : best;
                    const uint32_t hi = __reduce_max_sync(0xffffffffu, (uint32_t)(best >> 32));
                    const uint32_t lo = __reduce_max_sync(0xffffffffu, (uint32_t)(best >> 32) == hi ? (uint32_t)best : 0u);
                    best = ((unsigned long long)hi << 32) | lo;
#pragma unroll
                    for (int e = 0; e < kVec; ++e)
                        if (key[e] == best) {
                            s.buf[atomicAdd(&s.n, 1)] = best;
                            key[e] = 0;
                        }
                }
            }
        }
        __syncthreads();
    }

    // this thread's share of the streamed sums
    float mx = kNegInf, sum = 0.f;
    auto add = [&](float m, float t) {
        if (m > mx) {
            sum *= exp_fast(mx - m);
            mx = m;
        }
        sum += t * exp_fast(m - (mx == kNegInf ? 0.f : mx));
    };
    for (int i = threadIdx.x; i < w.parts; i += kLogitsThreads) {
        const float2 v = w.part[(size_t)row * w.parts + i];
        add(v.x, v.y);
    }
    // the listed tokens, then those of the path that are not listed, one a thread
    if (known) {
        const float rep = a.rep ? a.rep[seq] : 1.f, inv = __frcp_rn(rep), freq = a.freq ? a.freq[seq] : 0.f, pres = a.pres ? a.pres[seq] : 0.f;
        const int2 range = w.range[seq];
        const int total = range.y + (path ? a.path_len : 0);
        uint4 entry = make_uint4(0, 0, 0, 0);
        T raw = Elem<T>::down(0.f);
        auto fetch = [&](int i) {                // the next entry and its logit are on their way while one is worked on
            entry.y = 0;
            if (i < range.y) entry = __ldg(w.entry + range.x + i);
            else if (i < total) {
                const int q = i - range.y, token = s.path[q];
                bool first = token >= 0 && token < a.V && !((listed[token >> 5] >> (token & 31)) & 1u);
                for (int j = 0; j < q; ++j) first &= s.path[j] != token;          // one of equal tokens stands for all
                if (first) entry = make_uint4((uint32_t)token, kCountMask + 1, 0, 0);   // marked; counted below
            }
            if (entry.y) raw = in[entry.x];
        };
        fetch(threadIdx.x);
        __syncthreads();
        int room = kLogitsCap - s.n;
        __syncthreads();                         // read by everyone before the first adds to it
        for (int i0 = 0; i0 < total; i0 += kLogitsThreads) {
            const uint4 e = entry;
            float l = Elem<T>::up(raw);
            const bool extra = i0 + (int)threadIdx.x >= range.y;
            fetch(i0 + kLogitsThreads + threadIdx.x);
            uint32_t order = 0;
            const int token = (int)e.x;
            if (e.y) {
                uint32_t n_out = extra ? 0 : e.y & kCountMask;
                if (on_path(token))
                    for (int q = 0; q < a.path_len; ++q) n_out += s.path[q] == token;
                if (n_out || (!extra && (e.y & kSeenBit))) l = l > 0.f ? divide(l, rep, inv) : __fmul_rn(l, rep);
                if (n_out) l = __fsub_rn(__fsub_rn(l, __fmul_rn(freq, (float)n_out)), pres);
                if (!extra && (e.y & kBiasBit)) l = __fadd_rn(l, __uint_as_float(e.z));
                if (nothing || (mask && !((__ldg(mask + (token >> 5)) >> (token & 31)) & 1u))) l = kNegInf;
                if (a.out) out[token] = Elem<T>::down(l);
                add(l, 1.f);
                order = logit_order(l);
            }
            if (a.k == 0) continue;
            if (order && order >= tau) s.buf[atomicAdd(&s.n, 1)] = logit_key(order, token);
            room -= kLogitsThreads;
            if (room < kLogitsThreads && i0 + kLogitsThreads < total) {           // uniform: room for one more turn at all times
                __syncthreads();
                const int n = s.n;
                rank_keys(n, a.k, s);
                if (threadIdx.x < 32 && threadIdx.x < a.k) s.buf[threadIdx.x] = s.best[threadIdx.x];
                if (threadIdx.x == 0) s.n = min(n, a.k);
                __syncthreads();
                if (n >= a.k) tau = max(tau, (uint32_t)(s.best[a.k - 1] >> 32));
                room = kLogitsCap - a.k;
            }
        }
    }
    // the row's log-sum-exp, added up in a fixed order, and its candidates
    const float m_w = warp_max(mx), s_w = warp_sum(sum * exp_fast(mx - (m_w == kNegInf ? 0.f : m_w)));
    if (lane == 0) { s.warp_m[warp] = m_w; s.warp_s[warp] = s_w; }
    __syncthreads();
    float m = s.warp_m[0], t = 0.f;
#pragma unroll
    for (int i = 1; i < kLogitsWarps; ++i) m = fmaxf(m, s.warp_m[i]);
    const float base = m == kNegInf ? 0.f : m;
#pragma unroll
    for (int i = 0; i < kLogitsWarps; ++i) t += s.warp_s[i] * exp_fast(s.warp_m[i] - base);
    const float lse = base + logf(t);
    if (threadIdx.x == 0 && a.out_lse) a.out_lse[row] = lse;
    if (a.k == 0) return;
    rank_keys(s.n, a.k, s);
    if (threadIdx.x < a.k) {
        const unsigned long long key = s.best[threadIdx.x];
        a.out_ids[(size_t)row * a.k + threadIdx.x] = key ? (int32_t)(0xffffffffu - (uint32_t)key) : kNoToken;
        a.out_logprobs[(size_t)row * a.k + threadIdx.x] = key ? logit_unorder((uint32_t)(key >> 32)) - lse : kNegInf;
    }
}

}  // namespace coral

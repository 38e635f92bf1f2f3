// Penalties for repeated tokens, biases and grammar masks on dense logits, with the candidates of the result in the same
// pass (the dense counterpart of the draft step's merge; the candidates feed the tree expansion).  Per token x of a row:
//   l1 = x seen ? (l > 0 ? l / rep : l * rep) : l      l2 = l1 - freq * count(x)      l3 = l2 - (count(x) > 0 ? pres : 0)
//   l4 = l3 + bias(x)      out = x allowed ? l4 : -inf            (each step one fp32 operation, in this order)
// Bound by the logits' bytes, so a row is streamed once, by a kernel with no more in it than that needs, and what is rare or
// needs a whole row is done by two small kernels around it:
//   logits_lists_kernel   per sequence: counts its token lists into a table in shared memory (whole numbers: the order of the
//                         atomics does not matter) and writes the listed tokens with their counts and biases in the tokens'
//                         order, a bitmap of them, and how many lie before each word of it;
//   logits_narrow_kernel, logits_wide_kernel
//                         read the logits, work on the listed tokens and those of the row's path, apply the mask, write the
//                         result, and keep the maximum of every 512 bytes and (maximum, sum of exponentials) of a warp's part;
//   logits_finish_kernel  per row: the log-sum-exp, and the candidates: only the k pieces of 512 bytes with the largest maxima
//                         can hold one, so only they are read again.
// 960 rows x 128256 in 16 sequences with lists, path, mask, result and 10 candidates: 206 us fp32, 198 us bf16; of those the
// lists 16 and the end of the rows 25.  Reading alone takes 97 / 62 us, reading and writing 161 / 87 (bytes: 75 / 38, 151 / 75).
// What bounds the stream is instructions (13 a logit for reading, 30 with everything; 60% of the issue slots).
// (Everything in one kernel, a cluster of blocks a row, took 850 us: candidates and lists cost each block a chain of barriers a
// row, and their code pushed the streaming loop out of the instruction cache.  Listed tokens adjusted by the thread that holds
// them took 500 to 600 us: a warp with one such token waits for its entry and runs the arithmetic for it alone.  Blocks of one
// span each took 355 / 288: a span's chain of loads with nothing else on its way.)
#pragma once
#include <cooperative_groups.h>

#include <type_traits>

#include "cp_async.cuh"
#include "element.cuh"

namespace coral {

constexpr int kLogitsThreads = 256;
constexpr int kLogitsWarps = kLogitsThreads / 32;
constexpr int kLogitsCap = 2048;                 // keys ranked by counting
constexpr int kListThreads = 1024;
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
    uint32_t* before;                            // [n_seq][mask_words] its entry of a word's first listed token, counted over all
    uint2* entry;                                // table word and bias of listed tokens, a sequence's from its lists' offsets on
    int32_t* token;                              // which tokens they are
    int2* range;                                 // [n_seq] first entry and number
    uint32_t* piece;                             // [M][pieces] largest value (logit_order) of 512 bytes of logits
    float2* part;                                // [M][parts] maximum and sum of what a warp took
    int pieces, parts, chunk;                    // chunk: spans of a row that a block takes; 0: the kernel for few rows
    int late;                                    // over the logits, in 16 bits: the last kernel stores listed tokens
    int final;                                   // over the logits, in 32 bits: the last kernel reads results, not logits
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

// e^(v - base) of two values.
__device__ __forceinline__ unsigned long long exp_pair(float v0, float v1, unsigned long long minus_base) {
    unsigned long long t = pair_of(v0, v1);
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(t) : "l"(t), "l"(minus_base));
    float2 f = halves(mul2(t, pair_of(1.4426950408889634f, 1.4426950408889634f)));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(f.x) : "f"(f.x));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(f.y) : "f"(f.y));
    return pair_of(f.x, f.y);
}
__device__ __forceinline__ unsigned long long add_pair(unsigned long long a, unsigned long long b) {
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(a) : "l"(a), "l"(b));
    return a;
}
// Sums of e^(v - base) over N values (a power of two), as two halves and as a tree.
template <int N>
__device__ __forceinline__ unsigned long long exp_sum(const float* val, unsigned long long minus_base) {
    if constexpr (N == 2) return exp_pair(val[0], val[1], minus_base);
    else return add_pair(exp_sum<N / 2>(val, minus_base), exp_sum<N / 2>(val + N / 2, minus_base));
}
// The warp's largest value; NaN only if every one is.
__device__ __forceinline__ float warp_top(float v) {
    asm("redux.sync.max.f32 %0, %0, 0xffffffff;" : "+f"(v));
    return v;
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
__global__ void __launch_bounds__(kListThreads, 1) logits_lists_kernel(const __grid_constant__ LogitsArgs a, const __grid_constant__ LogitsWork w) {
    namespace cg = cooperative_groups;
    extern __shared__ __align__(16) uint32_t tables[];
    constexpr int kWords = kListWindow / 32;
    __shared__ uint32_t s_bits[kWords];
    __shared__ int s_warp[kListThreads / 32], s_total[2][kListCluster];      // every block's total, pushed by it
    auto cluster = cg::this_cluster();
    const int seq = blockIdx.x / kListCluster, rank = blockIdx.x % kListCluster, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t* places = tables + kListWindow;
    pdl_launch_dependents();
    cluster.barrier_arrive();                    // every block has started before another writes to it
    long long p0 = 0, p1 = 0, o0 = 0, o1 = 0, b0 = 0, b1 = 0;
    if (a.prompt) list_range(a.prompt_off, seq, a.prompt_total, p0, p1);
    if (a.output) list_range(a.output_off, seq, a.output_total, o0, o1);
    if (a.bias_tokens) list_range(a.bias_off, seq, a.bias_total, b0, b1);
    const long long first = p0 + o0 + b0;        // a sequence has room for as many entries as its lists are long
    long long at = first;
    int turn = 0;
    for (int base = 0; base < a.V; base += kListCluster * kListWindow, turn ^= 1) {
        const int lo = base + rank * kListWindow, n = min(kListWindow, a.V - lo);           // n < 1: behind the last token
        const int words = (a.bias_tokens ? 2 : 1) * kListWindow;
        for (int i = threadIdx.x * 4; i < words; i += kListThreads * 4) *reinterpret_cast<uint4*>(tables + i) = make_uint4(0, 0, 0, 0);
        for (int i = threadIdx.x; i < kWords; i += kListThreads) s_bits[i] = 0;
        __syncthreads();
        auto each = [&](const int32_t* tokens, long long from, long long to, auto put) {
            for (long long i = from + threadIdx.x; i < to; i += 4 * kListThreads) {
                int32_t t[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) t[u] = i + u * kListThreads < to ? tokens[i + u * kListThreads] : -1;
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int x = t[u] - lo;
                    if (t[u] < lo || x >= n) continue;
                    // whoever finds the word empty is the first to list the token
                    if (put(x, (uint32_t)(i + u * kListThreads - from) + 1u) == 0) atomicOr(&s_bits[x >> 5], 1u << (x & 31));
                }
            }
        };
        if (a.prompt) each(a.prompt, p0, p1, [&](int x, uint32_t) { return atomicOr(tables + x, kSeenBit); });
        if (a.output) each(a.output, o0, o1, [&](int x, uint32_t) { return atomicAdd(tables + x, 1u); });
        if (a.bias_tokens)
            each(a.bias_tokens, b0, b1, [&](int x, uint32_t place) {
                atomicMax(places + x, place);
                return atomicOr(tables + x, kBiasBit);
            });
        __syncthreads();
        // entries before each word of the bitmap: over the block, then over the cluster
        const uint32_t bits = threadIdx.x < kWords ? s_bits[threadIdx.x] : 0;
        int upto = __popc(bits);
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += v;
        }
        if (lane == 31) s_warp[warp] = upto;
        __syncthreads();
        int before = upto - __popc(bits), total = 0;
#pragma unroll
        for (int i = 0; i < kWords / 32; ++i) {
            before += i < warp ? s_warp[i] : 0;
            total += s_warp[i];
        }
        if (base == 0) cluster.barrier_wait();
        if (threadIdx.x < kListCluster) *cluster.map_shared_rank(&s_total[turn][rank], threadIdx.x) = total;
        cluster.sync();                          // (a buffer is written again behind the next one's, when all have read it)
        long long next = at;
#pragma unroll
        for (int c = 0; c < kListCluster; ++c) {
            if (c < rank) before += s_total[turn][c];
            next += s_total[turn][c];
        }
        if (threadIdx.x < kWords && (int)threadIdx.x * 32 < n) {
            const size_t word = (size_t)seq * a.mask_words + lo / 32 + threadIdx.x;
            w.bitmap[word] = bits;
            w.before[word] = (uint32_t)(at + before);
            for (uint32_t left = bits; left; left &= left - 1, ++before) {
                const int x = threadIdx.x * 32 + __ffs(left) - 1;
                w.entry[at + before] = make_uint2(tables[x], 0);
                w.token[at + before] = lo + x;
                tables[x] = (uint32_t)before;    // by which the biases find it
            }
        }
        if (a.bias_tokens) {
            __syncthreads();
            for (long long i = b0 + threadIdx.x; i < b1; i += kListThreads) {
                const int t = a.bias_tokens[i], x = t - lo;
                if (t >= lo && x < n && places[x] == (uint32_t)(i - b0) + 1u) w.entry[at + tables[x]].y = __float_as_uint(a.bias_values[i]);
            }
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
__device__ __forceinline__ void store_edge(T* to, const float (&val)[N], int p, int shift, int end, uint32_t listed) {
#pragma unroll
    for (int e = 0; e < N; ++e)
        if (p + e >= shift && p + e < end && !((listed >> e) & 1u)) to[e] = Elem<T>::down(val[e]);
}
// Bits of a row's bitmap for the n tokens from j0 on, which need not be a multiple of n.
__device__ __noinline__ uint32_t mask_bits(const uint32_t* mask, int j0, int n, int V) {
    if (j0 >= V) return 0;
    const uint32_t w0 = mask[max(j0, 0) / 32], w1 = mask[min(j0 + n - 1, V - 1) / 32];
    return j0 < 0 ? w0 << -j0 : __funnelshift_r(w0, w1, j0 & 31);
}


// A row's parameters for tokens of its lists and its path.
struct LogitsRow {
    float rep, inv, freq, pres;
    const uint32_t *listed, *before;             // of the row's sequence; null: none
    const int32_t* path;                         // null: none
};
__device__ __forceinline__ LogitsRow row_params(const LogitsArgs& a, const LogitsWork& w, int row, int seq) {
    LogitsRow r{1.f, 1.f, 0.f, 0.f, nullptr, nullptr, nullptr};
    if (!w.bitmap || seq < 0 || seq >= a.n_seq) return r;              // a row of no sequence has no lists and no penalties
    if (a.rep) r.rep = a.rep[seq];
    if (a.freq) r.freq = a.freq[seq];
    if (a.pres) r.pres = a.pres[seq];
    r.inv = __frcp_rn(r.rep);
    r.listed = w.bitmap + (size_t)seq * a.mask_words;
    r.before = w.before + (size_t)seq * a.mask_words;
    if (a.path) r.path = a.path + (size_t)row * a.path_len;
    return r;
}

// Penalties and bias of a token with this entry (zeros: it is on the path only).
__device__ __forceinline__ float adjust_inline(float l, int token, uint2 e, const LogitsRow& r, int path_len) {
    uint32_t n = e.x & kCountMask;
    if (r.path)
        for (int q = 0; q < path_len; ++q) n += r.path[q] == token;
    if (n || (e.x & kSeenBit)) l = l > 0.f ? divide(l, r.rep, r.inv) : __fmul_rn(l, r.rep);
    if (n) l = __fsub_rn(__fsub_rn(l, __fmul_rn(r.freq, (float)n)), r.pres);
    if (e.x & kBiasBit) l = __fadd_rn(l, __uint_as_float(e.y));
    return l;
}
__device__ __noinline__ float adjust(float l, int token, uint2 e, const LogitsRow& r, int path_len) {
    return adjust_inline(l, token, e, r, path_len);
}
// The entry of the first listed token from token j on: the number of those before it.
__device__ __forceinline__ uint32_t entry_at(const LogitsRow& r, int j) {
    return __ldcg(r.before + (j >> 5)) + __popc(__ldcg(r.listed + (j >> 5)) & ((1u << (j & 31)) - 1));
}
__device__ __forceinline__ bool is_listed(const LogitsRow& r, int token) { return (__ldcg(r.listed + (token >> 5)) >> (token & 31)) & 1u; }
__device__ __forceinline__ uint2 entry_of(const LogitsRow& r, const LogitsWork& w, int token) {
    return is_listed(r, token) ? __ldcg(w.entry + entry_at(r, token)) : make_uint2(0, 0);
}

// A row as a block of the streaming kernels sees it.
template <typename T>
struct LogitsIn {
    const T* in;
    T* out;                                      // null: no result is written
    int shift, end, seq;
    bool nothing, vec_out;                       // no token is allowed; vectors of the result start on 16 bytes as those read do
    const uint32_t* mask;                        // null: every token is allowed
    __device__ __forceinline__ LogitsIn(const LogitsArgs& a, int row, bool lists) {
        seq = !lists ? -1 : a.row_seq ? a.row_seq[row] : row;
        const int mr = !a.mask ? -1 : a.mask_rows ? a.mask_rows[row] : row;
        in = reinterpret_cast<const T*>(a.logits) + (size_t)row * a.ld_in;
        out = a.out ? reinterpret_cast<T*>(a.out) + (size_t)row * a.ld_out : nullptr;
        shift = (int)((reinterpret_cast<uintptr_t>(in) & 15) / sizeof(T));
        end = a.V + shift;
        nothing = a.mask && mr >= a.n_masks;                                       // no such mask: allow nothing
        mask = mr >= 0 && !nothing ? a.mask + (size_t)mr * a.mask_words : nullptr;
        vec_out = out && (int)((reinterpret_cast<uintptr_t>(out) & 15) / sizeof(T)) == shift;
    }
    __device__ __forceinline__ bool whole(int p) const { return p >= shift && p + LogitsVec<T>::kVec <= end; }
    // the word of the mask that holds the vector at p, where one word does
    __device__ __forceinline__ uint32_t keep_word(int p, int V) const { return mask && shift == 0 ? __ldg(mask + (min(p, V - 1) >> 5)) : 0; }
    // Masks and writes the vector at p; the largest of its values.  skip: positions that are not written.  PLAIN: the vector is
    // whole, it can be stored whole, and one word of the mask holds it.
    template <bool PLAIN>
    __device__ __forceinline__ float finish(float (&val)[LogitsVec<T>::kVec], int p, uint32_t word, uint32_t skip, int V) const {
        constexpr int kVec = LogitsVec<T>::kVec;
        if (mask || nothing) {
            const uint32_t keep = nothing ? 0u : PLAIN || shift == 0 ? word >> (p & 31) : mask_bits(mask, p - shift, kVec, V);
#pragma unroll
            for (int e = 0; e < kVec; ++e)
                if (!(keep & (1u << e))) val[e] = kNegInf;
        }
        if (out) {
            T* to = out - shift + p;
            if ((PLAIN || (vec_out && whole(p))) && !skip) {
                uint4 o;
                T* t = reinterpret_cast<T*>(&o);
#pragma unroll
                for (int e = 0; e < kVec; ++e) t[e] = Elem<T>::down(val[e]);
                __stcs(reinterpret_cast<uint4*>(to), o);
            } else store_edge(to, val, p, shift, end, skip);
        }
        float m = val[0];
#pragma unroll
        for (int e = 1; e < kVec; ++e) m = fmaxf(m, val[e]);
        return m;
    }
};

// Few rows: a block of 8 warps takes 8 pieces, so that many SMs share a row.  grid: M * ceil(pieces / 8).
// LISTS: the call has token lists, paths or biases.
template <typename T, bool LISTS>
__global__ void __launch_bounds__(kLogitsThreads) logits_narrow_kernel(const __grid_constant__ LogitsArgs a, const __grid_constant__ LogitsWork w) {
    constexpr int kVec = LogitsVec<T>::kVec, kPiece = LogitsVec<T>::kPiece, kSpan = kLogitsWarps * kPiece;
    __shared__ __align__(16) float s_adjusted[LISTS ? kSpan : 1];
    __shared__ uint32_t s_special[LISTS ? kSpan / 32 : 1];
    const int per_row = (w.pieces + kLogitsWarps - 1) / kLogitsWarps;
    const int row = blockIdx.x / per_row, block = blockIdx.x - row * per_row, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    pdl_launch_dependents();                     // the last kernel waits for this one's end, its launch need not
    const LogitsIn<T> r(a, row, LISTS);
    const int p_block = block * kSpan, p = p_block + threadIdx.x * kVec;
    const uint4 raw = r.whole(p) ? __ldcs(reinterpret_cast<const uint4*>(r.in - r.shift + p)) : load_edge(r.in, p, r.shift, r.end);
    const uint32_t word = r.keep_word(p, a.V);
    uint32_t special = 0;
    float val[kVec];
#pragma unroll
    for (int e = 0; e < kVec; ++e) val[e] = Elem<T>::up(reinterpret_cast<const T*>(&raw)[e]);
    if (LISTS) {
        const LogitsRow par = row_params(a, w, row, r.seq);
        for (int i = threadIdx.x; i < kSpan / 32; i += kLogitsThreads) s_special[i] = 0;
        pdl_wait();                              // what follows of the lists comes from the kernel before
        if (par.listed) {                        // one thread a token that is listed or on the path, wherever it lies in the block
            const int lo = max(p_block - r.shift, 0), hi = min(p_block + kSpan - r.shift, a.V);
            uint32_t first = 0;
            int n = 0;                           // (the last block of a row may lie behind its end)
            if (lo < hi) {
                first = entry_at(par, lo);
                if (hi < a.V) n = (int)(entry_at(par, hi) - first);
                else {
                    const int2 range = __ldcg(w.range + r.seq);
                    n = range.x + range.y - (int)first;
                }
            }
            __syncthreads();
            const int total = n + (par.path ? a.path_len : 0);
#pragma unroll 1
            for (int i = threadIdx.x; i < total; i += kLogitsThreads) {
                int token;
                uint2 entry = make_uint2(0, 0);
                if (i < n) {
                    token = __ldcg(w.token + first + i);
                    entry = __ldcg(w.entry + first + i);
                    if (token < lo || token >= hi) continue;           // decreasing offsets: another sequence wrote here
                } else {
                    token = par.path[i - n];
                    if (token < lo || token >= hi || is_listed(par, token)) continue;
                }
                const int at = token + r.shift - p_block;
                s_adjusted[at] = adjust_inline(Elem<T>::up(r.in[token]), token, entry, par, a.path_len);
                atomicOr(&s_special[at >> 5], 1u << (at & 31));
            }
            __syncthreads();
            special = (s_special[(p - p_block) >> 5] >> (p & 31)) & ((1u << kVec) - 1);
#pragma unroll
            for (int e = 0; e < kVec; ++e)
                if ((special >> e) & 1u) val[e] = s_adjusted[p - p_block + e];
        }
    }
    const float top = warp_top(r.template finish<false>(val, p, word, w.late ? special : 0, a.V)), base = top > kNegInf ? top : 0.f;
    const float2 two = halves(exp_sum<kVec>(val, pair_of(-base, -base)));
    const float sum = warp_sum(two.x + two.y);
    const int piece = block * kLogitsWarps + warp;
    if (lane == 0) {
        if (piece < w.pieces) w.piece[(size_t)row * w.pieces + piece] = logit_order(top);
        w.part[(size_t)row * w.parts + piece] = make_float2(top > kNegInf ? top : kNegInf, sum);
    }
}

// Many rows: a block takes w.chunk neighbouring spans of a row one after the other.  Every thread copies its own vectors of the
// next spans into its own slots, so that loads are in flight all the time, and the next listed tokens' entries are loaded a span
// ahead (the tokens are in order: those of a span are the next ones below its end).
// grid: M * ceil(spans / chunk)
constexpr int kWideSpan = 4096;
template <typename T>
struct LogitsWide {
    static constexpr int kNV = kWideSpan * (int)sizeof(T) / (16 * kLogitsThreads), kStages = sizeof(T) == 4 ? 3 : 4;
    static constexpr int kRaw = kStages * kWideSpan * (int)sizeof(T);
    // 32 bits: listed tokens are adjusted where they lie; 16 bits: in fp32 copies behind them
    static constexpr int smem(bool lists) { return kRaw + (lists && sizeof(T) == 2 ? kWideSpan * 4 : 0); }
};
template <typename T, bool LISTS>
__global__ void __launch_bounds__(kLogitsThreads, 4) logits_wide_kernel(const __grid_constant__ LogitsArgs a, const __grid_constant__ LogitsWork w) {
    constexpr int kVec = LogitsVec<T>::kVec, kPiece = LogitsVec<T>::kPiece, kNV = LogitsWide<T>::kNV, kStages = LogitsWide<T>::kStages;
    extern __shared__ __align__(16) uint4 wide_raw[];                  // [kStages][kNV][threads]
    __shared__ uint32_t s_special[2][LISTS ? kWideSpan / 32 : 1];
    constexpr int kSpanPieces = kWideSpan / kPiece;
    const int spans = (w.pieces + kSpanPieces - 1) / kSpanPieces, per_row = w.parts / kLogitsWarps;
    const int row = blockIdx.x / per_row, block = blockIdx.x - row * per_row, s0 = block * w.chunk, s1 = min(s0 + w.chunk, spans);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    pdl_launch_dependents();
    const LogitsIn<T> r(a, row, LISTS);
    auto inner = [&](int s) { return s * kWideSpan >= r.shift && (s + 1) * kWideSpan <= r.end; };
    const bool plain_row = (!r.out || r.vec_out) && (!r.mask || r.shift == 0);
    int to_stage = 0;
    auto load = [&](int s) {
        uint4* to = wide_raw + to_stage * (kNV * kLogitsThreads) + threadIdx.x;
        const T* from = r.in - r.shift + (size_t)s * kWideSpan + threadIdx.x * kVec;
        if (s < s1) {
            if (inner(s)) {
#pragma unroll
                for (int i = 0; i < kNV; ++i) cp_async16(to + i * kLogitsThreads, from + i * kLogitsThreads * kVec);
            } else {
#pragma unroll 1
                for (int i = 0; i < kNV; ++i) {
                    const int p = s * kWideSpan + (i * kLogitsThreads + threadIdx.x) * kVec;
                    if (r.whole(p)) cp_async16(to + i * kLogitsThreads, from + i * kLogitsThreads * kVec);
                    else to[i * kLogitsThreads] = load_edge(r.in, p, r.shift, r.end);
                }
            }
        }
        cp_async_commit();
        to_stage = to_stage + 1 == kStages ? 0 : to_stage + 1;
    };
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) load(s0 + i);
    const LogitsRow par = row_params(a, w, row, r.seq);
    uint32_t word[kNV];                          // the next span's words of the mask
#pragma unroll
    for (int i = 0; i < kNV; ++i) word[i] = r.keep_word(s0 * kWideSpan + (i * kLogitsThreads + threadIdx.x) * kVec, a.V);
    constexpr int kNone = 0x7fffffff;
    int token = kNone, path_token = kNone, next = 0, last = 0;         // the thread's next listed token, its token of the path; entries
    uint2 entry = make_uint2(0, 0);
    auto fetch = [&] {
        token = kNone;
        if (next + (int)threadIdx.x < last) {
            token = __ldcg(w.token + next + threadIdx.x);
            entry = __ldcg(w.entry + next + threadIdx.x);
        }
    };
    if (LISTS) {
        if (threadIdx.x < kWideSpan / 32) s_special[0][threadIdx.x] = 0;
        pdl_wait();                              // what follows of the lists comes from the kernel before
        if (par.listed) {
            const int lo = max(s0 * kWideSpan - r.shift, 0);
            if (lo < a.V) {                      // (the last span of a row may lie behind its end)
                const int2 range = __ldcg(w.range + r.seq);
                next = (int)entry_at(par, lo);
                last = range.x + range.y;
            }
            fetch();
            if (par.path && warp * 32 < a.path_len) {
                if ((int)threadIdx.x < a.path_len) path_token = par.path[threadIdx.x];
                if (path_token < 0 || path_token >= a.V || is_listed(par, path_token)) path_token = kNone;
                // one thread a token: it is adjusted in place, and the count has its repeats already
                if (__ffs(__match_any_sync(0xffffffffu, path_token)) - 1 != lane) path_token = kNone;
#pragma unroll 8
                for (int q = 0; q < warp * 32; ++q)
                    if (par.path[q] == path_token) path_token = kNone;
            }
        }
    }
    float base = kNegInf;                        // the warp's largest value so far, and the thread's sums of e^(value - base)
    unsigned long long sum = pair_of(0.f, 0.f);
    int stage = 0;
#pragma unroll 1
    for (int s = s0; s < s1; ++s, stage = stage + 1 == kStages ? 0 : stage + 1) {
        uint4* raw = wide_raw + stage * (kNV * kLogitsThreads);
        float* adjusted = reinterpret_cast<float*>(sizeof(T) == 4 ? raw : wide_raw + LogitsWide<T>::kRaw / 16);
        const int p_span = s * kWideSpan;
        cp_async_wait<kStages - 2>();
        if (LISTS && par.listed) {               // one thread a token that is listed or on the path, wherever it lies in the span
            if (sizeof(T) == 2)
#pragma unroll
                for (int i = 0; i < kNV; ++i) {
                    const int v = i * kLogitsThreads + threadIdx.x;
                    const uint4 x = raw[v];
#pragma unroll
                    for (int e = 0; e < kVec; e += 4) {
                        const T* t = reinterpret_cast<const T*>(&x) + e;
                        *reinterpret_cast<float4*>(adjusted + v * kVec + e) = make_float4(Elem<T>::up(t[0]), Elem<T>::up(t[1]), Elem<T>::up(t[2]), Elem<T>::up(t[3]));
                    }
                }
            __syncthreads();
            uint32_t* marks = s_special[(s - s0) & 1];
            auto put = [&](int t, uint2 e) {
                const int at = t + r.shift - p_span;
                adjusted[at] = adjust_inline(adjusted[at], t, e, par, a.path_len);
                if (w.late) atomicOr(&marks[at >> 5], 1u << (at & 31));
            };
            if (w.late && threadIdx.x < kWideSpan / 32) s_special[(s - s0 + 1) & 1][threadIdx.x] = 0;
            const int lo = p_span - r.shift, hi = lo + kWideSpan;
            if (path_token >= lo && path_token < hi) put(path_token, make_uint2(0, 0));
            int found;
            do {
                const bool here = token >= lo && token < hi;           // (below lo: decreasing offsets, another sequence wrote here)
                if (here) put(token, entry);
                found = __syncthreads_count(here);
                next += found;
                if (found) fetch();
            } while (found == kLogitsThreads);
        }
        load(s + kStages - 1);
        auto work = [&](auto plain) {
            float val[kNV][kVec], top[kNV];
#pragma unroll
            for (int i = 0; i < kNV; ++i) {
                const int v = i * kLogitsThreads + threadIdx.x, p = p_span + v * kVec;
                uint32_t skip = 0;
                if (LISTS && sizeof(T) == 2 && par.listed) {
#pragma unroll
                    for (int e = 0; e < kVec; e += 4) *reinterpret_cast<float4*>(&val[i][e]) = *reinterpret_cast<const float4*>(adjusted + v * kVec + e);
                    if (w.late) skip = (s_special[(s - s0) & 1][(v * kVec) >> 5] >> (p & 31)) & ((1u << kVec) - 1);
                } else {
                    const uint4 x = raw[v];
#pragma unroll
                    for (int e = 0; e < kVec; ++e) val[i][e] = Elem<T>::up(reinterpret_cast<const T*>(&x)[e]);
                }
                top[i] = warp_top(r.template finish<decltype(plain)::value>(val[i], p, word[i], skip, a.V));
            }
            if (r.mask)
#pragma unroll
                for (int i = 0; i < kNV; ++i) word[i] = r.keep_word(p_span + kWideSpan + (i * kLogitsThreads + threadIdx.x) * kVec, a.V);
            float all = top[0];
#pragma unroll
            for (int i = 1; i < kNV; ++i) all = fmaxf(all, top[i]);
            if (all > base) {
                const float f = exp_fast(base - all);
                sum = mul2(sum, pair_of(f, f));
                base = all;
            }
            const float from = base > kNegInf ? base : 0.f;
            sum = add_pair(sum, exp_sum<kNV * kVec>(&val[0][0], pair_of(-from, -from)));
            const int piece = s * kSpanPieces + warp + lane * kLogitsWarps;
            if (a.k && lane < kNV && piece < w.pieces) {
                float t = top[0];
#pragma unroll
                for (int i = 1; i < kNV; ++i) t = lane == i ? top[i] : t;
                w.piece[(size_t)row * w.pieces + piece] = logit_order(t);
            }
        };
        if (plain_row && inner(s)) work(std::true_type{});
        else work(std::false_type{});
    }
    const float2 two = halves(sum);
    const float total = warp_sum(two.x + two.y);
    if (lane == 0) w.part[(size_t)row * w.parts + block * kLogitsWarps + warp] = make_float2(base, total);
    cp_async_wait<0>();
}

// ---- the end of a row ----------------------------------------------------------------------------------------
template <int WARPS>
struct LogitsShared {
    unsigned long long buf[kLogitsCap];
    uint32_t value[WARPS][256];           // a piece of a warp's (logit_order)
    unsigned long long best[32];
    unsigned long long warp_key[WARPS];
    uint32_t warp_u[32];
    float warp_m[WARPS], warp_s[WARPS];
    int n;
};

// Largest key of the block, in every thread.
template <int WARPS>
__device__ __forceinline__ unsigned long long block_max_key(unsigned long long key, LogitsShared<WARPS>& s) {
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
    for (int w = 0; w < WARPS; ++w) best = s.warp_key[w] > best ? s.warp_key[w] : best;
    return best;
}

// Ranks the n distinct keys of s.buf by counting the larger ones and leaves the best k in s.best, descending (0 behind the
// last).  Up to 16 neighbouring lanes share the counting for one key.  Begins and ends with a barrier.
template <int WARPS>
__device__ __noinline__ void rank_keys(int n, int k, LogitsShared<WARPS>& s) {
    __syncthreads();
    if (threadIdx.x < 32) s.best[threadIdx.x] = 0;
    __syncthreads();
    const int log2s = n <= WARPS * 32 / 16 ? 4 : n <= WARPS * 32 / 8 ? 3 : n <= WARPS * 32 / 4 ? 2 : n <= WARPS * 32 / 2 ? 1 : 0;
    const int share = 1 << log2s;
    for (int i = 0; (i >> log2s) < n; i += WARPS * 32) {
        const int at = (i + threadIdx.x) >> log2s;
        const unsigned long long mine = at < n ? s.buf[at] : ~0ull;
        int r = 0;
        for (int j = threadIdx.x & (share - 1); j < n; j += share) r += s.buf[j] > mine ? 1 : 0;
        for (int o = share >> 1; o > 0; o >>= 1) r += __shfl_xor_sync(0xffffffffu, r, o);
        if (at < n && (threadIdx.x & (share - 1)) == 0 && r < k) s.best[r] = mine;
    }
    __syncthreads();
}

// The rank of every lane's key among the first n lanes' (distinct ones, n <= 32); 32 and more behind them.
__device__ __forceinline__ int warp_rank(unsigned long long key, int n) {
    int r = (int)(threadIdx.x & 31) < n ? 0 : 32;
    for (int j = 0; j < n; ++j) r += __shfl_sync(0xffffffffu, key, j) > key ? 1 : 0;
    return r;
}

// grid: M blocks of 16 warps, or of 8 where those would take several rounds (one row 16 and 17 us a call, 960 rows 209 and 206).
template <typename T, int WARPS>
__global__ void __launch_bounds__(WARPS * 32) logits_finish_kernel(const __grid_constant__ LogitsArgs a, const __grid_constant__ LogitsWork w) {
    constexpr int kVec = LogitsVec<T>::kVec, kPiece = LogitsVec<T>::kPiece, kMost = 32 / WARPS, kHeld = 64 / WARPS;
    constexpr int kTops = 32 / WARPS;               // of a warp's values, for a first bound
    __shared__ LogitsShared<WARPS> s;
    const int row = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const T* in = reinterpret_cast<const T*>(a.logits) + (size_t)row * a.ld_in;
    T* out = reinterpret_cast<T*>(a.out) + (a.out ? (size_t)row * a.ld_out : 0);
    const int shift = (int)((reinterpret_cast<uintptr_t>(in) & 15) / sizeof(T)), end = a.V + shift;
    const int seq = !w.bitmap ? -1 : a.row_seq ? a.row_seq[row] : row, mr = !a.mask ? -1 : a.mask_rows ? a.mask_rows[row] : row;
    const bool nothing = mr >= a.n_masks && a.mask;
    const uint32_t* const mask = mr >= 0 && !nothing ? a.mask + (size_t)mr * a.mask_words : nullptr;
    if (threadIdx.x == 0) s.n = 0;
    const LogitsRow par = row_params(a, w, row, seq);
    pdl_wait();

    // this thread's share of the streamed sums, and of the pieces' maxima
    float mx = kNegInf, sum = 0.f;
    auto add = [&](float m, float t) {
        if (m > mx) {
            sum *= exp_fast(mx - m);
            mx = m;
        }
        sum += t * exp_fast(m - (mx == kNegInf ? 0.f : mx));
    };
    const uint32_t* piece = w.piece + (size_t)row * w.pieces;
    uint32_t held[kHeld], top = 0;               // the thread's first pieces; those of very long rows are read again
    if (a.k) {
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            const int at = threadIdx.x + i * WARPS * 32;
            held[i] = at < w.pieces ? piece[at] : 0;
        }
#pragma unroll
        for (int i = 0; i < kHeld; ++i) top = max(top, held[i]);
        for (int i = threadIdx.x + kHeld * WARPS * 32; i < w.pieces; i += WARPS * 32) top = max(top, piece[i]);
    }
#pragma unroll 4
    for (int i = threadIdx.x; i < w.parts; i += WARPS * 32) {
        const float2 v = w.part[(size_t)row * w.parts + i];
        add(v.x, v.y);
    }

    uint32_t tau = 0;                            // a lower bound of the k-th candidate (logit_order)
    if (a.k) {
        // the k largest of the warps' largest values: k distinct ones, so the k-th bounds what is asked for
        auto bound_of = [&](uint32_t v) {
#pragma unroll
            for (int i = 0; i < kTops; ++i) { // (the barrier behind it also covers s.n)
                const uint32_t t = __reduce_max_sync(0xffffffffu, v);
                if (lane == 0) s.warp_u[warp * kTops + i] = t;
                if (lane == __ffs(__ballot_sync(0xffffffffu, v == t)) - 1) v = 0;
            }
            __syncthreads();
            return kth_largest(s.warp_u[lane], 32, a.k);
        };
        // the k pieces with the largest maxima (equal ones: the lower)
        tau = bound_of(top);
        const uint32_t floor = max(tau, 1u);
        auto collect = [&](uint32_t v, int i) {
            if (v < floor) return;
            const int at = atomicAdd(&s.n, 1);
            if (at < kLogitsCap) s.buf[at] = logit_key(v, i);
        };
        if (top >= floor) {
#pragma unroll
            for (int i = 0; i < kHeld; ++i) collect(held[i], threadIdx.x + i * WARPS * 32);
            for (int i = threadIdx.x + kHeld * WARPS * 32; i < w.pieces; i += WARPS * 32) collect(piece[i], i);
        }
        __syncthreads();
        const int n = s.n, n_pieces = min(n, a.k);
        // piece number i of this warp, in pos[i]; -1: none
        int pos[kMost];
        if (n <= 32) {
            const unsigned long long key = lane < n ? s.buf[lane] : 0;
            const int r = warp_rank(key, n);
#pragma unroll
            for (int i = 0; i < kMost; ++i) {
                const int want = warp + i * WARPS;
                const unsigned long long k_i = __shfl_sync(0xffffffffu, key, (__ffs(__ballot_sync(0xffffffffu, r == want)) - 1) & 31);
                pos[i] = want < n_pieces ? (int)(0xffffffffu - (uint32_t)k_i) : -1;
            }
            if (n >= a.k)
                tau = max(tau, (uint32_t)(__shfl_sync(0xffffffffu, key, (__ffs(__ballot_sync(0xffffffffu, r == a.k - 1)) - 1) & 31) >> 32));
        } else {
            if (n <= kLogitsCap) rank_keys(n, a.k, s);
            else {                               // very many pieces with one maximum: k rounds over them
                unsigned long long last = ~0ull;
                for (int i = 0; i < a.k; ++i) {
                    unsigned long long key = 0;
                    for (int j = threadIdx.x; j < w.pieces; j += WARPS * 32) {
                        const unsigned long long mine = logit_key(piece[j], j);
                        if (mine < last && mine > key) key = mine;
                    }
                    last = block_max_key(key, s);
                    if (threadIdx.x == 0) s.best[i] = last;
                }
                __syncthreads();
            }
#pragma unroll
            for (int i = 0; i < kMost; ++i) {
                const int want = warp + i * WARPS;
                pos[i] = want < n_pieces ? (int)(0xffffffffu - (uint32_t)s.best[want]) : -1;
            }
            tau = max(tau, (uint32_t)(s.best[a.k - 1] >> 32));
        }
        // Their values that may be candidates.  With few pieces their maxima bound little: a first pass takes a bound from lanes'
        // maxima over all their values.
#pragma unroll 1
        for (int pass = n_pieces < a.k ? 0 : 1; pass < 2; ++pass) {
            uint32_t most = 0;
            if (pass == 1) {
                __syncthreads();
                if (threadIdx.x == 0) s.n = 0;
                __syncthreads();
            }
#pragma unroll 1
            for (int i = 0; i < kMost; ++i) {
                int at_piece = pos[0];
#pragma unroll
                for (int j = 1; j < kMost; ++j) at_piece = i == j ? pos[j] : at_piece;
                if (at_piece < 0) break;         // (the warp's others are none either)
                const int p = at_piece * kPiece + lane * kVec, j0 = p - shift;
                const uint4 v = p >= shift && p + kVec <= end ? *reinterpret_cast<const uint4*>(in - shift + p) : load_edge(in, p, shift, end);
                const uint32_t keep = nothing ? 0u : mask ? mask_bits(mask, j0, kVec, a.V) : ~0u;
                uint32_t special = 0, val[kVec]; // listed or on the path; logit_order, 0: no candidate
                if (par.listed && !w.final) {
                    special = mask_bits(par.listed, j0, kVec, a.V);
                    if (par.path)
                        for (int q = 0; q < a.path_len; ++q) {
                            const int at = par.path[q] - j0;
                            if (at >= 0 && at < kVec) special |= 1u << at;
                        }
                }
                uint32_t in_row = 0;
#pragma unroll
                for (int e = 0; e < kVec; ++e) {
                    if (p + e >= shift && p + e < end) in_row |= 1u << e;
                    const bool use = (keep >> e) & 1u && p + e >= shift && p + e < end;
                    val[e] = use ? logit_order(Elem<T>::up(reinterpret_cast<const T*>(&v)[e])) : 0;
                }
                if (__any_sync(0xffffffffu, special & keep & in_row)) {
                    uint32_t* mine = s.value[warp] + lane * kVec;
#pragma unroll
                    for (int e = 0; e < kVec; ++e) mine[e] = val[e];
                    for (uint32_t left = special & keep & in_row & ((1u << kVec) - 1); left; left &= left - 1) {
                        const int e = __ffs(left) - 1, j = j0 + e;
                        mine[e] = logit_order(adjust(Elem<T>::up(in[j]), j, entry_of(par, w, j), par, a.path_len));
                    }
#pragma unroll
                    for (int e = 0; e < kVec; ++e) val[e] = mine[e];
                    __syncwarp();
                }
                if (pass == 0) {
#pragma unroll
                    for (int e = 0; e < kVec; ++e) most = max(most, val[e]);
                    continue;
                }
                int found = 0;
#pragma unroll
                for (int e = 0; e < kVec; ++e) {
                    if (val[e] < tau) val[e] = 0;
                    found += val[e] != 0;
                }
                const int all = __reduce_add_sync(0xffffffffu, found);
                if (all <= a.k) {
                    if (found)
#pragma unroll
                        for (int e = 0; e < kVec; ++e)
                            if (val[e]) s.buf[atomicAdd(&s.n, 1)] = logit_key(val[e], j0 + e);
                } else                           // values that pile up: the best k of the piece
#pragma unroll 1
                    for (int t = 0; t < a.k; ++t) {
                        unsigned long long best = 0;
#pragma unroll
                        for (int e = 0; e < kVec; ++e) {
                            const unsigned long long key = logit_key(val[e], j0 + e);
                            best = key > best ? key : best;
                        }
                        const uint32_t hi = __reduce_max_sync(0xffffffffu, (uint32_t)(best >> 32));
                        const uint32_t lo = __reduce_max_sync(0xffffffffu, (uint32_t)(best >> 32) == hi ? (uint32_t)best : 0u);
                        best = ((unsigned long long)hi << 32) | lo;
#pragma unroll
                        for (int e = 0; e < kVec; ++e)
                            if (val[e] && logit_key(val[e], j0 + e) == best) {
                                s.buf[atomicAdd(&s.n, 1)] = best;
                                val[e] = 0;
                            }
                    }
            }
            if (pass == 0) tau = max(tau, bound_of(most));
        }
        __syncthreads();
    }

    if (w.late && par.listed) {                  // every reader of the logits is done: the listed tokens and the path's can be stored
        const int2 range = w.range[seq];
        const int total = range.y + (par.path ? a.path_len : 0);
        __syncthreads();
        for (int i = threadIdx.x; i < total; i += WARPS * 32) {
            int token = i < range.y ? __ldcg(w.token + range.x + i) : par.path[i - range.y];
            if (i >= range.y) {                  // a path token that is listed, or an equal one before it, is stored already
                bool first = token >= 0 && token < a.V && !((__ldcg(par.listed + (token >> 5)) >> (token & 31)) & 1u);
                for (int q = 0; q < i - range.y && first; ++q) first = par.path[q] != token;
                if (!first) continue;
            }
            float l = adjust(Elem<T>::up(in[token]), token, entry_of(par, w, token), par, a.path_len);
            if (nothing || (mask && !((mask[token >> 5] >> (token & 31)) & 1u))) l = kNegInf;
            out[token] = Elem<T>::down(l);
        }
    }
    // the row's log-sum-exp, added up in a fixed order, and its candidates
    const float m_w = warp_max(mx), s_w = warp_sum(sum * exp_fast(mx - (m_w == kNegInf ? 0.f : m_w)));
    if (lane == 0) { s.warp_m[warp] = m_w; s.warp_s[warp] = s_w; }
    __syncthreads();
    float m = s.warp_m[0], t = 0.f;
#pragma unroll
    for (int i = 1; i < WARPS; ++i) m = fmaxf(m, s.warp_m[i]);
    const float base = m == kNegInf ? 0.f : m;
#pragma unroll
    for (int i = 0; i < WARPS; ++i) t += s.warp_s[i] * exp_fast(s.warp_m[i] - base);
    const float lse = base + logf(t);
    if (threadIdx.x == 0 && a.out_lse) a.out_lse[row] = lse;
    if (a.k == 0) return;
    const int n = s.n;
    unsigned long long key = 0;
    int at = threadIdx.x;                        // the thread's key and its place
    if (n <= 32) {
        if (warp) return;
        key = lane < n ? s.buf[lane] : 0;
        at = warp_rank(key, n);
        if (lane >= n) at = lane;                // places without a key
    } else {
        rank_keys(n, a.k, s);
        if (at < a.k) key = s.best[at];
    }
    if (at < a.k) {
        a.out_ids[(size_t)row * a.k + at] = key ? (int32_t)(0xffffffffu - (uint32_t)key) : kNoToken;
        a.out_logprobs[(size_t)row * a.k + at] = key ? logit_unorder((uint32_t)(key >> 32)) - lse : kNegInf;
    }
}

}  // namespace coral

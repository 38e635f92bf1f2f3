// Penalties for repeated tokens, biases and grammar masks on dense logits, with the candidates of the result in the same
// pass (the dense counterpart of the draft step's merge; the candidates feed the tree expansion).  Per token x of a row:
//   l1 = x seen ? (l > 0 ? l / rep : l * rep) : l      l2 = l1 - freq * count(x)      l3 = l2 - (count(x) > 0 ? pres : 0)
//   l4 = l3 + bias(x)      out = x allowed ? l4 : -inf            (each step one fp32 operation, in this order)
// Bound by the logits' bytes, so a row is read once.  A cluster of blocks owns a row and deals its 8192-token chunks among
// its blocks.  The row's token lists are short against V but long against a chunk, so the blocks read them together, once,
// and each entry is counted with one shared-memory atomic in the block that owns its token (distributed shared memory):
// whole numbers, so their order does not matter.  The 16 logits a thread holds meanwhile are already on their way.
// Candidates: keys (value, lower id first) above a bound that at least k tokens reach are collected and ranked by counting;
// the bound is the smallest of the warps' largest values at first and the k-th key found so far later on.
#pragma once
#include <cooperative_groups.h>

#include "element.cuh"

namespace coral {

constexpr int kLogitsThreads = 512;
constexpr int kLogitsWarps = kLogitsThreads / 32;
constexpr int kLogitsPer = 16;                               // logits per thread and chunk
constexpr int kLogitsChunk = kLogitsThreads * kLogitsPer;    // 8192
constexpr int kLogitsCap = 1024;                             // candidates ranked by counting
constexpr int kLogitsMaxCluster = 16;

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

struct LogitsShared {
    unsigned long long buf[kLogitsCap];          // [0, n_top): the best keys so far, descending; then new candidates
    unsigned long long warp_key[kLogitsWarps];
    float warp_f[kLogitsWarps], warp_s[kLogitsWarps];
    uint32_t warp_u[kLogitsWarps];
    int n, n_top;
    float row_max, row_sum;
};

// Largest key of the block.  Ends with a barrier, so it may be called again at once.
__device__ __forceinline__ unsigned long long block_max_key(unsigned long long key, LogitsShared& s) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const unsigned long long other = __shfl_xor_sync(0xffffffffu, key, o);
        key = other > key ? other : key;
    }
    if ((threadIdx.x & 31) == 0) s.warp_key[threadIdx.x >> 5] = key;
    __syncthreads();
    unsigned long long best = 0;
#pragma unroll
    for (int w = 0; w < kLogitsWarps; ++w) best = s.warp_key[w] > best ? s.warp_key[w] : best;
    __syncthreads();
    return best;
}

// Ranks the s.n keys of s.buf and leaves the best k of them there in descending order.  Keys are distinct.
__device__ __forceinline__ void rank_candidates(int n, int k, LogitsShared& s) {
    unsigned long long mine[kLogitsCap / kLogitsThreads];
    int rank[kLogitsCap / kLogitsThreads];
#pragma unroll
    for (int i = 0; i < kLogitsCap / kLogitsThreads; ++i) {
        const int at = threadIdx.x + i * kLogitsThreads;
        rank[i] = k;
        if (at >= n) continue;
        mine[i] = s.buf[at];
        int r = 0;
        for (int j = 0; j < n; ++j) r += s.buf[j] > mine[i] ? 1 : 0;
        rank[i] = r;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kLogitsCap / kLogitsThreads; ++i)
        if (rank[i] < k) s.buf[rank[i]] = mine[i];
    if (threadIdx.x == 0) s.n_top = s.n = n < k ? n : k;
    __syncthreads();
}

// Adds a chunk's values to the block's best keys.  order[e]: logit_order of value e, token(e): its id; warps_used: warps that
// hold tokens of this chunk.
template <typename F>
__device__ __forceinline__ void chunk_candidates(const uint32_t (&order)[kLogitsPer], F token, int warps_used, int k, LogitsShared& s) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    unsigned long long floor_key = 0;            // candidates are above this key
    if (s.n_top == k) floor_key = s.buf[k - 1];
    else {
        // every used warp has q values of at least tau, and q * warps_used >= k
        const int q = (k + warps_used - 1) / warps_used;
        uint32_t best = 0, tau = 0;
#pragma unroll
        for (int e = 0; e < kLogitsPer; ++e) best = order[e] > best ? order[e] : best;
        for (int i = 0; i < q; ++i) {
            tau = __reduce_max_sync(0xffffffffu, best);
            const uint32_t who = __ballot_sync(0xffffffffu, best == tau);
            if (lane == __ffs(who) - 1) best = 0;
        }
        if (lane == 0) s.warp_u[warp] = tau;
        __syncthreads();
        tau = 0xffffffffu;
        for (int w = 0; w < warps_used; ++w) tau = s.warp_u[w] < tau ? s.warp_u[w] : tau;
        floor_key = tau ? ((unsigned long long)tau << 32) - 1 : 0;      // equal values are candidates too
    }
    const uint32_t floor_order = (uint32_t)(floor_key >> 32);
#pragma unroll
    for (int e = 0; e < kLogitsPer; ++e) {
        if (order[e] < floor_order || order[e] == 0) continue;
        const unsigned long long key = logit_key(order[e], token(e));
        if (key <= floor_key) continue;
        const int at = atomicAdd(&s.n, 1);
        if (at < kLogitsCap) s.buf[at] = key;
    }
    __syncthreads();
    const int n = s.n;
    __syncthreads();                             // every thread has read it before the next chunk counts on
    if (n <= kLogitsCap) {
        if (n > s.n_top) rank_candidates(n, k, s);
        return;
    }
    // more candidates than the buffer holds (values that pile up at the bound): k rounds over the registers
    const int had = s.n_top;
    unsigned long long old = threadIdx.x < had ? s.buf[threadIdx.x] : 0, last = ~0ull;
    __syncthreads();
    int found = 0;
    for (; found < k; ++found) {
        unsigned long long best = old < last ? old : 0;
#pragma unroll
        for (int e = 0; e < kLogitsPer; ++e) {
            const unsigned long long key = logit_key(order[e], token(e));
            if (key < last && key > best) best = key;
        }
        best = block_max_key(best, s);
        if (best == 0) break;
        if (threadIdx.x == 0) s.buf[found] = best;
        last = best;
    }
    if (threadIdx.x == 0) s.n_top = s.n = found;
    __syncthreads();
}

__device__ __forceinline__ void list_range(const long long* off, int seq, long long total, long long& a, long long& b) {
    a = off[seq];
    b = off[seq + 1];
    a = a < 0 ? 0 : a > total ? total : a;
    b = b < a ? a : b > total ? total : b;
}

// grid: M clusters of C blocks.  dynamic shared memory: kLogitsChunk words if there are token lists (bit 31: seen, below: count),
// kLogitsChunk more if there are biases (1 + place of the last entry of the token).
template <typename T>
__global__ void __launch_bounds__(kLogitsThreads, 2) logits_kernel(LogitsArgs a, int C) {
    namespace cg = cooperative_groups;
    constexpr int kVec = 16 / (int)sizeof(T), kVecs = kLogitsPer / kVec;
    extern __shared__ __align__(16) uint32_t tables[];
    __shared__ LogitsShared s;
    const int row = blockIdx.x / C, rank = blockIdx.x % C;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int seq = a.row_seq ? a.row_seq[row] : row;
    const bool known = seq >= 0 && seq < a.n_seq;            // a row of no sequence has no lists and no penalties
    const bool lists = a.prompt || a.output || a.path, biases = a.bias_tokens != nullptr;
    uint32_t* counts = tables;
    uint32_t* bias_at = tables + (lists ? kLogitsChunk : 0);

    const T* in = reinterpret_cast<const T*>(a.logits) + (size_t)row * a.ld_in;
    T* out = a.out ? reinterpret_cast<T*>(a.out) + (size_t)row * a.ld_out : nullptr;
    // positions p = token + shift start on 16 bytes: a vector of the row is loaded whole unless it holds an end of the row
    const int shift = (int)((reinterpret_cast<uintptr_t>(in) & 15) / sizeof(T));
    const bool vec_out = out && (int)((reinterpret_cast<uintptr_t>(out) & 15) / sizeof(T)) == shift;
    const int end = a.V + shift;
    const int chunks = (end - 1) / kLogitsChunk + 1, passes = (chunks + C - 1) / C;

    const float rep = known && a.rep ? a.rep[seq] : 1.f, freq = known && a.freq ? a.freq[seq] : 0.f,
                pres = known && a.pres ? a.pres[seq] : 0.f;
    const uint32_t* mask = nullptr;
    bool nothing = false;
    if (a.mask) {
        const int mr = a.mask_rows ? a.mask_rows[row] : row;
        if (mr >= a.n_masks) nothing = true;                 // no such mask: allow nothing
        else if (mr >= 0) mask = a.mask + (size_t)mr * a.mask_words;
    }
    if (threadIdx.x == 0) { s.n = 0; s.n_top = 0; }

    float mx = kNegInf, sum = 0.f;
    for (int pass = 0; pass < passes; ++pass) {
        const int chunk = pass * C + rank;
        const int p0 = chunk * kLogitsChunk;                 // may lie past the end: then this block only helps
        uint4 raw[kVecs];
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            const int p = p0 + (threadIdx.x + i * kLogitsThreads) * kVec;
            if (p >= shift && p + kVec <= end) raw[i] = __ldcs(reinterpret_cast<const uint4*>(in - shift + p));
            else {
                T* r = reinterpret_cast<T*>(&raw[i]);
#pragma unroll
                for (int e = 0; e < kVec; ++e) r[e] = p + e >= shift && p + e < end ? in[p + e - shift] : Elem<T>::down(0.f);
            }
        }
        if (lists || biases) {
            const int words = (lists ? kLogitsChunk : 0) + (biases ? kLogitsChunk : 0);
            for (int i = threadIdx.x * 4; i < words; i += kLogitsThreads * 4)
                *reinterpret_cast<uint4*>(tables + i) = make_uint4(0, 0, 0, 0);
            auto cluster = cg::this_cluster();
            if (C > 1) cluster.sync();
            else __syncthreads();
            // the table word of a token of this pass, in the block that owns it
            auto word = [&](uint32_t* table, int token) -> uint32_t* {
                if (token < 0 || token >= a.V) return nullptr;
                const int p = token + shift, c = p / kLogitsChunk;
                if (c / C != pass) return nullptr;
                uint32_t* at = table + p % kLogitsChunk;
                return C > 1 ? cluster.map_shared_rank(at, c % C) : at;
            };
            const int first = rank * kLogitsThreads + threadIdx.x, step = C * kLogitsThreads;
            long long lo, hi;
            if (a.prompt && known) {
                list_range(a.prompt_off, seq, a.prompt_total, lo, hi);
                for (long long i = lo + first; i < hi; i += step)
                    if (uint32_t* w = word(counts, a.prompt[i])) atomicOr(w, 0x80000000u);
            }
            if (a.output && known) {
                list_range(a.output_off, seq, a.output_total, lo, hi);
                for (long long i = lo + first; i < hi; i += step)
                    if (uint32_t* w = word(counts, a.output[i])) atomicAdd(w, 1u);
            }
            if (a.path)
                for (int i = first; i < a.path_len; i += step)
                    if (uint32_t* w = word(counts, a.path[(size_t)row * a.path_len + i])) atomicAdd(w, 1u);
            if (biases && known) {
                list_range(a.bias_off, seq, a.bias_total, lo, hi);
                for (long long i = lo + first; i < hi; i += step)
                    if (uint32_t* w = word(bias_at, a.bias_tokens[i])) atomicMax(w, (uint32_t)(i - lo) + 1u);
            }
            if (C > 1) cluster.sync();
            else __syncthreads();
        } else if (pass == 0) __syncthreads();               // s.n is set
        if (p0 >= end) continue;

        uint32_t order[kLogitsPer];
        float val[kLogitsPer];
        float top = kNegInf;
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            const int at = (threadIdx.x + i * kLogitsThreads) * kVec, p = p0 + at, j0 = p - shift;
            const T* r = reinterpret_cast<const T*>(&raw[i]);
            float f[kVec];
#pragma unroll
            for (int e = 0; e < kVec; ++e) f[e] = Elem<T>::up(r[e]);
            if (lists) {
#pragma unroll
                for (int e = 0; e < kVec; e += 4) {
                    const uint4 w4 = *reinterpret_cast<const uint4*>(counts + at + e);
                    if ((w4.x | w4.y | w4.z | w4.w) == 0) continue;
                    const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
                    for (int o = 0; o < 4; ++o) {
                        if (w[o] == 0) continue;
                        float l = f[e + o];
                        l = l > 0.f ? __fdiv_rn(l, rep) : __fmul_rn(l, rep);
                        const uint32_t n = w[o] & 0x7fffffffu;
                        if (n) l = __fsub_rn(__fsub_rn(l, __fmul_rn(freq, (float)n)), pres);
                        f[e + o] = l;
                    }
                }
            }
            if (biases) {
                long long lo, hi;
#pragma unroll
                for (int e = 0; e < kVec; e += 4) {
                    const uint4 w4 = *reinterpret_cast<const uint4*>(bias_at + at + e);
                    if ((w4.x | w4.y | w4.z | w4.w) == 0) continue;
                    list_range(a.bias_off, seq, a.bias_total, lo, hi);
                    const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
                    for (int o = 0; o < 4; ++o)
                        if (w[o]) f[e + o] = __fadd_rn(f[e + o], a.bias_values[lo + w[o] - 1]);
                }
            }
            if (mask && p < end) {
                const int a0 = j0 < 0 ? 0 : j0, a1 = j0 + kVec - 1 < a.V ? j0 + kVec - 1 : a.V - 1;
                const uint32_t w0 = __ldg(mask + (a0 >> 5)), w1 = __ldg(mask + (a1 >> 5));
#pragma unroll
                for (int e = 0; e < kVec; ++e) {
                    const int j = j0 + e;
                    const uint32_t w = (j >> 5) == (a0 >> 5) ? w0 : w1;
                    if (!((w >> (j & 31)) & 1u)) f[e] = kNegInf;
                }
            }
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                if (nothing) f[e] = kNegInf;
                const bool in_row = p + e >= shift && p + e < end;
                val[i * kVec + e] = in_row ? f[e] : kNegInf;
                top = fmaxf(top, val[i * kVec + e]);
            }
            if (out) {
                if (vec_out && p >= shift && p + kVec <= end) {
                    uint4 o;
                    T* t = reinterpret_cast<T*>(&o);
#pragma unroll
                    for (int e = 0; e < kVec; ++e) t[e] = Elem<T>::down(f[e]);
                    __stcs(reinterpret_cast<uint4*>(out - shift + p), o);
                } else {
#pragma unroll
                    for (int e = 0; e < kVec; ++e)
                        if (p + e >= shift && p + e < end) out[j0 + e] = Elem<T>::down(f[e]);
                }
            }
        }
        // running maximum and sum of exponentials of this thread's logits
        const float m_new = fmaxf(mx, top);
        const float base = m_new == kNegInf ? 0.f : m_new;
        sum *= expf(mx - base);
#pragma unroll
        for (int e = 0; e < kLogitsPer; ++e) sum += expf(val[e] - base);
        mx = m_new;
        if (a.k) {
#pragma unroll
            for (int e = 0; e < kLogitsPer; ++e) order[e] = logit_order(val[e]);
            const int first = p0 < shift ? shift : p0, last = p0 + kLogitsChunk < end ? p0 + kLogitsChunk : end;
            const int vecs = (last - 1 - p0) / kVec - (first - p0) / kVec + 1;
            chunk_candidates(order, [&](int e) { return p0 + (threadIdx.x + (e / kVec) * kLogitsThreads) * kVec + e % kVec - shift; },
                             vecs >= kLogitsThreads ? kLogitsWarps : (vecs + 31) / 32, a.k, s);
        }
    }

    // the block's maximum and sum, in a fixed order
    float m_w = warp_max(mx);
    const float b_w = m_w == kNegInf ? 0.f : m_w;
    float s_w = warp_sum(sum * expf(mx - b_w));
    if (lane == 0) { s.warp_f[warp] = m_w; s.warp_s[warp] = s_w; }
    __syncthreads();
    if (threadIdx.x == 0) {
        float m = kNegInf, t = 0.f;
        for (int w = 0; w < kLogitsWarps; ++w) m = fmaxf(m, s.warp_f[w]);
        const float b = m == kNegInf ? 0.f : m;
        for (int w = 0; w < kLogitsWarps; ++w) t += s.warp_s[w] * expf(s.warp_f[w] - b);
        s.row_max = m;
        s.row_sum = t;
    }
    __syncthreads();
    if (C > 1) {
        auto cluster = cg::this_cluster();
        cluster.sync();
        if (rank == 0) {
            if (threadIdx.x == 0) {
                float m = kNegInf, t = 0.f;
                for (int c = 0; c < C; ++c) m = fmaxf(m, cluster.map_shared_rank(&s, c)->row_max);
                const float b = m == kNegInf ? 0.f : m;
                for (int c = 0; c < C; ++c) {
                    const LogitsShared* o = cluster.map_shared_rank(&s, c);
                    t += o->row_sum * expf(o->row_max - b);
                }
                s.warp_f[0] = m;
                s.warp_s[0] = t;
            }
            if (a.k) {
                const int had = s.n_top;
                __syncthreads();
                const int c = 1 + threadIdx.x / a.k, i = threadIdx.x % a.k;
                if (c < C) {
                    const LogitsShared* o = cluster.map_shared_rank(&s, c);
                    if (i < o->n_top) {
                        const int at = atomicAdd(&s.n, 1);
                        s.buf[at] = o->buf[i];
                    }
                }
                __syncthreads();
                const int n = s.n;
                if (n > had) rank_candidates(n, a.k, s);
            }
            __syncthreads();
            if (threadIdx.x == 0) { s.row_max = s.warp_f[0]; s.row_sum = s.warp_s[0]; }
        }
        cluster.sync();                                      // the other blocks' shared memory has been read
        if (rank != 0) return;
    }
    const float base = s.row_max == kNegInf ? 0.f : s.row_max;
    const float lse = base + logf(s.row_sum);
    if (threadIdx.x == 0 && a.out_lse) a.out_lse[row] = lse;
    if (threadIdx.x < a.k) {
        const unsigned long long key = threadIdx.x < s.n_top ? s.buf[threadIdx.x] : 0;
        a.out_ids[(size_t)row * a.k + threadIdx.x] = key ? (int32_t)(0xffffffffu - (uint32_t)key) : kNoToken;
        a.out_logprobs[(size_t)row * a.k + threadIdx.x] = key ? logit_unorder((uint32_t)(key >> 32)) - lse : kNegInf;
    }
}

}  // namespace coral

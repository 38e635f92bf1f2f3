// C ABI of the operators around the draft step: argument checks and kernel launches.  See include/coral_lmhead.h.
#include "coral_lmhead.h"

#include <cuda_runtime.h>

#include <algorithm>

#include "block_norm.cuh"
#include "launch.cuh"
#include "logits.cuh"
#include "q4.cuh"
#include "q4_tc.cuh"

using namespace coral;

namespace {

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline int elem_size(int type) { return type == CORAL_TYPE_F32 ? 4 : 2; }

bool device_sms(int* sms) {
    int dev = 0;
    return cudaGetDevice(&dev) == cudaSuccess && cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess;
}

// The attribute is per kernel and device; above 48 KB, static shared memory (at most 16 KB in kernels that have both) counted in, it has
// to be raised before the launch.
template <typename K>
bool allow_smem(K kernel, size_t bytes) {
    return bytes <= 32 * 1024 ||
           cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == cudaSuccess;
}

// ---- block norm ----------------------------------------------------------------------------------------------
constexpr int kNormFwdThreadsPerSm = 1024, kNormBwdThreadsPerSm = 512;
constexpr int kNormSmallBlock = 256;             // threads of a block while a row fits two chunks a thread
constexpr size_t kNormSmemPerSm = 200 * 1024;
constexpr int kNormMaxBlocksPerSm = 16;
constexpr int kNormSmCap = 160;                 // most SMs the partial rows of the workspace are sized for

struct NormPlan {
    int nv, threads, grid, stages;
    size_t smem;
};

// nv: 8-column chunks a thread keeps.  Blocks of up to 256 threads, several a SM, so that one block's row sums wait while
// another's row is worked on (16384 x 4096 forward: 109 us, 133 with one chunk a thread and 512 threads).  Threads are the
// chunks over nv rounded up to a warp: a row of 3584 columns runs 224 threads and wastes none.
void norm_block(int H, int* nv, int* threads) {
    static_assert(kNormMaxRowBytes / 2 / 8 <= 4 * kNormMaxThreads, "rows of 16 bits fit four chunks a thread");
    const int chunks = H / 8;
    *nv = chunks <= kNormSmallBlock ? 1 : chunks <= 2 * kNormMaxThreads ? 2 : 4;
    *threads = ((chunks + *nv - 1) / *nv + 31) / 32 * 32;
}

int norm_blocks_per_sm(int threads, int threads_per_sm) {
    const int blocks = threads_per_sm / threads;
    return blocks < 1 ? 1 : blocks > kNormMaxBlocksPerSm ? kNormMaxBlocksPerSm : blocks;
}

NormPlan norm_plan(int M, int H, int type, int tensors, int threads_per_sm, int sms) {
    NormPlan p{};
    norm_block(H, &p.nv, &p.threads);
    int blocks = norm_blocks_per_sm(p.threads, threads_per_sm);
    const size_t stage = (size_t)tensors * p.nv * p.threads * 8 * elem_size(type);
    size_t stages = kNormSmemPerSm / blocks / stage;
    if (stages < 1) {                            // very wide fp32 rows: one block a SM
        blocks = 1;
        stages = 1;
    }
    p.stages = stages > 4 ? 4 : (int)stages;
    if (sms > kNormSmCap) sms = kNormSmCap;
    const int most = sms * blocks, turns = (M - 1) / most + 1;
    p.grid = (M - 1) / turns + 1;                // no more blocks than the busiest one's rows ask for
    p.smem = stage * p.stages;
    return p;
}

// Most partial rows a backward call can write.
int norm_max_grid(int H) {
    int nv, threads;
    norm_block(H, &nv, &threads);
    return norm_blocks_per_sm(threads, kNormBwdThreadsPerSm) * kNormSmCap;
}

bool norm_args_ok(const coral_lmhead_norm_args* a) {
    if (!a || a->struct_size != sizeof(*a)) return false;
    if (a->type != CORAL_TYPE_F32 && a->type != CORAL_TYPE_BF16 && a->type != CORAL_TYPE_F16) return false;
    if (a->M < 1 || a->H < 8 || a->H % 8 != 0 || (long long)a->H * elem_size(a->type) > kNormMaxRowBytes) return false;
    if (a->gate_mode < CORAL_GATE_NONE || a->gate_mode > CORAL_GATE_FULL) return false;
    if ((a->gate_mode == CORAL_GATE_NONE) != (a->gate_dev == nullptr)) return false;
    if (!(a->eps >= 0.f) || !a->x_dev) return false;
    if (!aligned(a->x_dev, 16) || !aligned(a->r_dev, 16) || !aligned(a->w_post_dev, 16) || !aligned(a->w_pre_dev, 16) ||
        !aligned(a->gate_dev, a->gate_mode == CORAL_GATE_ROW ? elem_size(a->type) : 16))
        return false;
    return true;
}

NormArgs norm_kernel_args(const coral_lmhead_norm_args* a) {
    NormArgs k{};
    k.M = a->M; k.H = a->H; k.gate_mode = a->gate_mode;
    k.alpha = a->alpha; k.eps = a->eps;
    k.x = a->x_dev; k.r = a->r_dev; k.gate = a->gate_dev; k.w_post = a->w_post_dev; k.w_pre = a->w_pre_dev;
    return k;
}

template <typename T, int NV>
int launch_norm(const NormArgs& k, const NormPlan& p, bool backward, cudaStream_t st) {
    if (backward) {
        if (!allow_smem(block_norm_backward_kernel<T, NV>, p.smem)) return CORAL_ERR_CUDA;
        block_norm_backward_kernel<T, NV><<<p.grid, p.threads, p.smem, st>>>(k, p.stages);
    } else {
        if (!allow_smem(block_norm_kernel<T, NV>, p.smem)) return CORAL_ERR_CUDA;
        block_norm_kernel<T, NV><<<p.grid, p.threads, p.smem, st>>>(k, p.stages);
    }
    return cudaGetLastError() == cudaSuccess ? CORAL_OK : CORAL_ERR_CUDA;
}

template <typename T>
int launch_norm_nv(const NormArgs& k, const NormPlan& p, bool backward, cudaStream_t st) {
    if (p.nv == 1) return launch_norm<T, 1>(k, p, backward, st);
    if constexpr (sizeof(T) == 4) {
        static_assert(kNormMaxRowBytes / 4 / 8 <= 2 * kNormMaxThreads, "fp32 rows never want four chunks a thread");
        return launch_norm<T, 2>(k, p, backward, st);
    } else return p.nv == 2 ? launch_norm<T, 2>(k, p, backward, st) : launch_norm<T, 4>(k, p, backward, st);
}

int launch_norm_type(int type, const NormArgs& k, const NormPlan& p, bool backward, cudaStream_t st) {
    if (type == CORAL_TYPE_BF16) return launch_norm_nv<__nv_bfloat16>(k, p, backward, st);
    if (type == CORAL_TYPE_F16) return launch_norm_nv<__half>(k, p, backward, st);
    return launch_norm_nv<float>(k, p, backward, st);
}

// ---- products with 4-bit weights -----------------------------------------------------------------------------
constexpr int kQ4MaxK = 65536;
constexpr size_t kQ4MaxSmem = 227 * 1024;

bool q4_config_ok(const coral_lmhead_q4_config* c) {
    if (!c || c->struct_size != sizeof(*c)) return false;
    if (c->group != 32 && c->group != 64 && c->group != 128) return false;
    if (c->N < 1 || c->K < c->group || c->K > kQ4MaxK || c->K % c->group != 0) return false;
    if (c->scale_type != CORAL_TYPE_BF16 && c->scale_type != CORAL_TYPE_F16) return false;
    return c->has_zeros == 0 || c->has_zeros == 1;
}

struct Q4Layout {
    int KB, T;
    size_t weights, scales;                      // bytes of the two parts; the scales follow the weights
};

Q4Layout q4_layout(const coral_lmhead_q4_config& c) {
    Q4Layout L;
    L.KB = (c.K + 127) / 128;
    L.T = (c.N - 1) / 16 + 1;
    const size_t blocks = (size_t)L.T * L.KB;
    L.weights = blocks * 1024;
    L.scales = blocks * 16 * (128 / c.group) * (c.has_zeros ? 4 : 2);
    return L;
}

// How many warps share a tile's columns: the split whose busiest warp has the least to do, joining the parts of a tile counted
// as three fifths of a column block (128256 x 4096, one row: 63 us with 2 warps, 76 with 16).
int q4_split(int T, int KB, int sms) {
    int best = 1;
    long long best_cost = -1;
    for (int s = 1; s <= kQ4Warps; s *= 2) {
        const long long teams = (long long)sms * (kQ4Warps / s);
        const long long cost = ((T + teams - 1) / teams) * (5 * ((KB + s - 1) / s) + 3);
        if (best_cost < 0 || cost < best_cost) { best = s; best_cost = cost; }
    }
    return best;
}

// Passes of 256 output rows on the tensor cores: every SM takes as many as all can, and those left over are split by columns, so
// that they do not cost a whole pass (152064 x 3584 has 594 of them for 148 SMs: 157 -> 138 us with 60 rows and groups of 128, 218 -> 185 with
// groups of 64; 4096 x 4096 has 16: 40 -> 19.5).  A part has 256 columns at least.
Q4Share q4_share(int T, int KB, int sms) {
    const int passes = (T - 1) / kQ4TcTiles + 1;
    Q4Share s{};
    s.full = passes / sms;
    s.tail = passes % sms;
    s.split = s.tail ? std::max(1, std::min({sms / s.tail, kQ4TcMaxSplit, KB / 2})) : 1;
    return s;
}
// ... and the most memory their parts take, whatever the number of SMs.
size_t q4_part_bytes(int T, int KB, int slab_rows) {
    const long long passes = (T - 1) / kQ4TcTiles + 1;
    const long long parts = std::min<long long>(kQ4TcMaxParts, passes * std::max(1, std::min(kQ4TcMaxSplit, KB / 2)));
    return (size_t)parts * slab_rows * 256 * sizeof(float);
}

// The passes over the rows of a call: up to 64 rows each on the tensor cores while more than 16 are left (152064 x 3584, groups of
// 64: 158 us at 17 rows and 185 at 64; the warps' MMA takes 103 for every 16), then up to 16 on the warps' MMA, fewer where
// long rows do not fit shared memory: 15 at K = 6144, 7 at 14336.  (The rule does not look at K, so that 8 to 16 long rows take
// several passes where 17 take one: 4096 x 14336, groups of 128, 8 rows 41 us, 16 rows 62, 17 rows 26.)  Rows that a block would spend long on scaling are laid out first, in the caller's workspace.
constexpr int kQ4StageUnits = 1024;              // 8-column pieces that a block of the product scales itself

struct Q4Pass {
    int first, rows, slab_rows;                  // slab_rows: 32 or 64 on the tensor cores, else 0
    bool staged;
    size_t at, back_bytes, sum_bytes, bytes;     // its part of the workspace
};

int q4_row_limit(int KB, int per) {
    const size_t row = (size_t)KB * 256 + 64, red = (size_t)2 * kQ4Warps * 16 * 8 * sizeof(float);
    auto fit = [&](int nt) {
        const size_t fixed = nt * red + (size_t)KB * per * 8 * nt * sizeof(float) + 1024;
        const size_t n = fixed < kQ4MaxSmem ? (kQ4MaxSmem - fixed) / row : 0;
        return n < (size_t)8 * nt ? (int)n : 8 * nt;
    };
    const int one = fit(1), two = fit(2);
    return two > one ? two : one;
}

// Pass `i` of a call, in order; false behind the last.  `at` is where the workspace part of the next pass starts.
bool q4_next_pass(const coral_lmhead_q4_config& c, int KB, int M, int* first, size_t* at, Q4Pass* p) {
    const int left = M - *first, per = 128 / c.group;
    if (left < 1) return false;
    *p = Q4Pass{};
    p->first = *first;
    auto up = [](size_t b) { return (b + 255) / 256 * 256; };
    if (left > kQ4PassRows) {
        p->rows = left < kQ4TcMaxRows ? left : kQ4TcMaxRows;
        p->slab_rows = p->rows <= 32 ? 32 : 64;
        p->staged = true;
        p->back_bytes = up(p->slab_rows * 4);
        p->bytes = p->back_bytes + up((size_t)((c.K + 63) / 64) * p->slab_rows * 128);
    } else {
        const int limit = q4_row_limit(KB, per);
        p->rows = left < limit ? left : limit;
        p->staged = p->rows * KB * 16 > kQ4StageUnits;
        if (p->staged) {
            p->back_bytes = up(p->rows * 4);
            p->sum_bytes = up((size_t)p->rows * KB * per * 4);
            p->bytes = p->back_bytes + p->sum_bytes + up((size_t)p->rows * KB * 256);
        }
    }
    // the status word comes first, then the parts of the widest tensor-core pass, the first one
    if (p->bytes && *at == 0) *at = 256 + (p->slab_rows ? q4_part_bytes((c.N - 1) / 16 + 1, KB, p->slab_rows) : 0);
    p->at = *at;
    *at += p->bytes;
    *first += p->rows;
    return true;
}

template <typename TX, int PER, bool ZEROS>
int launch_q4_pass(const Q4View& q, const Q4Pass& p, const void* x_all, void* out_all, int out_type, unsigned char* ws, bool first,
                   int sms, cudaStream_t st) {
    const TX* x = static_cast<const TX*>(x_all) + (size_t)p.first * q.K;
    void* out = static_cast<unsigned char*>(out_all) + (size_t)p.first * q.N * elem_size(out_type);
    Q4Staged s{};
    if (p.staged) {
        s.status = first ? reinterpret_cast<int*>(ws) : nullptr;
        s.back = reinterpret_cast<int*>(ws + p.at);
        s.sums = reinterpret_cast<float*>(ws + p.at + p.back_bytes);
        s.x = reinterpret_cast<uint4*>(ws + p.at + p.back_bytes + p.sum_bytes);
        q4_stage_kernel<TX, PER><<<p.slab_rows ? p.slab_rows : p.rows, 256, 0, st>>>(x, p.rows, q.K, q.KB, p.slab_rows, s);
        if (cudaGetLastError() != cudaSuccess) return CORAL_ERR_CUDA;
    }
    if (p.slab_rows) {
        Q4Share share = q4_share(q.T, q.KB, sms);
        share.part = reinterpret_cast<float*>(ws + 256);
        const int grid = share.full ? sms : share.tail * share.split;
        DeviceState* state = reinterpret_cast<DeviceState*>(ws);
        auto run = [&](auto kernel, size_t smem) {
            return allow_smem(kernel, smem) && launch_pdl(kernel, dim3(grid), dim3(kQ4TcThreads), smem, st, q, s, share, p.rows, out,
                                                          out_type, state) == cudaSuccess;
        };
        const bool ok = p.slab_rows == 32 ? run(q4_tc_kernel<32, PER, ZEROS>, q4_tc_smem_bytes<32>())
                                          : run(q4_tc_kernel<64, PER, ZEROS>, q4_tc_smem_bytes<64>());
        if (!ok) return CORAL_ERR_CUDA;
        if (share.split > 1 && launch_pdl(q4_join_kernel, dim3(share.tail, p.rows), dim3(256), 0, st, share, (const int*)s.back, share.full * sms * 256, p.slab_rows,
                                          q.N, out, out_type) != cudaSuccess)
            return CORAL_ERR_CUDA;
        return CORAL_OK;
    }
    const int split = q4_split(q.T, q.KB, sms);
    const long long units = (long long)q.T * split;              // warps that have a tile to work on
    int warps = kQ4Warps;
    while (warps > split && warps > 4 && units < (long long)sms * warps) warps /= 2;
    const long long teams = warps / split, blocks = (q.T + teams - 1) / teams;
    const int nt = p.rows <= 8 ? 1 : 2;
    const size_t smem = (size_t)p.rows * (q.KB * 256 + 64) + (size_t)q.KB * PER * 8 * nt * sizeof(float) +
                        (size_t)2 * warps * 16 * 8 * nt * sizeof(float);
    auto run = [&](auto kernel) {
        return allow_smem(kernel, smem) && launch_pdl(kernel, dim3((unsigned)(blocks < sms ? blocks : sms)), dim3(warps * 32), smem, st, q, x,
                                                      s, p.rows, out, out_type, split) == cudaSuccess;
    };
    return (nt == 1 ? run(q4_rows_kernel<TX, 1, PER, ZEROS>) : run(q4_rows_kernel<TX, 2, PER, ZEROS>)) ? CORAL_OK : CORAL_ERR_CUDA;
}

template <typename TX, int PER>
int launch_q4_zeros(const coral_lmhead_q4_config& c, const Q4View& q, const Q4Pass& p, const void* x, void* out, int out_type,
                    unsigned char* ws, bool first, int sms, cudaStream_t st) {
    return c.has_zeros ? launch_q4_pass<TX, PER, true>(q, p, x, out, out_type, ws, first, sms, st)
                       : launch_q4_pass<TX, PER, false>(q, p, x, out, out_type, ws, first, sms, st);
}

template <typename TX>
int launch_q4(const coral_lmhead_q4_config& c, const Q4View& q, const Q4Pass& p, const void* x, void* out, int out_type,
              unsigned char* ws, bool first, int sms, cudaStream_t st) {
    if (c.group == 128) return launch_q4_zeros<TX, 1>(c, q, p, x, out, out_type, ws, first, sms, st);
    if (c.group == 64) return launch_q4_zeros<TX, 2>(c, q, p, x, out, out_type, ws, first, sms, st);
    return launch_q4_zeros<TX, 4>(c, q, p, x, out, out_type, ws, first, sms, st);
}

// ---- logits ----------------------------------------------------------------------------------------------------
constexpr int kLogitsMaxV = 1 << 30;
static_assert(CORAL_MAX_PATH <= kLogitsThreads, "logits_wide_kernel has a thread a token of a path");
constexpr int kLogitsMaxChunk = 8;
constexpr int kLogitsEndBlocks = 4 * 148;        // blocks of 16 warps that are resident at once
constexpr int kLogitsWideBlocks = 4 * 148;       // resident at once
constexpr int kLogitsWideFrom = 8 * 8 * 148;     // pieces of a call (8 blocks a SM of the kernel for few rows)

bool logits_args_ok(const coral_lmhead_logits_args* a) {
    if (!a || a->struct_size != sizeof(*a)) return false;
    if (a->type != CORAL_TYPE_F32 && a->type != CORAL_TYPE_BF16 && a->type != CORAL_TYPE_F16) return false;
    if (!a->logits_dev || a->M < 1 || a->V < 1 || a->V > kLogitsMaxV || a->n_seq < 0) return false;
    if (a->ld_logits < a->V || (a->out_logits_dev && a->ld_out < a->V)) return false;
    if (a->out_logits_dev == a->logits_dev && a->ld_out != a->ld_logits) return false;
    if (!a->row_seq_dev && a->n_seq != 0 && a->n_seq < a->M) return false;     // row m is sequence m
    if (a->k_tokens < 0 || a->k_tokens > CORAL_MAX_K_TOKENS || a->k_tokens > a->V) return false;
    if (a->k_tokens > 0 ? !a->out_ids_dev || !a->out_logprobs_dev : a->out_ids_dev || a->out_logprobs_dev) return false;
    if (!a->out_logits_dev && !a->out_lse_dev && a->k_tokens == 0) return false;
    if ((a->prompt_tokens_dev != nullptr) != (a->prompt_offsets_dev != nullptr) || a->prompt_total < 0 || a->prompt_total > 0x7fffffff) return false;
    if ((a->output_tokens_dev != nullptr) != (a->output_offsets_dev != nullptr) || a->output_total < 0 || a->output_total > 0x7fffffff) return false;
    if ((a->bias_tokens_dev != nullptr) != (a->bias_offsets_dev != nullptr) ||
        (a->bias_tokens_dev != nullptr) != (a->bias_values_dev != nullptr) || a->bias_total < 0 || a->bias_total > 0x7fffffff)
        return false;
    if (a->path_len < 0 || a->path_len > CORAL_MAX_PATH || (a->path_tokens_dev != nullptr) != (a->path_len > 0)) return false;
    if (a->mask_words_dev ? a->n_masks < 1 : a->mask_rows_dev != nullptr) return false;
    if (a->mask_words_dev && !a->mask_rows_dev && a->n_masks < a->M) return false;
    const size_t e = elem_size(a->type);
    if (!aligned(a->logits_dev, e) || !aligned(a->out_logits_dev, e)) return false;
    for (const void* p : {(const void*)a->row_seq_dev, (const void*)a->prompt_tokens_dev, (const void*)a->output_tokens_dev,
                          (const void*)a->path_tokens_dev, (const void*)a->bias_tokens_dev, (const void*)a->bias_values_dev,
                          (const void*)a->repetition_dev, (const void*)a->frequency_dev, (const void*)a->presence_dev,
                          (const void*)a->mask_words_dev, (const void*)a->mask_rows_dev, (const void*)a->out_ids_dev,
                          (const void*)a->out_logprobs_dev, (const void*)a->out_lse_dev})
        if (!aligned(p, 4)) return false;
    return aligned(a->prompt_offsets_dev, 8) && aligned(a->output_offsets_dev, 8) && aligned(a->bias_offsets_dev, 8);
}

// What the call needs of its lists: without a penalty the token lists change nothing, without a sequence nothing has any.
LogitsArgs logits_kernel_args(const coral_lmhead_logits_args* a) {
    LogitsArgs k{};
    k.logits = a->logits_dev; k.out = a->out_logits_dev;
    k.ld_in = a->ld_logits; k.ld_out = a->ld_out;
    k.M = a->M; k.V = a->V; k.n_seq = a->n_seq; k.path_len = a->path_len; k.n_masks = a->n_masks;
    k.mask_words = (a->V + 31) / 32; k.k = a->k_tokens;
    k.row_seq = a->row_seq_dev;
    if (a->n_seq > 0 && (a->repetition_dev || a->frequency_dev || a->presence_dev)) {
        k.prompt = a->prompt_tokens_dev; k.prompt_off = reinterpret_cast<const long long*>(a->prompt_offsets_dev);
        k.output = a->output_tokens_dev; k.output_off = reinterpret_cast<const long long*>(a->output_offsets_dev);
        k.path = a->path_tokens_dev;
        k.rep = a->repetition_dev; k.freq = a->frequency_dev; k.pres = a->presence_dev;
    }
    if (k.prompt) k.prompt_total = a->prompt_total;
    if (k.output) k.output_total = a->output_total;
    if (a->n_seq > 0 && a->bias_tokens_dev) {
        k.bias_tokens = a->bias_tokens_dev; k.bias_off = reinterpret_cast<const long long*>(a->bias_offsets_dev);
        k.bias_values = a->bias_values_dev;
        k.bias_total = a->bias_total;
    }
    k.mask = a->mask_words_dev; k.mask_rows = a->mask_rows_dev;
    k.out_ids = a->out_ids_dev; k.out_logprobs = a->out_logprobs_dev; k.out_lse = a->out_lse_dev;
    return k;
}

struct LogitsPlan {
    bool lists;
    int chunk, pieces, parts, blocks;            // spans a block takes (0: few rows); pieces of 512 bytes, parts and blocks of a row
    size_t before, entry, token, range, piece, part, bytes;         // offsets in the workspace; the bitmap comes first
};

// Spans a block takes: as many as make the least of rounds of resident blocks times (spans + what starting a block costs):
// 512 rows of 32000 in fp32 71 us with 8 at most that leave no SM without a block, 62 so; 60 rows of 152064 50 and 48.  More than
// 8 gain nothing (960 rows of 128256: 213 and 213).
int logits_chunk(int M, int spans) {
    int best = 1;
    long long best_cost = -1;
    for (int c = 1; c <= kLogitsMaxChunk; ++c) {
        const long long blocks = (long long)M * ((spans - 1) / c + 1);
        const long long cost = ((blocks - 1) / kLogitsWideBlocks + 1) * (2 * c + 3);
        if (best_cost < 0 || cost < best_cost) { best = c; best_cost = cost; }
    }
    return best;
}

// Rows of 128256 with lists, path, mask, result and candidates, fp32 / bf16: 1 row 30 / 36 us with the kernel for few rows,
// 32 / 40 with the other; 12 rows 36 / 36 and 34 / 36; 60 rows 60 / 52 and 48 / 50; 120 rows 85 / 69 and 60 / 62.
LogitsPlan logits_plan(const LogitsArgs& k, int type) {
    LogitsPlan p{};
    p.lists = k.prompt || k.output || k.path || k.bias_tokens;
    const int vec = 16 / elem_size(type), span = 32 * vec;
    p.pieces = (int)((k.V + vec - 2LL) / span) + 1;                        // of a row that starts as late as it can
    const int spans = (p.pieces - 1) / (kWideSpan / span) + 1;
    if ((long long)k.M * p.pieces >= kLogitsWideFrom) p.chunk = logits_chunk(k.M, spans);
    p.blocks = p.chunk ? (spans - 1) / p.chunk + 1 : (p.pieces - 1) / kLogitsWarps + 1;
    p.parts = p.blocks * kLogitsWarps;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t from = at; at = (at + bytes + 255) / 256 * 256; return from; };
    if (p.lists) {
        take((size_t)k.n_seq * k.mask_words * 4);
        p.before = take((size_t)k.n_seq * k.mask_words * 4);
        const size_t listed = (size_t)(k.prompt_total + k.output_total + k.bias_total);
        p.entry = take(listed * 8);
        p.token = take(listed * 4);
        p.range = take((size_t)k.n_seq * 8);
    }
    p.piece = take((size_t)k.M * p.pieces * 4);
    p.part = take((size_t)k.M * p.parts * 8);
    p.bytes = at;
    return p;
}

template <typename T>
int launch_logits(const LogitsArgs& k, const LogitsPlan& p, unsigned char* ws, cudaStream_t st) {
    LogitsWork w{};
    w.piece = reinterpret_cast<uint32_t*>(ws + p.piece);
    w.part = reinterpret_cast<float2*>(ws + p.part);
    w.pieces = p.pieces;
    w.parts = p.parts;
    if (p.lists) {
        w.bitmap = reinterpret_cast<uint32_t*>(ws);
        w.before = reinterpret_cast<uint32_t*>(ws + p.before);
        w.entry = reinterpret_cast<uint2*>(ws + p.entry);
        w.token = reinterpret_cast<int32_t*>(ws + p.token);
        // the candidates' pieces are read again, and 16 bits of a listed token's result are not its logit any more
        w.late = k.out == k.logits && sizeof(T) == 2 && k.k > 0;
        w.final = k.out == k.logits && sizeof(T) == 4;
        w.range = reinterpret_cast<int2*>(ws + p.range);
        const size_t smem = (size_t)kListWindow * 4 * (k.bias_tokens ? 2 : 1);
        if (!allow_smem(logits_lists_kernel, smem)) return CORAL_ERR_CUDA;
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3((unsigned)k.n_seq * kListCluster);
        cfg.blockDim = dim3(kListThreads);
        cfg.dynamicSmemBytes = smem;
        cfg.stream = st;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = kListCluster;
        attr[0].val.clusterDim.y = 1;
        attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        if (cudaLaunchKernelEx(&cfg, logits_lists_kernel, k, w) != cudaSuccess) return CORAL_ERR_CUDA;
    }
    const dim3 grid((unsigned)k.M * p.blocks), block(kLogitsThreads);
    w.chunk = p.chunk;
    const size_t smem = p.chunk ? LogitsWide<T>::smem(p.lists) : 0;
    if (p.lists) {
        auto kernel = p.chunk ? logits_wide_kernel<T, true> : logits_narrow_kernel<T, true>;
        if (!allow_smem(kernel, smem) || launch_pdl(kernel, grid, block, smem, st, k, w) != cudaSuccess) return CORAL_ERR_CUDA;
    } else {
        auto kernel = p.chunk ? logits_wide_kernel<T, false> : logits_narrow_kernel<T, false>;
        if (!allow_smem(kernel, smem)) return CORAL_ERR_CUDA;
        kernel<<<grid, block, smem, st>>>(k, w);
        if (cudaGetLastError() != cudaSuccess) return CORAL_ERR_CUDA;
    }
    const bool many = k.M > kLogitsEndBlocks;
    auto finish = many ? logits_finish_kernel<T, 8> : logits_finish_kernel<T, 16>;
    return launch_pdl(finish, dim3(k.M), dim3(many ? 256 : 512), 0, st, k, w) == cudaSuccess ? CORAL_OK : CORAL_ERR_CUDA;
}

}  // namespace

extern "C" {

int coral_lmhead_logits_workspace_bytes(const coral_lmhead_logits_args* a, size_t* bytes) {
    if (!bytes || !logits_args_ok(a)) return CORAL_ERR_INVALID;
    const LogitsArgs k = logits_kernel_args(a);
    const LogitsPlan p = logits_plan(k, a->type);
    if ((long long)k.M * p.blocks > 0x7fffffffLL || k.output_total > kCountMask || k.prompt_total + k.output_total + k.bias_total > 0x7fffffffLL ||
        (p.lists && k.n_seq > 0x7fffffff / kListCluster))
        return CORAL_ERR_TOO_LARGE;
    *bytes = p.bytes;
    return CORAL_OK;
}

int coral_lmhead_logits_process(const coral_lmhead_logits_args* a, void* workspace_dev, void* stream) {
    size_t bytes = 0;
    const int rc = coral_lmhead_logits_workspace_bytes(a, &bytes);
    if (rc != CORAL_OK) return rc;
    if (!workspace_dev || !aligned(workspace_dev, 256)) return CORAL_ERR_INVALID;
    const LogitsArgs k = logits_kernel_args(a);
    const LogitsPlan p = logits_plan(k, a->type);
    unsigned char* ws = static_cast<unsigned char*>(workspace_dev);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (a->type == CORAL_TYPE_BF16) return launch_logits<__nv_bfloat16>(k, p, ws, st);
    if (a->type == CORAL_TYPE_F16) return launch_logits<__half>(k, p, ws, st);
    return launch_logits<float>(k, p, ws, st);
}

int coral_lmhead_q4_packed_bytes(const coral_lmhead_q4_config* cfg, size_t* bytes) {
    if (!q4_config_ok(cfg) || !bytes) return CORAL_ERR_INVALID;
    const Q4Layout L = q4_layout(*cfg);
    *bytes = L.weights + L.scales;
    return CORAL_OK;
}

int coral_lmhead_q4_pack(const coral_lmhead_q4_config* cfg, const void* Wq_dev, const void* scales_dev, const void* zeros_dev,
                         void* packed_dev, void* stream) {
    if (!q4_config_ok(cfg) || !Wq_dev || !scales_dev || !packed_dev || (zeros_dev != nullptr) != (cfg->has_zeros != 0))
        return CORAL_ERR_INVALID;
    if (!aligned(Wq_dev, 16) || !aligned(scales_dev, 2) || !aligned(packed_dev, 256)) return CORAL_ERR_INVALID;
    const Q4Layout L = q4_layout(*cfg);
    const size_t pieces = L.weights / 16;
    const size_t blocks = (pieces + 255) / 256;
    if (blocks > 0x7fffffffu) return CORAL_ERR_TOO_LARGE;
    q4_pack_kernel<<<(unsigned)blocks, 256, 0, static_cast<cudaStream_t>(stream)>>>(
        static_cast<const unsigned char*>(Wq_dev), static_cast<const uint16_t*>(scales_dev),
        static_cast<const unsigned char*>(zeros_dev), cfg->N, cfg->K, L.KB, cfg->group, static_cast<uint4*>(packed_dev),
        static_cast<unsigned char*>(packed_dev) + L.weights, pieces);
    return cudaGetLastError() == cudaSuccess ? CORAL_OK : CORAL_ERR_CUDA;
}

int coral_lmhead_q4_workspace_bytes(const coral_lmhead_q4_config* cfg, int M, size_t* bytes) {
    if (!q4_config_ok(cfg) || !bytes || M < 1) return CORAL_ERR_INVALID;
    const int KB = q4_layout(*cfg).KB;
    int first = 0;
    size_t at = 0;
    for (Q4Pass p; q4_next_pass(*cfg, KB, M, &first, &at, &p);) {}
    *bytes = at;
    return CORAL_OK;
}

int coral_lmhead_q4_linear(const coral_lmhead_q4_config* cfg, const void* packed_dev, const void* x_dev, int x_type, int M,
                           void* out_dev, int out_type, void* workspace_dev, void* stream) {
    if (!q4_config_ok(cfg) || !packed_dev || !x_dev || !out_dev || M < 1) return CORAL_ERR_INVALID;
    if (x_type != CORAL_TYPE_BF16 && x_type != CORAL_TYPE_F16) return CORAL_ERR_INVALID;
    if (out_type != CORAL_TYPE_F32 && out_type != CORAL_TYPE_BF16 && out_type != CORAL_TYPE_F16) return CORAL_ERR_INVALID;
    if (!aligned(packed_dev, 256) || !aligned(x_dev, 16) || !aligned(out_dev, elem_size(out_type)) || !aligned(workspace_dev, 256))
        return CORAL_ERR_INVALID;
    size_t bytes = 0;
    coral_lmhead_q4_workspace_bytes(cfg, M, &bytes);
    if (bytes && !workspace_dev) return CORAL_ERR_INVALID;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int sms = 0;
    if (!device_sms(&sms)) return CORAL_ERR_CUDA;
    if (sms > kQ4TcMaxParts) sms = kQ4TcMaxParts;
    const Q4Layout L = q4_layout(*cfg);
    Q4View q{};
    q.w = static_cast<const uint4*>(packed_dev);
    q.sz = static_cast<const unsigned char*>(packed_dev) + L.weights;
    q.N = cfg->N; q.K = cfg->K; q.KB = L.KB; q.T = L.T;
    q.scale_half = cfg->scale_type == CORAL_TYPE_F16;
    unsigned char* ws = static_cast<unsigned char*>(workspace_dev);
    int first = 0;
    size_t at = 0;
    bool fresh = true;
    for (Q4Pass p; q4_next_pass(*cfg, L.KB, M, &first, &at, &p);) {
        const int rc = x_type == CORAL_TYPE_BF16 ? launch_q4<__nv_bfloat16>(*cfg, q, p, x_dev, out_dev, out_type, ws, fresh && p.staged, sms, st)
                                                 : launch_q4<__half>(*cfg, q, p, x_dev, out_dev, out_type, ws, fresh && p.staged, sms, st);
        if (rc != CORAL_OK) return rc;
        if (p.staged) fresh = false;
    }
    return CORAL_OK;
}

int coral_lmhead_q4_status(const void* workspace_dev, void* stream) {
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int status = CORAL_OK;
    if (workspace_dev && cudaMemcpyAsync(&status, workspace_dev, sizeof status, cudaMemcpyDeviceToHost, st) != cudaSuccess) return CORAL_ERR_CUDA;
    if (cudaStreamSynchronize(st) != cudaSuccess) return CORAL_ERR_CUDA;
    return status;
}

int coral_lmhead_block_norm(const coral_lmhead_norm_args* a, void* stream) {
    if (!norm_args_ok(a) || (!a->out_y_dev && !a->out_h_dev)) return CORAL_ERR_INVALID;
    if ((a->out_h_dev != nullptr) && !a->w_pre_dev) return CORAL_ERR_INVALID;
    if (!aligned(a->out_y_dev, 16) || !aligned(a->out_h_dev, 16)) return CORAL_ERR_INVALID;
    int sms = 0;
    if (!device_sms(&sms)) return CORAL_ERR_CUDA;
    NormArgs k = norm_kernel_args(a);
    k.y = a->out_y_dev;
    k.h = a->out_h_dev;
    const int tensors = 1 + (k.r ? 1 : 0) + (k.gate_mode == CORAL_GATE_FULL ? 1 : 0);
    return launch_norm_type(a->type, k, norm_plan(a->M, a->H, a->type, tensors, kNormFwdThreadsPerSm, sms), false,
                            static_cast<cudaStream_t>(stream));
}

int coral_lmhead_block_norm_backward_bytes(int M, int H, size_t* bytes) {
    if (!bytes || M < 1 || H < 8 || H % 8 != 0 || H > kNormMaxRowBytes / 2) return CORAL_ERR_INVALID;
    const int rows = M < norm_max_grid(H) ? M : norm_max_grid(H);
    *bytes = (size_t)rows * 3 * H * sizeof(float);
    return CORAL_OK;
}

int coral_lmhead_block_norm_backward(const coral_lmhead_norm_args* a, void* workspace_dev, void* stream) {
    if (!norm_args_ok(a) || !workspace_dev || !aligned(workspace_dev, 256) || !a->out_dx_dev) return CORAL_ERR_INVALID;
    if ((!a->dy_dev && !a->dh_dev) || (a->dh_dev && !a->w_pre_dev)) return CORAL_ERR_INVALID;
    if ((a->out_dr_dev && !a->r_dev) || (a->out_dgate_dev && !a->gate_dev)) return CORAL_ERR_INVALID;
    if ((a->out_dw_pre_dev && !a->w_pre_dev) || (a->out_dw_post_dev && !a->w_post_dev)) return CORAL_ERR_INVALID;
    if (!aligned(a->dy_dev, 16) || !aligned(a->dh_dev, 16) || !aligned(a->out_dx_dev, 16) || !aligned(a->out_dr_dev, 16) ||
        !aligned(a->out_dgate_dev, a->gate_mode == CORAL_GATE_FULL ? 16 : 4) || !aligned(a->out_dw_pre_dev, 4) ||
        !aligned(a->out_dw_post_dev, 4))
        return CORAL_ERR_INVALID;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int sms = 0;
    if (!device_sms(&sms)) return CORAL_ERR_CUDA;
    NormArgs k = norm_kernel_args(a);
    k.dy = a->dy_dev; k.dh = a->dh_dev;
    k.dx = a->out_dx_dev; k.dr = a->out_dr_dev;
    k.dgate = a->gate_mode == CORAL_GATE_CHANNEL ? nullptr : a->out_dgate_dev;
    k.part = static_cast<float*>(workspace_dev);
    float* d_gate = a->gate_mode == CORAL_GATE_CHANNEL ? static_cast<float*>(a->out_dgate_dev) : nullptr;
    k.want = (a->out_dw_pre_dev ? 1 : 0) | (a->out_dw_post_dev ? 2 : 0) | (d_gate ? 4 : 0);
    const int tensors = 1 + (k.r ? 1 : 0) + (k.dy ? 1 : 0) + (k.dh ? 1 : 0) + (k.gate_mode == CORAL_GATE_FULL ? 1 : 0);
    const NormPlan p = norm_plan(a->M, a->H, a->type, tensors, kNormBwdThreadsPerSm, sms);
    const int rc = launch_norm_type(a->type, k, p, true, st);
    if (rc != CORAL_OK) return rc;
    if (!k.want) return CORAL_OK;
    if (launch_pdl(block_norm_columns_kernel, dim3((a->H + 31) / 32, 3), dim3(kNormColWarps * 32), 0, st, k.part, p.grid, a->H,
                   a->out_dw_pre_dev, a->out_dw_post_dev, d_gate) != cudaSuccess)
        return CORAL_ERR_CUDA;
    return CORAL_OK;
}

}  // extern "C"

// C ABI of the drafter's attention: argument checks and kernel launches.  See include/coral_lmhead.h.
#include "coral_lmhead.h"

#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "kv4_tc.cuh"
#include "launch.cuh"
#include "prompt_attention.cuh"
#include "qk_rotate.cuh"
#include "tensor_map.cuh"

using namespace coral;

namespace {

constexpr int kSms = 148;                          // of a B200: what grids and workspaces are sized for

bool type16(int type) { return type == CORAL_TYPE_BF16 || type == CORAL_TYPE_F16; }

// Rows of `heads` heads of D columns, ld apart.
bool rows_ok(const void* p, int64_t ld, int heads, int D, int esize) {
    return p && aligned(p, 16) && ld >= (int64_t)heads * D && ld <= (1LL << 40) && ld * esize % 16 == 0;
}

// ---- norm and rotation of queries and keys -------------------------------------------------------------------
constexpr int kQkMaxHeads = 4096;
constexpr int kQkBlocks = 2;                       // resident blocks a SM; a block of a backward call has a partial row of column sums

bool qk_args_ok(const coral_lmhead_qk_args* a) {
    if (!a || a->struct_size != sizeof(*a)) return false;
    if (a->type != CORAL_TYPE_F32 && !type16(a->type)) return false;
    if (a->T < 1 || a->D < 8 || a->D > kQkMaxD || a->D % 8 != 0 || a->rot < 0 || a->rot > a->D || a->rot % 8 != 0) return false;
    if (a->n_q < 0 || a->n_k < 0 || a->n_q > kQkMaxHeads || a->n_k > kQkMaxHeads || a->n_q + a->n_k < 1) return false;
    if ((a->style != CORAL_ROPE_HALVES && a->style != CORAL_ROPE_PAIRS) || !(a->eps >= 0.f)) return false;
    if (!a->positions_dev || !aligned(a->positions_dev, 4) || !aligned(a->freqs_dev, 4) || (a->rot && !a->freqs_dev)) return false;
    return aligned(a->w_q_dev, 16) && aligned(a->w_k_dev, 16);
}

// Two granules an item, of eight columns where the members of a pair lie a multiple of eight apart, else of four.
bool qk_eight(const coral_lmhead_qk_args* a) { return a->style == CORAL_ROPE_PAIRS || a->rot % 16 == 0; }

// Threads a head if that is 4 or 8 and each has a whole item (heads of 64 and 128 columns, as a rule), else 0.
int qk_whole(const coral_lmhead_qk_args* a, const QkArgs& k) {
    const int N = qk_eight(a) ? 8 : 4;
    return N == 8 && k.items == k.lanes && a->D % 16 == 0 && (k.lanes == 4 || k.lanes == 8) ? k.lanes : 0;
}

QkArgs qk_kernel_args(const coral_lmhead_qk_args* a) {
    QkArgs k{};
    k.T = a->T; k.n_q = a->n_q; k.n_k = a->n_k; k.D = a->D; k.rot = a->rot; k.eps = a->eps;
    const int N = qk_eight(a) ? 8 : 4, turned = a->style == CORAL_ROPE_HALVES ? a->rot : 0;
    k.items = turned / 2 / N + (a->D - turned + 2 * N - 1) / (2 * N);
    for (k.lanes = 1; k.lanes < k.items; k.lanes *= 2) {}
    // a warp takes all heads of a token, or as few at a time as give every warp of the GPU some, since each computes the angles anew
    const int rows = 32 / k.lanes, most = std::max(a->n_q, a->n_k);
    k.shares = (int)std::clamp((16LL * kSms + a->T - 1) / a->T, 1LL, (long long)(most + rows - 1) / rows);
    for (int i = 0; i < 2; ++i) {
        const int heads = i ? a->n_k : a->n_q;
        k.span[i] = (heads + k.shares - 1) / k.shares;
    }
    k.pos = a->positions_dev; k.freq = a->freqs_dev;
    k.x[0] = a->q_dev; k.x[1] = a->k_dev; k.ld_x[0] = a->ld_q; k.ld_x[1] = a->ld_k;
    k.w[0] = a->w_q_dev; k.w[1] = a->w_k_dev;
    return k;
}

// Blocks of a call: no more than have turns, or than are resident.
int qk_grid(const QkArgs& k) {
    const long long turns = (long long)k.T * k.shares;
    return (int)std::min((turns + kQkWarps - 1) / kQkWarps, (long long)kQkBlocks * kSms);
}

template <typename T, bool HALVES, int N, int L>
cudaError_t launch_qk_kernel(const QkArgs& k, bool backward, int grid, cudaStream_t st) {
    if (!backward) return launch_pdl(qk_rotate_kernel<T, HALVES, N, L>, dim3(grid), dim3(kQkThreads), 0, st, k);
    constexpr size_t smem = (size_t)kQkSlots<T, N> * kQkStep<T, N>;
    static_assert(kQkStatic<N> <= kMostStatic, "what allow_smem counts with");
    if (!allow_smem(qk_rotate_backward_kernel<T, HALVES, N, L>, smem)) return cudaErrorUnknown;
    return launch_pdl(qk_rotate_backward_kernel<T, HALVES, N, L>, dim3(grid), dim3(kQkThreads), smem, st, k);
}

template <typename T>
int launch_qk(const coral_lmhead_qk_args* a, const QkArgs& k, bool backward, int grid, cudaStream_t st) {
    const int L = qk_whole(a, k);
    cudaError_t e;
    if (a->style == CORAL_ROPE_PAIRS)
        e = L == 8 ? launch_qk_kernel<T, false, 8, 8>(k, backward, grid, st) : L == 4 ? launch_qk_kernel<T, false, 8, 4>(k, backward, grid, st)
                   : launch_qk_kernel<T, false, 8, 0>(k, backward, grid, st);
    else if (qk_eight(a))
        e = L == 8 ? launch_qk_kernel<T, true, 8, 8>(k, backward, grid, st) : L == 4 ? launch_qk_kernel<T, true, 8, 4>(k, backward, grid, st)
                   : launch_qk_kernel<T, true, 8, 0>(k, backward, grid, st);
    else
        e = launch_qk_kernel<T, true, 4, 0>(k, backward, grid, st);
    return e == cudaSuccess ? CORAL_OK : CORAL_ERR_CUDA;
}

int launch_qk_type(const coral_lmhead_qk_args* a, const QkArgs& k, bool backward, int grid, cudaStream_t st) {
    if (a->type == CORAL_TYPE_BF16) return launch_qk<__nv_bfloat16>(a, k, backward, grid, st);
    if (a->type == CORAL_TYPE_F16) return launch_qk<__half>(a, k, backward, grid, st);
    return launch_qk<float>(a, k, backward, grid, st);
}

// ---- cache in 4 bits -----------------------------------------------------------------------------------------
bool kv4_config_ok(const coral_lmhead_kv4_config* c) {
    if (!c || c->struct_size != sizeof(*c) || !type16(c->type)) return false;
    if (c->D != 64 && c->D != 128) return false;
    if ((c->group != 32 && c->group != 64 && c->group != 128) || c->group > c->D) return false;
    if (c->n_pages < 1 || c->page < kKv4Block || c->page % kKv4Block != 0 || c->n_heads < 1 || c->n_heads > kQkMaxHeads) return false;
    return (int64_t)c->n_pages * c->page <= 0x7fffffff && (int64_t)c->n_pages * c->page / kKv4Block * c->n_heads <= 0x7fffffff;
}

Kv4Cache kv4_cache(const coral_lmhead_kv4_config* c, const void* base) {
    Kv4Cache k{};
    k.base = static_cast<unsigned char*>(const_cast<void*>(base));
    k.slots = c->n_pages * c->page;
    k.n_k = c->n_heads; k.page = c->page; k.groups = c->D / c->group;
    k.share = c->group == 32 ? 2 : c->group == 64 ? 3 : 4;
    k.heads = Divide(c->n_heads);
    k.subs = Divide(c->page / kKv4Block);
    return k;
}

int launch_kv4_rows(const coral_lmhead_kv4_config* c, bool store, const void* cache, const Kv4Rows& r, cudaStream_t st) {
    const bool wide = c->D == 128, bf16 = c->type == CORAL_TYPE_BF16;
    const int per = kKv4RowThreads / (c->D / 8);
    const dim3 grid((r.rows - 1) / per + 1, 2);
    void (*f)(Kv4Cache, Kv4Rows);
    if (store) f = bf16 ? (wide ? kv4_store_kernel<__nv_bfloat16, 128> : kv4_store_kernel<__nv_bfloat16, 64>) : (wide ? kv4_store_kernel<__half, 128> : kv4_store_kernel<__half, 64>);
    else f = bf16 ? (wide ? kv4_load_kernel<__nv_bfloat16, 128> : kv4_load_kernel<__nv_bfloat16, 64>) : (wide ? kv4_load_kernel<__half, 128> : kv4_load_kernel<__half, 64>);
    return launch_pdl(f, grid, dim3(kKv4RowThreads), 0, st, kv4_cache(c, cache), r) == cudaSuccess ? CORAL_OK : CORAL_ERR_CUDA;
}

// From how many rows of a key head on (query tokens times heads of its group) the tensor-core kernel takes a call.  us, warp MMAs | tensor
// cores, groups of 32 and of 128 columns of 128, bf16: 8 x 3000 tokens 36 rows 65 and 60 | 48 and 46, 128 rows 128 and 117 | 52 and 50; 60000
// tokens 36 rows 144 and 131 | 94 and 91; 4000 tokens 36 rows 21 and 19 | 20.  Up to 32 rows two row groups share what they unpack, and the warp
// MMAs take 37 and 34, 76 and 70, 16 (the tensor cores the same as for 36).
constexpr long long kKv4ManyFrom = 33;

struct Kv4Plan {
    int nr, row_groups, row_blocks, splits;        // nr 0: kv4_many_kernel
    long long units;                               // blocks without the split
    size_t ml, o, bytes;                           // offsets in the workspace and its size
};

bool kv4_attention_ok(const coral_lmhead_kv4_config* c, const coral_lmhead_kv4_attention_args* a) {
    if (!kv4_config_ok(c) || !a || a->struct_size != sizeof(*a)) return false;
    if (a->n_seq < 0 || a->n_rows < 0 || a->max_q < 1 || a->width < 1 || a->ld_table < a->width || !std::isfinite(a->scale)) return false;
    if (a->n_q < 1 || a->n_q > kQkMaxHeads || a->n_q % c->n_heads != 0) return false;
    if (a->tree_mask_dev && a->max_q > kKv4MaxTree) return false;
    if (!a->q_offsets_dev && (int64_t)a->n_seq * a->max_q > a->n_rows) return false;
    if (!a->table_dev || !aligned(a->table_dev, 4) || !a->lens_dev || !aligned(a->lens_dev, 4) || !aligned(a->q_offsets_dev, 8) ||
        !aligned(a->tree_mask_dev, 8) || !aligned(a->out_lse_dev, 4))
        return false;
    return rows_ok(a->q_dev, a->ld_q, a->n_q, c->D, 2) && rows_ok(a->out_dev, a->ld_out, a->n_q, c->D, 2);
}

Kv4Plan kv4_plan(const coral_lmhead_kv4_config* c, const coral_lmhead_kv4_attention_args* a) {
    Kv4Plan p{};
    const long long rows = (long long)a->max_q * (a->n_q / c->n_heads);
    p.nr = rows <= 8 ? 1 : rows < kKv4ManyFrom ? 2 : 0;
    static_assert(kKv4ManyFrom <= 2 * 8 * 2 + 1, "two row groups of two tiles of eight rows are what kv4_attention_kernel takes");
    p.row_groups = p.nr && rows > 8 * p.nr ? 2 : 1;
    p.row_blocks = p.nr ? 1 : (int)((rows - 1) / 256 + 1);
    p.units = (long long)a->n_seq * c->n_heads * p.row_blocks;
    // The number of parts whose rounds of resident blocks take the least, a block counted as its tokens plus 512 for what it begins and
    // ends with (64 sequences of up to 4096 tokens, 256 blocks unsplit: 58 us in 5 parts, 35 in one).  A part has a span at least.
    const long long resident = (p.nr == 1 ? 2 : 1) * kSms, tokens = (long long)a->width * c->page, spans = (tokens - 1) / (kKv4SpanBlocks * kKv4Block) + 1;
    const long long most = std::min(spans, (long long)kKv4MaxSplits);
    long long best = -1;
    p.splits = 1;
    for (int rounds = 1; rounds <= 8 && p.units; ++rounds) {
        const long long s = std::clamp(rounds * resident / p.units, 1LL, most), cost = (p.units * s - 1 + resident) / resident * ((tokens - 1) / s + 1 + 512);
        if (best < 0 || cost < best) {
            best = cost;
            p.splits = (int)s;
        }
    }
    size_t at = 256;
    if (p.splits > 1) {
        const size_t n = (size_t)p.splits * a->n_rows * a->n_q;
        p.ml = at;
        at += (n * 8 + 255) / 256 * 256;
        p.o = at;
        at += n * c->D * 4;
    }
    p.bytes = at;
    return p;
}

template <typename T, int D, int NG, int NR>
cudaError_t launch_kv4(Kv4Args k, const Kv4Plan& p, cudaStream_t st) {
    constexpr int chunk = kKv4Chunk<NG, NR> * Kv4Rowset<T, D, NG, NR>::kBytes, outputs = kKv4Warps * 8 * NR * D * 4;
    const int streams = kKv4Warps / p.row_groups;
    k.slots = std::min(kKv4Ring<NR> / (streams * chunk), kKv4MaxSlots);
    const size_t smem = std::max(streams * k.slots * chunk, outputs);          // the warps' outputs take the ring's place
    if (!allow_smem(kv4_attention_kernel<T, D, NG, NR>, smem)) return cudaErrorUnknown;
    return launch_pdl(kv4_attention_kernel<T, D, NG, NR>, dim3((unsigned)(p.units * p.splits)), dim3(kKv4Threads), smem, st, k);
}

template <typename T, int D, int NG>
cudaError_t launch_kv4_rows_by(const Kv4Args& k, const Kv4Plan& p, cudaStream_t st) {
    if (p.nr) return p.nr == 1 ? launch_kv4<T, D, NG, 1>(k, p, st) : launch_kv4<T, D, NG, 2>(k, p, st);
    constexpr size_t smem = kt_smem_bytes<D, NG>();
    if (!allow_smem(kv4_many_kernel<T, D, NG>, smem)) return cudaErrorUnknown;
    return launch_pdl(kv4_many_kernel<T, D, NG>, dim3((unsigned)(p.units * p.splits)), dim3(kKtThreads), smem, st, k);
}

template <typename T, int D>
int launch_kv4_groups(const Kv4Args& k, const Kv4Plan& p, cudaStream_t st) {
    cudaError_t e = cudaErrorUnknown;
    if (k.c.groups == 1) e = launch_kv4_rows_by<T, D, 1>(k, p, st);
    else if (k.c.groups == 2) e = launch_kv4_rows_by<T, D, 2>(k, p, st);
    else if constexpr (D == 128) e = launch_kv4_rows_by<T, D, 4>(k, p, st);
    if (e != cudaSuccess) return CORAL_ERR_CUDA;
    if (p.splits == 1) return CORAL_OK;
    const long long rows = (long long)k.n_seq * k.max_q * k.n_q;
    // up to 8 parts: a warp a row; more: four
    const bool few = p.splits <= 8;
    const unsigned blocks = (unsigned)(few ? (rows - 1) / kKv4JoinWarps + 1 : rows);
    return launch_pdl(few ? kv4_join_kernel<T, D, 1> : kv4_join_kernel<T, D, kKv4JoinWarps>, dim3(blocks), dim3(kKv4JoinWarps * 32), 0, st, k) == cudaSuccess ? CORAL_OK : CORAL_ERR_CUDA;
}

// ---- attention over prompts ----------------------------------------------------------------------------------
bool prompt_args_ok(const coral_lmhead_prompt_args* a) {
    if (!a || a->struct_size != sizeof(*a) || !type16(a->type)) return false;
    if (a->n_seq < 0 || a->T < 0 || a->Tk < 0 || a->n_k < 1 || a->n_q < a->n_k || a->n_q > kQkMaxHeads || a->n_q % a->n_k != 0) return false;
    if (a->D < 8 || a->D > 128 || a->D % 8 != 0 || !(a->scale > 0.f) || !std::isfinite(a->scale)) return false;
    if (!a->q_offsets_dev || !aligned(a->q_offsets_dev, 8) || !aligned(a->k_offsets_dev, 8) || !aligned(a->out_lse_dev, 4)) return false;
    if (!a->k_offsets_dev && a->Tk != a->T) return false;
    return rows_ok(a->q_dev, a->ld_q, a->n_q, a->D, 2) && rows_ok(a->out_dev, a->ld_out, a->n_q, a->D, 2) &&
           (a->Tk == 0 || (rows_ok(a->k_dev, a->ld_k, a->n_k, a->D, 2) && rows_ok(a->v_dev, a->ld_v, a->n_k, a->D, 2)));
}

// Rows [T x heads x D] in boxes of 64 columns x `heads_box` heads x `tokens` tokens, 128-byte swizzle; columns past D read as zero.
bool make_rows_map(CUtensorMap* map, int type, const void* base, int T, int heads, int D, long long ld, int heads_box, int tokens) {
    static const EncodeTiledFn enc = encode_tiled_fn();
    if (!enc) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)heads, (cuuint64_t)T};
    const cuuint64_t strides[2] = {(cuuint64_t)D * 2, (cuuint64_t)ld * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)heads_box, (cuuint32_t)tokens}, ones[3] = {1, 1, 1};
    return enc(map, type == CORAL_TYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(base), dims,
               strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int DB>
int launch_prompt(const coral_lmhead_prompt_args* a, const PaArgs& k, unsigned blocks, cudaStream_t st) {
    CUtensorMap q, kk, v;
    if (!make_rows_map(&q, a->type, a->q_dev, a->T, a->n_q, a->D, a->ld_q, k.gp, 128 / k.gp)) return CORAL_ERR_CUDA;
    kk = v = q;                                    // without keys there are no loads of them
    if (a->Tk && (!make_rows_map(&kk, a->type, a->k_dev, a->Tk, a->n_k, a->D, a->ld_k, 1, kPaKeys) ||
                  !make_rows_map(&v, a->type, a->v_dev, a->Tk, a->n_k, a->D, a->ld_v, 1, kPaKeys)))
        return CORAL_ERR_CUDA;
    constexpr size_t smem = pa_smem_bytes<DB>();
    if (!allow_smem(prompt_attention_kernel<T, DB>, smem)) return CORAL_ERR_CUDA;
    return launch_pdl(prompt_attention_kernel<T, DB>, dim3(blocks), dim3(kPaThreads), smem, st, k, q, kk, v) == cudaSuccess ? CORAL_OK : CORAL_ERR_CUDA;
}

}  // namespace

extern "C" {

int coral_lmhead_qk_rotate(const coral_lmhead_qk_args* a, void* stream) {
    if (!qk_args_ok(a)) return CORAL_ERR_INVALID;
    const int e = elem_size(a->type);
    if (a->n_q && (!rows_ok(a->q_dev, a->ld_q, a->n_q, a->D, e) || !rows_ok(a->out_q_dev, a->ld_out_q, a->n_q, a->D, e))) return CORAL_ERR_INVALID;
    if (a->n_k && (!rows_ok(a->k_dev, a->ld_k, a->n_k, a->D, e) || !rows_ok(a->out_k_dev, a->ld_out_k, a->n_k, a->D, e))) return CORAL_ERR_INVALID;
    QkArgs k = qk_kernel_args(a);
    k.y[0] = a->out_q_dev; k.y[1] = a->out_k_dev; k.ld_y[0] = a->ld_out_q; k.ld_y[1] = a->ld_out_k;
    return launch_qk_type(a, k, false, qk_grid(k), static_cast<cudaStream_t>(stream));
}

int coral_lmhead_qk_rotate_backward_bytes(int T, int n_q, int n_k, int D, size_t* bytes) {
    if (!bytes || T < 1 || n_q < 0 || n_k < 0 || n_q + n_k < 1 || n_q > kQkMaxHeads || n_k > kQkMaxHeads || D < 8 || D > kQkMaxD || D % 8 != 0)
        return CORAL_ERR_INVALID;
    const long long turns = (long long)T * std::max(n_q, n_k);        // at most: a head each
    *bytes = (size_t)std::min((turns + kQkWarps - 1) / kQkWarps, (long long)kQkBlocks * kSms) * 2 * D * sizeof(float);
    return CORAL_OK;
}

int coral_lmhead_qk_rotate_backward(const coral_lmhead_qk_args* a, void* workspace_dev, void* stream) {
    if (!qk_args_ok(a)) return CORAL_ERR_INVALID;
    const int e = elem_size(a->type);
    if (a->n_q && (!rows_ok(a->dout_q_dev, a->ld_dout_q, a->n_q, a->D, e) || !rows_ok(a->dq_dev, a->ld_dq, a->n_q, a->D, e) ||
                   (a->w_q_dev && !rows_ok(a->q_dev, a->ld_q, a->n_q, a->D, e))))
        return CORAL_ERR_INVALID;
    if (a->n_k && (!rows_ok(a->dout_k_dev, a->ld_dout_k, a->n_k, a->D, e) || !rows_ok(a->dk_dev, a->ld_dk, a->n_k, a->D, e) ||
                   (a->w_k_dev && !rows_ok(a->k_dev, a->ld_k, a->n_k, a->D, e))))
        return CORAL_ERR_INVALID;
    if ((a->dw_q_dev && (!a->w_q_dev || !a->n_q)) || (a->dw_k_dev && (!a->w_k_dev || !a->n_k)) || !aligned(a->dw_q_dev, 4) || !aligned(a->dw_k_dev, 4))
        return CORAL_ERR_INVALID;
    const bool want = a->dw_q_dev || a->dw_k_dev;
    if ((want && !workspace_dev) || !aligned(workspace_dev, 256)) return CORAL_ERR_INVALID;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    QkArgs k = qk_kernel_args(a);
    k.dy[0] = a->dout_q_dev; k.dy[1] = a->dout_k_dev; k.ld_dy[0] = a->ld_dout_q; k.ld_dy[1] = a->ld_dout_k;
    k.y[0] = a->dq_dev; k.y[1] = a->dk_dev; k.ld_y[0] = a->ld_dq; k.ld_y[1] = a->ld_dk;
    k.part = want ? static_cast<float*>(workspace_dev) : nullptr;
    const int grid = qk_grid(k);
    const int rc = launch_qk_type(a, k, true, grid, st);
    if (rc != CORAL_OK || !want) return rc;
    return launch_pdl(qk_columns_kernel, dim3((a->D + 31) / 32, 2), dim3(kQkColWarps * 32), 0, st, k.part, grid, a->D, a->dw_q_dev, a->dw_k_dev) == cudaSuccess
               ? CORAL_OK : CORAL_ERR_CUDA;
}

int coral_lmhead_prompt_attention(const coral_lmhead_prompt_args* a, void* workspace_dev, void* stream) {
    if (!prompt_args_ok(a) || !workspace_dev || !aligned(workspace_dev, 256)) return CORAL_ERR_INVALID;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (a->n_seq == 0 || a->T == 0) return cudaMemsetAsync(workspace_dev, 0, sizeof(DeviceState), st) == cudaSuccess ? CORAL_OK : CORAL_ERR_CUDA;
    PaArgs k{};
    k.n_seq = a->n_seq; k.T = a->T; k.Tk = a->Tk; k.n_q = a->n_q; k.n_k = a->n_k; k.G = a->n_q / a->n_k; k.D = a->D;
    // heads side by side in a tile: the largest power of two that divides a group
    for (k.gp = 1; k.gp < 128 && k.G % (2 * k.gp) == 0; k.gp *= 2) ++k.gp_log2;
    k.c = a->scale * 1.4426950408889634f;
    k.q_offsets = a->q_offsets_dev; k.k_offsets = a->k_offsets_dev;
    k.q = a->q_dev; k.k = a->k_dev; k.v = a->v_dev;
    k.ld_q = a->ld_q; k.ld_k = a->ld_k; k.ld_v = a->ld_v; k.ld_out = a->ld_out;
    k.out = a->out_dev; k.lse = a->out_lse_dev;
    k.st = static_cast<DeviceState*>(workspace_dev);
    const int per = 256 / k.gp;                        // tokens of a pair of tiles; sequences have at most T / per + n_seq pairs in all
    const long long slots = std::min((long long)a->T, (long long)a->T / per + a->n_seq), units = slots * a->n_k * (k.G / k.gp);
    if (units > 0x7fffffffLL) return CORAL_ERR_TOO_LARGE;
    k.units = (int)units;
    const unsigned blocks = (unsigned)std::min(units, (long long)kSms);
    if (a->type == CORAL_TYPE_BF16)
        return a->D > 64 ? launch_prompt<__nv_bfloat16, 2>(a, k, blocks, st) : launch_prompt<__nv_bfloat16, 1>(a, k, blocks, st);
    return a->D > 64 ? launch_prompt<__half, 2>(a, k, blocks, st) : launch_prompt<__half, 1>(a, k, blocks, st);
}

int coral_lmhead_kv4_bytes(const coral_lmhead_kv4_config* c, size_t* bytes) {
    if (!kv4_config_ok(c) || !bytes) return CORAL_ERR_INVALID;
    *bytes = (size_t)c->n_pages * (c->page / kKv4Block) * c->n_heads * kv4_cache(c, nullptr).block_bytes(c->D);
    return CORAL_OK;
}

int coral_lmhead_kv4_store(const coral_lmhead_kv4_config* c, void* cache_dev, const void* k_dev, int64_t ld_k, const void* v_dev, int64_t ld_v,
                           const int64_t* slots_dev, int T, void* stream) {
    if (!kv4_config_ok(c) || !cache_dev || !aligned(cache_dev, 256) || T < 0) return CORAL_ERR_INVALID;
    if (!rows_ok(k_dev, ld_k, c->n_heads, c->D, 2) || !rows_ok(v_dev, ld_v, c->n_heads, c->D, 2) || !slots_dev || !aligned(slots_dev, 8)) return CORAL_ERR_INVALID;
    if ((int64_t)T * c->n_heads > 0x7fffffff - kKv4RowThreads) return CORAL_ERR_TOO_LARGE;
    if (T == 0) return CORAL_OK;
    const Kv4Rows r{slots_dev, T * c->n_heads, const_cast<void*>(k_dev), const_cast<void*>(v_dev), ld_k, ld_v};
    return launch_kv4_rows(c, true, cache_dev, r, static_cast<cudaStream_t>(stream));
}

int coral_lmhead_kv4_load(const coral_lmhead_kv4_config* c, const void* cache_dev, const int64_t* slots_dev, int T, void* out_k_dev, int64_t ld_k,
                          void* out_v_dev, int64_t ld_v, void* stream) {
    if (!kv4_config_ok(c) || !cache_dev || !aligned(cache_dev, 256) || T < 0 || !slots_dev || !aligned(slots_dev, 8)) return CORAL_ERR_INVALID;
    if ((!out_k_dev && !out_v_dev) || (out_k_dev && !rows_ok(out_k_dev, ld_k, c->n_heads, c->D, 2)) || (out_v_dev && !rows_ok(out_v_dev, ld_v, c->n_heads, c->D, 2)))
        return CORAL_ERR_INVALID;
    if ((int64_t)T * c->n_heads > 0x7fffffff - kKv4RowThreads) return CORAL_ERR_TOO_LARGE;
    if (T == 0) return CORAL_OK;
    const Kv4Rows r{slots_dev, T * c->n_heads, out_k_dev, out_v_dev, ld_k, ld_v};
    return launch_kv4_rows(c, false, cache_dev, r, static_cast<cudaStream_t>(stream));
}

int coral_lmhead_kv4_attention_bytes(const coral_lmhead_kv4_config* c, const coral_lmhead_kv4_attention_args* a, size_t* bytes) {
    if (!bytes || !kv4_attention_ok(c, a)) return CORAL_ERR_INVALID;
    const Kv4Plan p = kv4_plan(c, a);
    if (p.units * p.splits > 0x7fffffffLL || (int64_t)a->n_seq * a->max_q * a->n_q > 0x7fffffffLL) return CORAL_ERR_TOO_LARGE;
    *bytes = p.bytes;
    return CORAL_OK;
}

int coral_lmhead_kv4_attention(const coral_lmhead_kv4_config* c, const void* cache_dev, const coral_lmhead_kv4_attention_args* a, void* workspace_dev,
                               void* stream) {
    size_t bytes = 0;
    const int rc = coral_lmhead_kv4_attention_bytes(c, a, &bytes);
    if (rc != CORAL_OK) return rc;
    if (!cache_dev || !aligned(cache_dev, 256) || !workspace_dev || !aligned(workspace_dev, 256)) return CORAL_ERR_INVALID;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const Kv4Plan p = kv4_plan(c, a);
    if (p.units == 0 || a->n_rows == 0) return cudaMemsetAsync(workspace_dev, 0, sizeof(DeviceState), st) == cudaSuccess ? CORAL_OK : CORAL_ERR_CUDA;
    unsigned char* ws = static_cast<unsigned char*>(workspace_dev);
    Kv4Args k{};
    k.c = kv4_cache(c, cache_dev);
    k.n_seq = a->n_seq; k.n_rows = a->n_rows; k.max_q = a->max_q; k.n_q = a->n_q; k.G = a->n_q / c->n_heads; k.width = a->width; k.n_pages = c->n_pages;
    k.row_groups = p.row_groups; k.row_blocks = p.row_blocks; k.splits = p.splits;
    k.scale2 = a->scale * 1.4426950408889634f;
    k.ld_table = a->ld_table; k.ld_q = a->ld_q; k.ld_out = a->ld_out;
    k.q = a->q_dev; k.table = a->table_dev; k.lens = a->lens_dev; k.q_offsets = a->q_offsets_dev;
    k.tree = reinterpret_cast<const unsigned long long*>(a->tree_mask_dev);
    k.out = a->out_dev; k.lse = a->out_lse_dev;
    k.part_ml = reinterpret_cast<float2*>(ws + p.ml);
    k.part_o = reinterpret_cast<float*>(ws + p.o);
    k.st = reinterpret_cast<DeviceState*>(ws);
    if (c->type == CORAL_TYPE_BF16) return c->D == 128 ? launch_kv4_groups<__nv_bfloat16, 128>(k, p, st) : launch_kv4_groups<__nv_bfloat16, 64>(k, p, st);
    return c->D == 128 ? launch_kv4_groups<__half, 128>(k, p, st) : launch_kv4_groups<__half, 64>(k, p, st);
}

int coral_lmhead_attention_status(const void* workspace_dev, void* stream) { return coral_lmhead_q4_status(workspace_dev, stream); }

}  // extern "C"

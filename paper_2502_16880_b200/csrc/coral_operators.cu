// C ABI of the operators around the draft step: argument checks and kernel launches.  See include/coral_lmhead.h.
#include "coral_lmhead.h"

#include <cuda_runtime.h>

#include "block_norm.cuh"
#include "launch.cuh"

using namespace coral;

namespace {

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline int elem_size(int type) { return type == CORAL_TYPE_F32 ? 4 : 2; }

bool device_sms(int* sms) {
    int dev = 0;
    return cudaGetDevice(&dev) == cudaSuccess && cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess;
}

// The attribute is per kernel and device; above 48 KB it has to be raised before the launch.
template <typename K>
bool allow_smem(K kernel, size_t bytes) {
    return bytes <= 48 * 1024 ||
           cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == cudaSuccess;
}

// ---- block norm ----------------------------------------------------------------------------------------------
constexpr int kNormFwdThreadsPerSm = 1024, kNormBwdThreadsPerSm = 512;
constexpr size_t kNormSmemPerSm = 200 * 1024;
constexpr int kNormMaxBlocksPerSm = 16;
constexpr int kNormSmCap = 160;                 // most SMs the partial rows of the workspace are sized for

struct NormPlan {
    int nv, threads, grid, stages;
    size_t smem;
};

// nv: 8-column chunks a thread keeps.  Threads are the chunks over nv rounded up to a warp, so that a row of 3584
// columns runs 448 threads and wastes none.
NormPlan norm_plan(int M, int H, int type, int tensors, int threads_per_sm, int sms) {
    NormPlan p{};
    const int chunks = H / 8;
    p.nv = chunks <= kNormMaxThreads ? 1 : chunks <= 2 * kNormMaxThreads ? 2 : 4;
    p.threads = ((chunks + p.nv - 1) / p.nv + 31) / 32 * 32;
    int blocks = threads_per_sm / p.threads;
    blocks = blocks < 1 ? 1 : blocks > kNormMaxBlocksPerSm ? kNormMaxBlocksPerSm : blocks;
    const size_t stage = (size_t)tensors * p.nv * p.threads * 8 * elem_size(type);
    size_t stages = kNormSmemPerSm / blocks / stage;
    if (stages < 1) {                            // very wide fp32 rows: one block a SM
        blocks = 1;
        stages = 1;
    }
    p.stages = stages > 4 ? 4 : (int)stages;
    if (sms > kNormSmCap) sms = kNormSmCap;
    const long long most = (long long)sms * blocks;
    p.grid = (int)(M < most ? M : most);
    p.smem = stage * p.stages;
    return p;
}

// Most partial rows a backward call can write.
int norm_max_grid(int H) {
    const int chunks = H / 8;
    const int threads = (((chunks > kNormMaxThreads ? kNormMaxThreads : chunks)) + 31) / 32 * 32;
    int blocks = kNormBwdThreadsPerSm / threads;
    blocks = blocks < 1 ? 1 : blocks > kNormMaxBlocksPerSm ? kNormMaxBlocksPerSm : blocks;
    return 2 * blocks * kNormSmCap;              // nv > 1 halves the threads at most, which doubles the blocks
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
    if (p.nv == 2) return launch_norm<T, 2>(k, p, backward, st);
    return launch_norm<T, 4>(k, p, backward, st);
}

int launch_norm_type(int type, const NormArgs& k, const NormPlan& p, bool backward, cudaStream_t st) {
    if (type == CORAL_TYPE_BF16) return launch_norm_nv<__nv_bfloat16>(k, p, backward, st);
    if (type == CORAL_TYPE_F16) return launch_norm_nv<__half>(k, p, backward, st);
    return launch_norm_nv<float>(k, p, backward, st);
}

}  // namespace

extern "C" {

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
    const int tensors = 1 + (k.r ? 1 : 0) + (k.dy ? 1 : 0) + (k.dh ? 1 : 0) + (k.gate_mode == CORAL_GATE_FULL ? 1 : 0);
    const NormPlan p = norm_plan(a->M, a->H, a->type, tensors, kNormBwdThreadsPerSm, sms);
    const int rc = launch_norm_type(a->type, k, p, true, st);
    if (rc != CORAL_OK) return rc;
    if (!a->out_dw_pre_dev && !a->out_dw_post_dev && !d_gate) return CORAL_OK;
    if (launch_pdl(block_norm_columns_kernel, dim3((a->H + 31) / 32, 3), dim3(kNormColWarps * 32), 0, st, k.part, p.grid, a->H,
                   a->out_dw_pre_dev, a->out_dw_post_dev, d_gate) != cudaSuccess)
        return CORAL_ERR_CUDA;
    return CORAL_OK;
}

}  // extern "C"

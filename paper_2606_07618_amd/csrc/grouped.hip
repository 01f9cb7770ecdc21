// Products of grouped rows with NVFP4 weights of each group's own: the experts of a mixture, y = x W_e^T and dx = dy W_e.
#include "grouped_plan.h"
#include "grouped_product.h"
#include "product_host.h"

namespace {

using namespace product_host;
using grouped_plan::GroupedPlan, grouped_plan::plan_grouped, grouped_plan::most_groups_of;
using grouped_plan::kLargeTile, grouped_plan::kLargeThreads, grouped_plan::kSmallTile, grouped_plan::kSmallThreads;
using grouped_plan::kFewThreads, grouped_plan::kFewFours;

constexpr int64_t kMostGroupedRows = 0x7FFFFFFF, kMostExperts = (int64_t)1 << 20;

using Large = grouped_product::Tile<256, 4>;
using Small = grouped_product::Tile<128, 2>;
static_assert(Large::M == kLargeTile && Large::N == kLargeTile && Large::kThreads == kLargeThreads &&
              Small::M == kSmallTile && Small::N == kSmallTile && Small::kThreads == kSmallThreads, "the plan's tiles");

int check_grouped(int64_t rows, int64_t experts, int64_t n, int64_t k, int block) {
    if (block != 16 && block != 32 && block != 64 && block != 128) return NVFP4_ERR_BLOCK;
    if (const int rc = check_dims(rows, n, k)) return rc;
    if (rows > kMostGroupedRows || experts < 0 || experts > kMostExperts || k % block) return NVFP4_ERR_SHAPE;
    return NVFP4_OK;
}

bool grouped_launchable(int64_t rows, int64_t experts, int64_t outer, bool turned) {
    const GroupedPlan plan = plan_grouped(rows, experts, outer, turned);
    return launchable(most_groups_of(rows, experts, outer, plan), plan.threads);
}

template <int R, int C, int H>
void launch_few(const grouped_product::Args& p, dim3 grid, hipStream_t stream) {
    hipLaunchKernelGGL((grouped_product::few_kernel<R, C, H>), grid, dim3(kFewThreads * H), 0, stream, p);
}

template <class T>
void launch_tiled(const grouped_product::Args& p, bool turned, dim3 grid, hipStream_t stream) {
    auto kernel = turned ? grouped_product::grouped_kernel<T, true> : grouped_product::grouped_kernel<T, false>;
    hipLaunchKernelGGL(kernel, grid, dim3(T::kThreads), 0, stream, p);
}

int run_grouped(grouped_product::Args p, bool turned, int block, hipStream_t stream) {
    const GroupedPlan plan = plan_grouped(p.rows, p.experts, p.outer, turned);
    p.shift = block == 16 ? 4 : block == 32 ? 5 : block == 64 ? 6 : 7;
    p.tiles_n = ceil_div(p.outer, plan.width);
    const dim3 grid((unsigned)most_groups_of(p.rows, p.experts, p.outer, plan));
    if (plan.height == Large::M) launch_tiled<Large>(p, turned, grid, stream);
    else if (plan.height == Small::M) launch_tiled<Small>(p, turned, grid, stream);
    else if (plan.height == 16) plan.width == 128 ? launch_few<2, 1, 1>(p, grid, stream) : launch_few<1, 1, kFewFours>(p, grid, stream);
    else plan.width == 128 ? launch_few<2, 2, 1>(p, grid, stream) : launch_few<1, 2, 1>(p, grid, stream);
    return launched();
}

int64_t grouped_grad_workspace(int64_t rows, int64_t n, int64_t ld) {
    return needs_pack(n, ld) ? up(rows * packed_ld(n) * 2, 256) : 0;
}

}  // namespace

extern "C" {

int nvfp4_grouped_product(const void* x, int64_t ldx, const int* offsets, const uint8_t* q, const uint8_t* scales, int block,
                          const float* tensor_scales, int64_t rows, int64_t experts, int64_t n, int64_t k, int out_dtype,
                          int clear, void* out, void* stream) {
    if (out_dtype != NVFP4_IN_F32 && out_dtype != NVFP4_IN_BF16) return NVFP4_ERR_DTYPE;
    if (const int rc = check_grouped(rows, experts, n, k, block)) return rc;
    if (ldx < k || ldx > kMaxLd || !grouped_launchable(rows, experts, n, false)) return NVFP4_ERR_SHAPE;
    if (rows == 0 || n == 0 || (experts == 0 && !clear)) return NVFP4_OK;
    if (!out || !offsets || (experts > 0 && (!tensor_scales || (k > 0 && (!x || !q || !scales))))) return NVFP4_ERR_NULL;
    if (!aligned(x, 16) || ldx % 8 || !aligned(q, 16) || !aligned(out, 16) || !aligned(tensor_scales, 4) || !aligned(offsets, 4))
        return NVFP4_ERR_ALIGN;
    grouped_product::Args p = {};
    p.x = static_cast<const char*>(x), p.ld = ldx * 2, p.rows = rows, p.offsets = offsets, p.experts = (int)experts;
    p.q = reinterpret_cast<const char*>(q), p.scales = scales, p.S = tensor_scales, p.n = n, p.k = k, p.inner = k, p.outer = n;
    p.out = out, p.out_f32 = out_dtype == NVFP4_IN_F32, p.clear = clear != 0;
    return run_grouped(p, false, block, (hipStream_t)stream);
}

int64_t nvfp4_grouped_product_grad_input_workspace_bytes(int64_t rows, int64_t n, int64_t ld) {
    if (const int rc = check_dims(rows, n, 0)) return rc;
    return grouped_grad_workspace(rows, n, ld);
}

int nvfp4_grouped_product_grad_input(const void* dy, int64_t ld, const int* offsets, const uint8_t* q, const uint8_t* scales,
                                     int block, const float* tensor_scales, int64_t rows, int64_t experts, int64_t n, int64_t k,
                                     int out_dtype, int clear, void* dx, void* workspace, size_t workspace_bytes, void* stream) {
    if (out_dtype != NVFP4_IN_F32 && out_dtype != NVFP4_IN_BF16) return NVFP4_ERR_DTYPE;
    if (const int rc = check_grouped(rows, experts, n, k, block)) return rc;
    if (ld < n || ld > kMaxLd || !grouped_launchable(rows, experts, k, true)) return NVFP4_ERR_SHAPE;
    if (rows == 0 || k == 0 || (experts == 0 && !clear)) return NVFP4_OK;
    if (!dx || !offsets || (experts > 0 && (!tensor_scales || (n > 0 && (!dy || !q || !scales))))) return NVFP4_ERR_NULL;
    if (!aligned(dy, 16) || !aligned(q, 16) || !aligned(dx, 16) || !aligned(tensor_scales, 4) || !aligned(offsets, 4))
        return NVFP4_ERR_ALIGN;
    if (const int rc = check_workspace(workspace, workspace_bytes, grouped_grad_workspace(rows, n, ld))) return rc;
    if (needs_pack(n, ld) && n > 0) {
        if (const int rc = pack_bf16_rows(dy, rows, n, ld, workspace, (hipStream_t)stream)) return rc;
        dy = workspace, ld = packed_ld(n);
    }
    grouped_product::Args p = {};
    p.x = static_cast<const char*>(dy), p.ld = ld * 2, p.rows = rows, p.offsets = offsets, p.experts = (int)experts;
    p.q = reinterpret_cast<const char*>(q), p.scales = scales, p.S = tensor_scales, p.n = n, p.k = k, p.inner = n, p.outer = k;
    p.out = dx, p.out_f32 = out_dtype == NVFP4_IN_F32, p.clear = clear != 0;
    return run_grouped(p, true, block, (hipStream_t)stream);
}

}  // extern "C"

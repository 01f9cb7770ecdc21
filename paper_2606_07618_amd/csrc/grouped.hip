// Products of grouped rows with NVFP4 weights of each group's own: the experts of a mixture, y = x W_e^T and dx = dy W_e.
#include "grouped_product.h"
#include "product_host.h"

namespace {

using namespace product_host;
using grouped_product::kFewThreads;

constexpr int64_t kMostGroupedRows = 0x7FFFFFFF, kMostExperts = (int64_t)1 << 20;

// Which kernel, by the rows that a group has on average (how many each has is known on the device alone; every kernel takes
// any number).  Few rows: 16 or 32 of a group at a time, and 128 weight rows a workgroup, or 64 where those would be few; up to
// 64 where tiles would keep less than half of the chip busy.  Measured, 50 rows a group: eight of [4096, 14336] 123 us in 32s,
// 144 in tiles; 16 of [1001, 2080] 25 and 37; 128 of [1536, 4096] 213 and 161.  The largest tile where groups fill it more than
// half and three quarters of the compute units have one (128 of 200 rows: 340 us, 454 in the smaller one).
struct GroupedPlan { int height, width, threads; };

// Fours of waves along the contraction, of 16 rows where workgroups are few.
constexpr int kFewFours = 2;

using Large = grouped_product::Tile<256, 4>;
using Small = grouped_product::Tile<128, 2>;

GroupedPlan plan_grouped(int64_t rows, int64_t experts, int64_t outer, bool turned) {
    const int64_t active = rows < experts ? rows : experts, each = active ? ceil_div(rows, active) : 0;
    if (!turned && (each <= 32 || (each <= 64 && active * ceil_div(outer, Small::N) < 512))) {
        const int height = each <= 16 ? 16 : 32;
        const int64_t tiles = active * ceil_div(each, height);
        const int width = tiles * ceil_div(outer, 128) >= 512 ? 128 : 64;
        return {height, width, kFewThreads * (height == 16 && width == 64 ? kFewFours : 1)};
    }
    if (each > 128 && active * ceil_div(each, 256) * ceil_div(outer, 256) >= 192) return {Large::M, Large::N, Large::kThreads};
    return {Small::M, Small::N, Small::kThreads};
}

// Workgroups: for the row tiles that there may be, each XCD as many, and one at least that finds rows of no group to clear;
// and for the parts that its last tiles are cut into.
int64_t most_groups_of(int64_t rows, int64_t experts, int64_t outer, const GroupedPlan& plan) {
    const int64_t tiles = rows / plan.height + (rows < experts ? rows : experts);
    const int64_t more = plan.height == Large::M ? grouped_product::kUnits : 1;
    return (ceil_div(tiles * ceil_div(outer, plan.width), kXcds) + more) * kXcds;
}

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
    if (plan.threads == Large::kThreads && plan.height == Large::M) launch_tiled<Large>(p, turned, grid, stream);
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

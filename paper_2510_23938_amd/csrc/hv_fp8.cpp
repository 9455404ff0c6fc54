// hv_fp8.cpp -- C ABI of the 8-bit operators: argument checks and launches.
#include "hv_fp8.h"
#include "hv_host.h"
#include "hv_inspect.h"

using namespace hvh;

namespace {

constexpr uint64_t kMaxRows = ((uint64_t)1 << 31) - 1;
constexpr uint64_t kMaxCols = (uint64_t)1 << 24;
constexpr uint64_t kMaxSide = (uint64_t)1 << 27;  // of a product: rows and columns, rounded up to tiles, count in 32 bits
constexpr uint64_t kMaxLd = (uint64_t)1 << 31;

static_assert(HV_BF16 == hv::kTypeBf16 && HV_F16 == hv::kTypeF16 && HV_F32 == hv::kTypeF32, "element types");

hv_status check_type(hv_type type) {
    if (type == HV_BF16 || type == HV_F16 || type == HV_F32) return HV_OK;
    return fail(HV_ERR_INVALID_ARG, "unknown element type %d", (int)type);
}

size_t size_of(hv_type type) { return type == HV_F32 ? 4 : 2; }

hv_status check_size(uint64_t rows, uint64_t cols) {
    if (rows > kMaxRows || cols > kMaxCols)
        return fail(HV_ERR_INVALID_ARG, "%llu x %llu exceeds the limit of %llu rows and %llu columns",
                    (unsigned long long)rows, (unsigned long long)cols, (unsigned long long)kMaxRows,
                    (unsigned long long)kMaxCols);
    return HV_OK;
}

hv_status check_product(uint64_t m, uint64_t n, uint64_t k) {
    if (m > kMaxSide || n > kMaxSide || k > kMaxCols)
        return fail(HV_ERR_INVALID_ARG, "m = %llu, n = %llu, k = %llu exceed the limits of 2^27, 2^27 and 2^24",
                    (unsigned long long)m, (unsigned long long)n, (unsigned long long)k);
    return HV_OK;
}

// A matrix operand that is read or written: present, at its element's alignment, rows apart.
hv_status check_matrix(const char* what, const void* p, size_t element, uint64_t ld, uint64_t cols) {
    if (p == nullptr) return fail(HV_ERR_INVALID_ARG, "%s is NULL", what);
    if ((uintptr_t)p % element != 0)
        return fail(HV_ERR_INVALID_ARG, "%s is not %zu-byte aligned", what, element);
    if (ld < cols || ld > kMaxLd)
        return fail(HV_ERR_INVALID_ARG, "%s: leading dimension %llu is below its %llu columns or above the limit of %llu",
                    what, (unsigned long long)ld, (unsigned long long)cols, (unsigned long long)kMaxLd);
    return HV_OK;
}

#define HV_TRY(call)                     \
    do {                                 \
        const hv_status st_ = (call);    \
        if (st_ != HV_OK) return st_;    \
    } while (0)

hv_status done(hipError_t e, const char* what) { return e == hipSuccess ? HV_OK : hip_fail(e, what); }

}  // namespace

extern "C" {

hv_status hv_fp8_quantize(hv_type type, const void* x, uint64_t ld_x, uint64_t rows, uint64_t cols,
                          uint32_t tile_rows, uint8_t* codes, uint64_t ld_codes, float* scales, hipStream_t stream) {
    HV_TRY(check_type(type));
    HV_TRY(check_size(rows, cols));
    if (tile_rows != 1 && tile_rows != 128)
        return fail(HV_ERR_INVALID_ARG, "tile_rows = %u is neither 1 nor 128", tile_rows);
    if (rows == 0 || cols == 0) return HV_OK;
    HV_TRY(check_matrix("x", x, size_of(type), ld_x, cols));
    HV_TRY(check_matrix("codes", codes, 1, ld_codes, cols));
    HV_TRY(check_matrix("scales", scales, sizeof(float), cols, cols));
    return done(hv::launch_fp8_quantize(type, x, ld_x, rows, cols, tile_rows == 128, codes, ld_codes, scales, stream),
                "quantisation kernel");
}

hv_status hv_fp8_rms_norm(hv_type type, const void* x, uint64_t ld_x, const void* residual, uint64_t ld_residual,
                          const void* weight, float eps, uint64_t rows, uint64_t cols, void* residual_out,
                          uint64_t ld_residual_out, uint8_t* codes, uint64_t ld_codes, float* scales,
                          hipStream_t stream) {
    HV_TRY(check_type(type));
    HV_TRY(check_size(rows, cols));
    if (!(eps >= 0.0f)) return fail(HV_ERR_INVALID_ARG, "eps = %g is negative or NaN", (double)eps);
    if (rows == 0 || cols == 0) return HV_OK;
    const size_t e = size_of(type);
    if ((residual == nullptr) != (residual_out == nullptr))
        return fail(HV_ERR_INVALID_ARG, "residual and residual_out come together or not at all");
    HV_TRY(check_matrix("x", x, e, ld_x, cols));
    if (residual != nullptr) {
        HV_TRY(check_matrix("residual", residual, e, ld_residual, cols));
        HV_TRY(check_matrix("residual_out", residual_out, e, ld_residual_out, cols));
        if ((residual_out == x && ld_residual_out != ld_x) ||
            (residual_out == residual && ld_residual_out != ld_residual))
            return fail(HV_ERR_INVALID_ARG, "residual_out overlaps an input with another leading dimension");
    }
    HV_TRY(check_matrix("weight", weight, e, cols, cols));
    HV_TRY(check_matrix("codes", codes, 1, ld_codes, cols));
    HV_TRY(check_matrix("scales", scales, sizeof(float), cols, cols));
    const hv::NormArgs a = {x,    ld_x, residual, ld_residual, weight, eps, rows, cols, residual_out, ld_residual_out,
                            codes, ld_codes, scales};
    return done(hv::launch_fp8_rms_norm(type, a, stream), "norm kernel");
}

hv_status hv_fp8_gated(hv_type type, const void* gate, uint64_t ld_gate, const void* up, uint64_t ld_up,
                       uint64_t rows, uint64_t cols, uint8_t* codes, uint64_t ld_codes, float* scales,
                       hipStream_t stream) {
    HV_TRY(check_type(type));
    HV_TRY(check_size(rows, cols));
    if (rows == 0 || cols == 0) return HV_OK;
    HV_TRY(check_matrix("gate", gate, size_of(type), ld_gate, cols));
    HV_TRY(check_matrix("up", up, size_of(type), ld_up, cols));
    HV_TRY(check_matrix("codes", codes, 1, ld_codes, cols));
    HV_TRY(check_matrix("scales", scales, sizeof(float), cols, cols));
    return done(hv::launch_fp8_gated(type, gate, ld_gate, up, ld_up, rows, cols, codes, ld_codes, scales, stream),
                "gated kernel");
}

size_t hv_fp8_matmul_workspace_bytes(hv_type type, int aligned, uint64_t m, uint64_t n, uint64_t k) {
    if (check_type(type) != HV_OK || check_product(m, n, k) != HV_OK || m == 0 || n == 0) return 0;
    return round_up(hv::fp8_matmul_workspace(type == HV_F32, aligned != 0, m, n, k));
}

hv_status hv_fp8_matmul(hv_type type, const uint8_t* a, uint64_t ld_a, const float* a_scales, const uint8_t* b,
                        uint64_t ld_b, const float* b_scales, uint64_t m, uint64_t n, uint64_t k, void* c,
                        uint64_t ld_c, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    HV_TRY(check_type(type));
    HV_TRY(check_product(m, n, k));
    if (m == 0 || n == 0) return HV_OK;
    if (k > 0) {
        HV_TRY(check_matrix("a", a, 1, ld_a, k));
        HV_TRY(check_matrix("b", b, 1, ld_b, k));
        HV_TRY(check_matrix("a_scales", a_scales, sizeof(float), k, k));
        HV_TRY(check_matrix("b_scales", b_scales, sizeof(float), k, k));
    }
    HV_TRY(check_matrix("c", c, size_of(type), ld_c, n));
    const bool aligned = ld_a % 16 == 0 && ld_b % 16 == 0 && (uintptr_t)a % 16 == 0 && (uintptr_t)b % 16 == 0;
    const bool tiles = hv::fp8_matmul_tiles(ld_a, ld_b);
    const size_t need = tiles ? hv_fp8_matmul_workspace_bytes(type, aligned, m, n, k) : 0;
    if (need > 0) {
        if (workspace == nullptr || workspace_bytes < need)
            return fail(HV_ERR_WORKSPACE, "workspace needs %zu bytes, got %zu%s", need, workspace_bytes,
                        workspace ? "" : " (NULL)");
        if ((uintptr_t)workspace % kAlign != 0) return fail(HV_ERR_WORKSPACE, "workspace is not 256-byte aligned");
    }
    const hv::MatmulArgs args = {a, ld_a, a_scales, b, ld_b, b_scales, m, n, k, c, ld_c, workspace};
    return done(hv::launch_fp8_matmul(type, args, stream), "product kernel");
}

hv_status hv_fp8_matmul_launches(hv_type type, int aligned, uint64_t m, uint64_t n, uint64_t k, int* launches, int* kind,
                                 uint64_t* rows, uint64_t* cols, uint32_t* splits) {
    HV_TRY(check_type(type));
    HV_TRY(check_product(m, n, k));
    if (launches == nullptr || kind == nullptr || rows == nullptr || cols == nullptr || splits == nullptr)
        return fail(HV_ERR_INVALID_ARG, "launches, kind, rows, cols and splits must be non-NULL");
    hv::MatmulPart parts[hv::kMatmulMostParts];
    *launches = m == 0 || n == 0 ? 0 : hv::fp8_matmul_parts(type == HV_F32, aligned != 0, true, m, n, k, parts);
    for (int i = 0; i < *launches; ++i) {
        kind[i] = parts[i].kind;
        rows[i] = parts[i].rows;
        cols[i] = parts[i].cols;
        splits[i] = parts[i].splits;
    }
    return HV_OK;
}

}  // extern "C"

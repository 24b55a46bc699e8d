// Low-rank adapters beside a pruned fully connected layer, many in one batch.
//
// Row i of the batch has adapter l = ids[i], or none (any value outside
// [0, L)).  With A [L][r][m], B [L][r][n] and a factor s_l:
//
//   forward   u[i][j]  = s_l sum_c x[i][c] A[l][j][c]
//             y[i][o]  = base[i][o] + sum_j u[i][j] B[l][j][o]
//   backward  g[i][j]  = s_l sum_o dy[i][o] B[l][j][o]
//             dx[i][c] = base[i][c] + sum_j g[i][j] A[l][j][c]
//             dA[l][j][c] = sum over rows i of l of g[i][j] x[i][c]
//             dB[l][j][o] = sum over rows i of l of u[i][j] dy[i][o]
//
// Both factors hold one row per rank, so that forward and backward are the
// same two kernels with the factors exchanged: lora_rows.hip (narrow product,
// then wide product) and lora_grad.hip (a factor's gradient).  Here: the entry
// points and their checks.
#include <initializer_list>

#include "lora.h"

namespace onexn {
namespace {

constexpr int32_t kMaxAdapters = 32767, kMaxRows = 1 << 26, kMaxFeatures = 1 << 27;   // what the grids hold

onexn_status launched(const char* fn) {
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return fail(ONEXN_ERR_HIP, "%s: launch failed: %s", fn, hipGetErrorString(err));
    return ONEXN_OK;
}

bool misaligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }
size_t bytes_of(onexn_dtype dt) { return dt == ONEXN_BF16 ? 2 : 4; }

// What both directions check: types, sizes, strides and the arrays that every call reads.
onexn_status check_common(const char* fn, onexn_dtype xdt, onexn_dtype odt, int32_t rows, int32_t m, int32_t n,
                          int32_t r, int32_t L, const void* A, const void* B, const int32_t* ids, const float* scale) {
    if ((xdt != ONEXN_F32 && xdt != ONEXN_BF16) || (odt != ONEXN_F32 && odt != ONEXN_BF16))
        return fail(ONEXN_ERR_DTYPE, "%s: unknown dtype", fn);
    if (odt != xdt && odt != ONEXN_F32)
        return fail(ONEXN_ERR_DTYPE, "%s: output dtype must be the input dtype or F32", fn);
    if (rows < 0 || m < 1 || n < 1 || r < 1 || L < 1)
        return fail(ONEXN_ERR_ARG, "%s: m, n, r and L must be positive, rows >= 0", fn);
    if (r > kMaxRank) return fail(ONEXN_ERR_UNSUPPORTED, "%s: rank %d beyond %d", fn, r, kMaxRank);
    if (int64_t(r) * m > INT32_MAX || int64_t(r) * n > INT32_MAX || L > kMaxAdapters || rows > kMaxRows ||
        m > kMaxFeatures || n > kMaxFeatures)
        return fail(ONEXN_ERR_UNSUPPORTED,
                    "%s: a factor beyond int32 indexing, more than %d adapters, %d rows or %d features", fn,
                    kMaxAdapters, kMaxRows, kMaxFeatures);
    if (!A || !B || (rows > 0 && !ids)) return fail(ONEXN_ERR_NULL, "%s: NULL pointer argument", fn);
    if (misaligned(A, bytes_of(xdt)) || misaligned(B, bytes_of(xdt)) || misaligned(ids, 4) || misaligned(scale, 4))
        return fail(ONEXN_ERR_ARG, "%s: an array is not aligned to its elements", fn);
    return ONEXN_OK;
}

// One [rows][width] array: present where the batch has rows, aligned, its rows apart.
onexn_status check_rows(const char* fn, const char* name, const void* p, bool required, onexn_dtype dt, int32_t rows,
                        int32_t width, int64_t stride) {
    if (!p) {
        if (required && rows > 0) return fail(ONEXN_ERR_NULL, "%s: NULL %s", fn, name);
        return ONEXN_OK;
    }
    if (stride < width || stride > INT64_MAX / 16 / (rows + 1LL))
        return fail(ONEXN_ERR_ARG, "%s: the row stride of %s is below its width or too large", fn, name);
    if (misaligned(p, bytes_of(dt))) return fail(ONEXN_ERR_ARG, "%s: %s is not aligned to its elements", fn, name);
    return ONEXN_OK;
}

// An output of the call is none of its other arrays (as far as their addresses show it).
onexn_status check_apart(const char* fn, const char* name, const void* out, std::initializer_list<const void*> others) {
    for (const void* o : others)
        if (out && out == o) return fail(ONEXN_ERR_ARG, "%s: %s must not overlap another array", fn, name);
    return ONEXN_OK;
}

// The result may be its base, row for row.
onexn_status check_in_place(const char* fn, const char* name, const void* y, int64_t stride, const void* base,
                            int64_t base_stride) {
    if (y && y == base && stride != base_stride)
        return fail(ONEXN_ERR_ARG, "%s: %s is its base, with another row stride", fn, name);
    return ONEXN_OK;
}

}  // namespace
}  // namespace onexn

using namespace onexn;

extern "C" onexn_status onexn_fc_lora_fwd(const void* x_dev, onexn_dtype xdt, int64_t x_stride, int32_t rows, int32_t m,
                                          const void* A_dev, const void* B_dev, int32_t n, int32_t r, int32_t L,
                                          const float* scale_dev, const int32_t* ids_dev, const void* base_dev,
                                          int64_t base_stride, void* y_dev, onexn_dtype ydt, int64_t y_stride,
                                          float* u_dev, void* stream) {
    clear_error();
    const char* fn = "fc_lora_fwd";
    if (onexn_status st = check_common(fn, xdt, ydt, rows, m, n, r, L, A_dev, B_dev, ids_dev, scale_dev)) return st;
    if (onexn_status st = check_rows(fn, "x", x_dev, true, xdt, rows, m, x_stride)) return st;
    if (onexn_status st = check_rows(fn, "base", base_dev, false, ydt, rows, n, base_stride)) return st;
    if (onexn_status st = check_rows(fn, "y", y_dev, true, ydt, rows, n, y_stride)) return st;
    if (onexn_status st = check_rows(fn, "u", u_dev, false, ONEXN_F32, rows, r, r)) return st;
    if (rows == 0) return ONEXN_OK;
    if (onexn_status st = check_apart(fn, "y", y_dev, {x_dev, A_dev, B_dev, ids_dev, scale_dev, u_dev})) return st;
    if (onexn_status st = check_apart(fn, "u", u_dev, {x_dev, A_dev, B_dev, ids_dev, scale_dev, base_dev})) return st;
    if (onexn_status st = check_in_place(fn, "y", y_dev, y_stride, base_dev, base_stride)) return st;
    const LoraRowsArgs a{x_dev, A_dev, B_dev, base_dev, y_dev, u_dev, scale_dev, ids_dev,
                     x_stride, base_stride, y_stride, rows, m, n, r, L};
    launch_lora_rows(a, xdt, ydt, static_cast<hipStream_t>(stream));
    return launched(fn);
}

extern "C" size_t onexn_fc_lora_bwd_workspace_bytes(int32_t rows, int32_t m, int32_t n, int32_t r, int32_t L) {
    if (rows < 0 || m < 1 || n < 1 || r < 1 || L < 1) return 0;
    return (size_t(rows) * r * 4 + 15) / 16 * 16 + 16 + lora_grad_workspace(rows, m, n, r, L);
}

extern "C" onexn_status onexn_fc_lora_bwd(const void* x_dev, onexn_dtype xdt, int64_t x_stride, int32_t rows, int32_t m,
                                          const void* A_dev, const void* B_dev, int32_t n, int32_t r, int32_t L,
                                          const float* scale_dev, const int32_t* ids_dev, const float* u_dev,
                                          const void* dy_dev, int64_t dy_stride, const void* base_dev,
                                          int64_t base_stride, void* dx_dev, onexn_dtype dxdt, int64_t dx_stride,
                                          float* dA_dev, float* dB_dev, void* workspace_dev, size_t workspace_bytes,
                                          void* stream) {
    clear_error();
    const char* fn = "fc_lora_bwd";
    if (onexn_status st = check_common(fn, xdt, dxdt, rows, m, n, r, L, A_dev, B_dev, ids_dev, scale_dev)) return st;
    if (!dx_dev && !dA_dev && !dB_dev) return fail(ONEXN_ERR_NULL, "%s: dx, dA and dB are all NULL", fn);
    if (onexn_status st = check_rows(fn, "x", x_dev, dA_dev != nullptr, xdt, rows, m, x_stride)) return st;
    if (onexn_status st = check_rows(fn, "u", u_dev, dB_dev != nullptr, ONEXN_F32, rows, r, r)) return st;
    if (onexn_status st = check_rows(fn, "dy", dy_dev, true, xdt, rows, n, dy_stride)) return st;
    if (onexn_status st = check_rows(fn, "base", base_dev, false, dxdt, rows, m, base_stride)) return st;
    if (onexn_status st = check_rows(fn, "dx", dx_dev, false, dxdt, rows, m, dx_stride)) return st;
    if (misaligned(dA_dev, 4) || misaligned(dB_dev, 4))
        return fail(ONEXN_ERR_ARG, "%s: dA or dB is not aligned to its elements", fn);
    if (rows > 0) {
        if (onexn_status st = check_apart(fn, "dx", dx_dev, {x_dev, A_dev, B_dev, ids_dev, scale_dev, u_dev, dy_dev})) return st;
        if (onexn_status st = check_in_place(fn, "dx", dx_dev, dx_stride, base_dev, base_stride)) return st;
        if (onexn_status st = check_apart(fn, "dA", dA_dev, {x_dev, A_dev, B_dev, ids_dev, scale_dev, u_dev, dy_dev,
                                                             base_dev, dx_dev, dB_dev})) return st;
        if (onexn_status st = check_apart(fn, "dB", dB_dev, {x_dev, A_dev, B_dev, ids_dev, scale_dev, u_dev, dy_dev,
                                                             base_dev, dx_dev})) return st;
    }
    const size_t need = onexn_fc_lora_bwd_workspace_bytes(rows, m, n, r, L);
    if (!workspace_dev) return fail(ONEXN_ERR_NULL, "%s: NULL workspace", fn);
    if (workspace_bytes < need)
        return fail(ONEXN_ERR_BUFSIZE, "%s: workspace of %zu bytes, %zu needed", fn, workspace_bytes, need);
    if (misaligned(workspace_dev, 16)) return fail(ONEXN_ERR_ARG, "%s: workspace must be 16-byte aligned", fn);
    hipStream_t s = static_cast<hipStream_t>(stream);
    float* g = static_cast<float*>(workspace_dev);
    if (rows > 0 && (dx_dev || dA_dev)) {
        const LoraRowsArgs a{dy_dev, B_dev, A_dev, base_dev, dx_dev, g, scale_dev, ids_dev,
                         dy_stride, base_stride, dx_stride, rows, n, m, r, L};
        launch_lora_rows(a, xdt, dxdt, s);
    }
    if (dA_dev || dB_dev) {
        void* more = static_cast<char*>(workspace_dev) + (size_t(rows) * r * 4 + 15) / 16 * 16;
        const LoraGradArgs a{x_dev, dy_dev, g, u_dev, dA_dev, dB_dev, ids_dev, more,
                             x_stride, dy_stride, rows, m, n, r, L};
        launch_lora_grad(a, xdt, s);
    }
    return launched(fn);
}

// hikonv_linear, hikonv_grouped_linear: argument checks and the choice of kernel.
#include <cstring>
#include <mutex>

#include "hikonv_cuda.cuh"
#include "hikonv_linear.h"

namespace hikonv {

static size_t element_bytes(int out_type) {
    return out_type == HIKONV_OUT_CODES ? 1 : out_type == HIKONV_OUT_SUMS || out_type == HIKONV_OUT_F32 ? 4 : 2;
}
// Whether two memory ranges have a byte in common.
static bool overlap(const void *a, size_t an, const void *b, size_t bn) {
    return a && b && an && bn && (uintptr_t)a < (uintptr_t)b + bn && (uintptr_t)b < (uintptr_t)a + an;
}
// Whether two matrices of M rows, so many bytes apart and long (no longer than apart), have a byte in common.  Rows equally far apart may lie
// between one another, as columns of one buffer do; where the distances differ, the ranges from the first byte to the last must be apart.
static bool rows_overlap(const void *a, size_t a_row, size_t a_bytes, const void *b, size_t b_row, size_t b_bytes, size_t M) {
    if (!overlap(a, (M - 1) * a_row + a_bytes, b, (M - 1) * b_row + b_bytes)) return false;
    if (M == 1 || a_row != b_row) return true;
    const size_t ahead = (uintptr_t)b >= (uintptr_t)a ? ((uintptr_t)b - (uintptr_t)a) % a_row
                                                      : (a_row - ((uintptr_t)a - (uintptr_t)b) % a_row) % a_row;    // of b's rows to a's before
    return ahead < a_bytes || ahead + b_bytes > a_row;
}

static int linear_run(const void *d_x, long long x_row, const void *d_w, int w_bits, const int32_t *d_offsets, int grouped, int E, int M,
                      int N, int K, int p, int q, int xs, int ws, void *d_out, long long out_row, const hikonv_epilogue_t *ep, void *workspace, size_t workspace_bytes,
                      void *stream) {
    const int rc = validate_codes(p, q);
    if (rc != HIKONV_OK) return rc;
    if (!ep || M < 0 || N < 1 || K < 1 || E < 1) return HIKONV_ERR_INVALID_ARG;
    if (E > HIKONV_MAX_GROUPS || M > (1 << 30) || N > (1 << 30)) return HIKONV_ERR_UNSUPPORTED;
    const int type = ep->out_type, real = type >= HIKONV_OUT_F32;
    if (type < HIKONV_OUT_SUMS || type > HIKONV_OUT_BF16) return HIKONV_ERR_INVALID_ARG;
    if (ep->activation < HIKONV_ACT_NONE || ep->activation > HIKONV_ACT_GELU) return HIKONV_ERR_INVALID_ARG;
    if (!real && (ep->activation || ep->d_x_scale || ep->d_w_scale || ep->d_residual)) return HIKONV_ERR_INVALID_ARG;
    if (type == HIKONV_OUT_SUMS && ep->d_bias) return HIKONV_ERR_INVALID_ARG;
    if (type == HIKONV_OUT_CODES) {
        if (ep->shift < 0 || ep->shift > 31 || ep->lo < -128 || ep->hi > 255 || ep->lo > ep->hi) return HIKONV_ERR_INVALID_ARG;
    } else if (ep->shift || ep->lo || ep->hi) {
        return HIKONV_ERR_INVALID_ARG;
    }
    if (w_bits != 8 && (w_bits != q || (q != 1 && q != 2 && q != 4))) return HIKONV_ERR_INVALID_ARG;
    if (((long long)K * w_bits) % 8 != 0) return HIKONV_ERR_UNSUPPORTED;
    const long long xmax = xs ? 1ll << (p - 1) : (1ll << p) - 1, wmax = ws ? 128 : (1ll << q) - 1;
    if (K * xmax * wmax > 0x7FFFFFFFll) return HIKONV_ERR_NO_FIT;
    if (M == 0) return HIKONV_OK;
    if (M == 1) x_row = K, out_row = N;                          // there is no second row
    const long long res_row = M == 1 ? N : ep->residual_row_stride;
    if (!d_x || !d_w || !d_out || (grouped && !d_offsets)) return HIKONV_ERR_INVALID_ARG;
    if (x_row < K || out_row < N || (ep->d_residual && res_row < N)) return HIKONV_ERR_INVALID_ARG;
    if (x_row >= (1ll << 40) || out_row >= (1ll << 40) || res_row >= (1ll << 40)) return HIKONV_ERR_INVALID_ARG;   // byte offsets stay in 64 bits
    const size_t elem = element_bytes(type);
    if ((uintptr_t)d_out % elem || (uintptr_t)ep->d_residual % elem || (uintptr_t)ep->d_bias % 4 || (uintptr_t)ep->d_x_scale % 4 ||
        (uintptr_t)ep->d_w_scale % 4 || (uintptr_t)d_offsets % 4)
        return HIKONV_ERR_INVALID_ARG;
    const long long w_row = (long long)K * w_bits / 8;
    const size_t out_bytes = ((size_t)(M - 1) * out_row + N) * elem, columns = (size_t)E * N * 4;
    if (rows_overlap(d_out, out_row * elem, N * elem, d_x, x_row, K, M) || overlap(d_out, out_bytes, d_w, (size_t)E * N * w_row) ||
        overlap(d_out, out_bytes, d_offsets, ((size_t)E + 1) * 4) || overlap(d_out, out_bytes, ep->d_x_scale, (size_t)M * 4) ||
        overlap(d_out, out_bytes, ep->d_w_scale, columns) || overlap(d_out, out_bytes, ep->d_bias, columns))
        return HIKONV_ERR_INVALID_ARG;
    if (ep->d_residual && !(ep->d_residual == d_out && res_row == out_row) &&
        rows_overlap(d_out, out_row * elem, N * elem, ep->d_residual, res_row * elem, N * elem, M))
        return HIKONV_ERR_INVALID_ARG;

    LinearParams k;
    memset(&k, 0, sizeof(k));
    k.x = (const uint8_t *)d_x; k.w = (const uint8_t *)d_w; k.offsets = d_offsets;
    k.x_row = x_row; k.w_row = w_row;
    k.M = M; k.N = N; k.K = K; k.E = E;
    k.x_signed = xs; k.w_signed = ws;
    k.x_u8 = !xs && p == 8; k.w_u8 = !ws && q == 8;
    k.w_bits = w_bits;
    k.down = w_bits < 8 && ws ? 8 - w_bits : 0;
    k.out_type = type; k.act = ep->activation;
    k.out = d_out; k.residual = ep->d_residual; k.bias = ep->d_bias;
    k.x_scale = ep->d_x_scale; k.w_scale = ep->d_w_scale;
    k.out_row = out_row; k.res_row = res_row;
    k.shift = ep->shift; k.lo = ep->lo; k.hi = ep->hi;
    const int rows = grouped ? ceil_div(M, E) : M;               // of a group, on average
    if (linear_rows_takes(k, rows)) return launch_linear_rows(k, (cudaStream_t)stream);
    // the copied rows lie over nothing that is read or written
    const size_t need = linear_tc_workspace(k);
    const struct { const void *at; size_t bytes; } operands[] = {
        {d_x, (size_t)(M - 1) * x_row + K}, {d_w, (size_t)E * N * w_row}, {d_out, out_bytes}, {d_offsets, ((size_t)E + 1) * 4},
        {ep->d_x_scale, (size_t)M * 4}, {ep->d_w_scale, columns}, {ep->d_bias, columns}, {ep->d_residual, ((size_t)(M - 1) * res_row + N) * elem}};
    for (const auto &o : operands)
        if (overlap(workspace, need, o.at, o.bytes)) return HIKONV_ERR_INVALID_ARG;
    return launch_linear_tc(k, workspace, workspace_bytes, (cudaStream_t)stream);
}

}  // namespace hikonv

using namespace hikonv;

extern "C" int hikonv_linear(const void *d_x, long long x_row_stride, const void *d_w, int w_store_bits, int M, int N, int K, int p, int q,
                             int x_signed, int w_signed, void *d_out, long long out_row_stride, const hikonv_epilogue_t *epilogue,
                             void *d_workspace, size_t workspace_bytes, void *stream) {
    return linear_run(d_x, x_row_stride, d_w, w_store_bits, nullptr, 0, 1, M, N, K, p, q, x_signed != 0, w_signed != 0, d_out, out_row_stride,
                      epilogue, d_workspace, workspace_bytes, stream);
}

extern "C" size_t hikonv_linear_workspace_bytes(const void *d_x, long long x_row_stride, const void *d_w, int w_store_bits, int E, int M, int N,
                                                int K) {
    if (E < 0 || M < 1 || N < 1 || K < 1 || (w_store_bits != 1 && w_store_bits != 2 && w_store_bits != 4 && w_store_bits != 8)) return 0;
    static const int32_t some = 0;                               // a layer of groups; the kernels' choice asks for no more than that
    LinearParams k;
    memset(&k, 0, sizeof(k));
    k.x = (const uint8_t *)d_x; k.w = (const uint8_t *)d_w; k.offsets = E > 0 ? &some : nullptr;
    k.x_row = M == 1 ? K : x_row_stride; k.w_row = (long long)K * w_store_bits / 8;
    k.M = M; k.N = N; k.K = K; k.E = E > 0 ? E : 1;
    k.w_bits = w_store_bits;
    return linear_rows_takes(k, E > 0 ? ceil_div(M, E) : M) ? 0 : linear_tc_workspace(k);
}

extern "C" int hikonv_grouped_linear(const void *d_x, long long x_row_stride, const void *d_w, int w_store_bits, const int32_t *d_offsets,
                                     int E, int T, int N, int K, int p, int q, int x_signed, int w_signed, void *d_out,
                                     long long out_row_stride, const hikonv_epilogue_t *epilogue, void *d_workspace, size_t workspace_bytes,
                                     void *stream) {
    return linear_run(d_x, x_row_stride, d_w, w_store_bits, d_offsets, 1, E, T, N, K, p, q, x_signed != 0, w_signed != 0, d_out,
                      out_row_stride, epilogue, d_workspace, workspace_bytes, stream);
}

extern "C" int hikonv_linear_wait_timeouts(unsigned int *h_count) {
    if (!h_count) return HIKONV_ERR_INVALID_ARG;
    constexpr int kDevices = 64;
    static std::mutex mutex;
    static unsigned int told[kDevices];                              // what earlier calls have reported
    *h_count = 0;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kDevices || cudaDeviceSynchronize() != cudaSuccess) return HIKONV_ERR_CUDA;
    std::lock_guard<std::mutex> lock(mutex);
    unsigned int total = 0;
    const int rc = read_linear_timeouts(&total);
    if (rc != HIKONV_OK) return rc;
    *h_count = total - told[dev];
    told[dev] = total;
    return HIKONV_OK;
}

extern "C" int hikonv_linear_wait_check(long long cycles, void *stream) {
    if (cycles < 0 || cycles > kWaitCycles) return HIKONV_ERR_INVALID_ARG;
    return launch_linear_wait_check(cycles, (cudaStream_t)stream);
}

// Rows of 8-bit values: entry points of q8rows.hpp.
#include <cmath>
#include <initializer_list>

#include "owt_host.hpp"
#include "q8rows.hpp"

namespace owt {

// more than an eighth of the 256 MB behind the L2 caches
template <class T> static bool big(int rows, int cols) { return (size_t)rows * cols * sizeof(T) > (32u << 20); }

// A launch counts its threads in 32 bits: rows that take more work-groups than half of that go in several launches.
constexpr long kLaunchThreads = 1L << 31;
template <class F> static void launches_of(int rows, long most, F f)
{
    const int each = (int)(most < rows ? most : rows);
    for (long first = 0; first < rows; first += each) f((size_t)first, (int)(rows - first < each ? rows - first : each));
}
template <class T> static Q8RowParams rows_from(Q8RowParams p, size_t first, int rows)
{
    p.x = (const T *)p.x + first * p.cols;
    if (p.res) p.res = (const T *)p.res + first * p.cols;
    if (p.h) p.h = (T *)p.h + first * p.cols;
    p.q += first * p.pitch;
    p.scale += first;
    if (p.rstd) p.rstd += first;
    p.rows = rows;
    return p;
}

// A row of n pieces: threads a row and pieces a thread.  Rows of up to 64 threads need no barrier, and short ones share a wavefront.
template <class T, bool NORM, bool RES, bool BIG>
static void launch_rows_as(const Q8RowParams &p, hipStream_t s)
{
    const long n = (long)(p.pitch / Piece<T>::V);
    auto go = [&](auto kernel, int tpr) {
        const int threads = tpr > 256 ? tpr : 256, rpw = threads / tpr;
        launches_of(p.rows, kLaunchThreads / threads * rpw, [&](size_t first, int rows) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)((rows + rpw - 1) / rpw)), dim3(threads), 0, s, rows_from<T>(p, first, rows));
        });
    };
    if (n <= 16) go(q8_rows_kernel<T, NORM, RES, 16, 1, false, BIG>, 16);
    else if (n <= 32) go(q8_rows_kernel<T, NORM, RES, 32, 1, false, BIG>, 32);
    else if (n <= 64) go(q8_rows_kernel<T, NORM, RES, 64, 1, false, BIG>, 64);
    else if (n <= 128) go(q8_rows_kernel<T, NORM, RES, 64, 2, false, BIG>, 64);
    else if (n <= 256) go(q8_rows_kernel<T, NORM, RES, 64, 4, false, BIG>, 64);
    else if (n <= 512) go(q8_rows_kernel<T, NORM, RES, 256, 2, false, BIG>, 256);
    else if (n <= 1024) go(q8_rows_kernel<T, NORM, RES, 256, 4, false, BIG>, 256);
    else if (n <= 2048) go(q8_rows_kernel<T, NORM, RES, 1024, 2, false, BIG>, 1024);
    else if (n <= 4096) go(q8_rows_kernel<T, NORM, RES, 1024, 4, false, BIG>, 1024);
    else go(q8_rows_kernel<T, NORM, RES, 1024, 1, true, BIG>, 1024);
}

template <class T, bool NORM, bool RES> static void launch_rows(const Q8RowParams &p, hipStream_t s)
{
    if (big<T>(p.rows, p.cols)) launch_rows_as<T, NORM, RES, true>(p, s);
    else launch_rows_as<T, NORM, RES, false>(p, s);
}

template <class T> static void launch_unpack(const signed char *q, const float *scale, void *x, int rows, int cols, hipStream_t s)
{
    const long n = ((long)cols + Piece<T>::V - 1) / Piece<T>::V;
    int lpr = 0;
    while (lpr < 8 && (1L << lpr) < n) lpr++;
    const unsigned segs = (unsigned)((n + (1L << lpr) - 1) >> lpr), rpw = 256u >> lpr;
    const size_t pitch = q8_pitch(cols);
    launches_of(rows, kLaunchThreads / 256 / segs * rpw, [&](size_t first, int n_rows) {
        hipLaunchKernelGGL(q8_unpack_kernel<T>, dim3((unsigned)((n_rows + rpw - 1) / rpw) * segs), dim3(256), 0, s, q + first * pitch, scale + first,
                           (T *)x + first * cols, n_rows, cols, pitch, lpr, segs);
    });
}

// Strips of rows that the backward pass sums the gain's gradient over, one in flight for each group of threads: as many as hide its loads
// (more would only be more partial sums to write and read), and few enough that all have the same number of rows, or one less.
static int bwd_strips(int rows, int tpr)
{
    const int most = tpr >= 1024 ? 256 : tpr >= 256 ? 1024 : 256 * 4 * (256 / tpr);
    const int each = (rows + most - 1) / most;
    return each > 0 ? (rows + each - 1) / each : 0;
}
struct BwdShape { int tpr, p; };
static BwdShape bwd_shape(int cols, int v)
{
    const int n = (cols + v - 1) / v;
    if (n <= 64) return {64, 1};
    if (n <= 128) return {64, 2};
    if (n <= 512) return {256, n <= 256 ? 1 : 2};
    if (n <= 1024) return {256, 4};
    return {1024, n <= 2048 ? 2 : n <= 4096 ? 4 : 8};
}
constexpr int kNormMaxCols = 32768;

template <class T, bool RES, bool BIG> static void launch_bwd_as(const Q8NormBwdParams &p, const BwdShape &f, hipStream_t s)
{
    auto go = [&](auto kernel) {
        const int threads = f.tpr > 256 ? f.tpr : 256, spw = threads / f.tpr;
        hipLaunchKernelGGL(kernel, dim3((unsigned)((p.strips + spw - 1) / spw)), dim3(threads), 0, s, p);
    };
    if (f.tpr == 64) { if (f.p == 1) go(rmsnorm_bwd_kernel<T, RES, 64, 1, BIG>); else go(rmsnorm_bwd_kernel<T, RES, 64, 2, BIG>); }
    else if (f.tpr == 256) {
        if (f.p == 1) go(rmsnorm_bwd_kernel<T, RES, 256, 1, BIG>);
        else if (f.p == 2) go(rmsnorm_bwd_kernel<T, RES, 256, 2, BIG>);
        else go(rmsnorm_bwd_kernel<T, RES, 256, 4, BIG>);
    } else {
        if (f.p == 2) go(rmsnorm_bwd_kernel<T, RES, 1024, 2, BIG>);
        else if (f.p == 4) go(rmsnorm_bwd_kernel<T, RES, 1024, 4, BIG>);
        else if constexpr (Piece<T>::V == 4) go(rmsnorm_bwd_kernel<T, RES, 1024, 8, BIG>);      // (16384 fp32 values and more)
    }
}

template <class T, bool RES> static void launch_bwd(const Q8NormBwdParams &p, const BwdShape &f, hipStream_t s)
{
    if (big<T>(p.rows, p.cols)) launch_bwd_as<T, RES, true>(p, f, s);
    else launch_bwd_as<T, RES, false>(p, f, s);
}

static owt_status check_rows(int rows, int cols, owt_dtype dtype)
{
    if (rows < 0 || cols <= 0) return fail(OWT_EINVAL, "rows must not be negative, cols must be positive");
    if (dtype != OWT_F32 && dtype != OWT_BF16) return fail(OWT_EINVAL, "unknown dtype %d", (int)dtype);
    if (cols > 0x7fffff00) return fail(OWT_EUNSUPPORTED, "rows of more than 2^31-256 values");
    return OWT_OK;
}
static owt_status check_pointers(std::initializer_list<const void *> required, std::initializer_list<const void *> optional)
{
    for (const void *p : required)
        if (!p) return fail(OWT_EINVAL, "a required pointer is NULL");
    for (const auto &l : {required, optional})
        for (const void *p : l)
            if (!aligned16(p)) return fail(OWT_EINVAL, "pointers must be 16-byte aligned");
    return OWT_OK;
}
static owt_status launched()
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? OWT_OK : fail(OWT_ELAUNCH, "HIP launch failed: %s", hipGetErrorString(e));
}

}  // namespace owt

using namespace owt;
#define OWT_TRY(e) do { const owt_status st_ = (e); if (st_ != OWT_OK) return st_; } while (0)

extern "C" {

size_t owt_q8_pitch(int cols) { return cols > 0 ? q8_pitch(cols) : 0; }

owt_status owt_q8_pack(int rows, int cols, owt_dtype dtype, const void *x, signed char *q, float *scale, void *hip_stream)
{
    OWT_TRY(check_rows(rows, cols, dtype));
    if (rows == 0) return OWT_OK;
    OWT_TRY(check_pointers({x, q, scale}, {}));
    Q8RowParams p{x, nullptr, nullptr, nullptr, q, scale, nullptr, rows, cols, q8_pitch(cols), 0.f};
    if (dtype == OWT_F32) launch_rows<float, false, false>(p, (hipStream_t)hip_stream);
    else launch_rows<bf16_t, false, false>(p, (hipStream_t)hip_stream);
    return launched();
}

owt_status owt_q8_unpack(int rows, int cols, owt_dtype dtype, const signed char *q, const float *scale, void *x, void *hip_stream)
{
    OWT_TRY(check_rows(rows, cols, dtype));
    if (rows == 0) return OWT_OK;
    OWT_TRY(check_pointers({x, q, scale}, {}));
    if (dtype == OWT_F32) launch_unpack<float>(q, scale, x, rows, cols, (hipStream_t)hip_stream);
    else launch_unpack<bf16_t>(q, scale, x, rows, cols, (hipStream_t)hip_stream);
    return launched();
}

owt_status owt_rmsnorm_q8_fwd(int rows, int cols, owt_dtype dtype, const void *x, const void *res_or_null, const float *gain_or_null, float eps,
                              void *h_or_null, signed char *q, float *scale, float *rstd_or_null, void *hip_stream)
{
    OWT_TRY(check_rows(rows, cols, dtype));
    if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(OWT_EINVAL, "eps must be finite and not negative");
    if (cols > kNormMaxCols) return fail(OWT_EUNSUPPORTED, "norm over more than %d values", kNormMaxCols);
    if (rows == 0) return OWT_OK;
    OWT_TRY(check_pointers({x, q, scale}, {res_or_null, gain_or_null, h_or_null, rstd_or_null}));
    if (h_or_null && !res_or_null) return fail(OWT_EINVAL, "h is written only where there is a residual: without one it is x");
    Q8RowParams p{x, res_or_null, gain_or_null, h_or_null, q, scale, rstd_or_null, rows, cols, q8_pitch(cols), eps};
    hipStream_t s = (hipStream_t)hip_stream;
    if (dtype == OWT_F32) { if (res_or_null) launch_rows<float, true, true>(p, s); else launch_rows<float, true, false>(p, s); }
    else { if (res_or_null) launch_rows<bf16_t, true, true>(p, s); else launch_rows<bf16_t, true, false>(p, s); }
    return launched();
}

size_t owt_rmsnorm_q8_workspace_bytes(int rows, int cols)
{
    if (check_rows(rows, cols, OWT_F32) != OWT_OK) return (size_t)-1;
    if (cols > kNormMaxCols) { fail(OWT_EUNSUPPORTED, "norm over more than %d values", kNormMaxCols); return (size_t)-1; }
    size_t most = 0;                    // of both storage types: a program may size its scratch before it knows
    for (int v : {4, 8}) {
        const size_t n = (size_t)bwd_strips(rows, bwd_shape(cols, v).tpr) * cols * sizeof(float);
        most = n > most ? n : most;
    }
    return most;
}

owt_status owt_rmsnorm_q8_bwd(int rows, int cols, owt_dtype dtype, const void *dy, const void *h, const float *gain_or_null, const float *rstd,
                              const void *dres_or_null, float alpha, float beta, void *dh, float *dgain_or_null, void *ws, size_t ws_bytes,
                              void *hip_stream)
{
    OWT_TRY(check_rows(rows, cols, dtype));
    if (!std::isfinite(alpha) || !std::isfinite(beta)) return fail(OWT_EINVAL, "alpha and beta must be finite");
    if (cols > kNormMaxCols) return fail(OWT_EUNSUPPORTED, "norm over more than %d values", kNormMaxCols);
    if (rows > 0) OWT_TRY(check_pointers({dy, h, rstd, dh}, {gain_or_null, dres_or_null}));
    OWT_TRY(check_pointers({}, {dgain_or_null}));
    const BwdShape f = bwd_shape(cols, dtype == OWT_F32 ? 4 : 8);
    const int strips = bwd_strips(rows, f.tpr);
    if (dgain_or_null) {
        const size_t need = (size_t)strips * cols * sizeof(float);
        if (ws_bytes < need) return fail(OWT_EWORKSPACE, "workspace too small: need %zu bytes, got %zu", need, ws_bytes);
        if (need && (!ws || !aligned16(ws))) return fail(OWT_EINVAL, "ws is NULL or misaligned");
    }
    hipStream_t s = (hipStream_t)hip_stream;
    if (rows > 0) {
        Q8NormBwdParams p{dy, h, dres_or_null, gain_or_null, rstd, dh, dgain_or_null ? (float *)ws : nullptr, rows, cols, strips};
        if (dtype == OWT_F32) { if (dres_or_null) launch_bwd<float, true>(p, f, s); else launch_bwd<float, false>(p, f, s); }
        else { if (dres_or_null) launch_bwd<bf16_t, true>(p, f, s); else launch_bwd<bf16_t, false>(p, f, s); }
        OWT_TRY(launched());
    }
    if (dgain_or_null) {
        hipLaunchKernelGGL(rmsnorm_dgain_kernel, dim3((cols + 15) / 16), dim3(256), 0, s, (const float *)ws, dgain_or_null, cols, strips, alpha, beta);
        OWT_TRY(launched());
    }
    return OWT_OK;
}

}  // extern "C"

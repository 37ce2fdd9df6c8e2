// Softmax cross-entropy on a dense shard's outputs, without the outputs: entry points, and kernels that are right for every size.
//
//   z[n][o] = bias[o] + sum_i x[n][i] w[o][i],   lse[n] = log sum_o exp z[n][o]
//   dz[n][o] = weight[n] (exp(z[n][o] - lse[n]) - [o is n's label]),   dx = dz w,   dw = alpha dz^T x + beta dw,   dbias likewise
//
// The classes are taken in pieces whose outputs fit the scratch; of a piece there is left the largest output and the sum of exponentials
// below it for each row (forward), or its part of dx and its rows of dw (backward, which computes the outputs again).
#include <cmath>

#include "owt_host.hpp"

namespace owt {

constexpr int kPiece = 4096;            // classes of a piece

struct SimpleProduct {
    const void *a, *b;                  // A[m][k] at m am + k ak, B[c][k] at c bc + k bk
    long am, ak, bc, bk;
    const int *rows;                    // labels of the rows that k counts: B is zero where there is none (may be null)
    int classes;
    int M, N;
    long K;
    const float *bias;                  // of columns, or null
    float alpha, beta;
    void *out;
    long ldo;
};

__device__ __forceinline__ bool has_class(int label, int classes) { return (unsigned)label < (unsigned)classes; }

// 64 x 64 results a work-group, 4 x 4 a thread, 16 of k a step
template <class TA, class TB, class TO>
__global__ void __launch_bounds__(256) simple_product_kernel(const SimpleProduct p)
{
    __shared__ float as[16][65], bs[16][65];
    const int tid = threadIdx.x, tm = tid / 16, tc = tid % 16;
    const int m0 = blockIdx.y * 64, c0 = blockIdx.x * 64;
    float acc[4][4] = {};
    for (long k0 = 0; k0 < p.K; k0 += 16) {
        for (int e = tid; e < 1024; e += 256) {
            const bool across = p.ak != 1;
            const int r = across ? e % 64 : e / 16, k = across ? e / 64 : e % 16;
            const long kk = k0 + k;
            as[k][r] = m0 + r < p.M && kk < p.K ? load1((const TA *)p.a + (m0 + r) * p.am + kk * p.ak, 0) : 0.f;
        }
        for (int e = tid; e < 1024; e += 256) {
            const bool across = p.bk != 1;
            const int r = across ? e % 64 : e / 16, k = across ? e / 64 : e % 16;
            const long kk = k0 + k;
            bs[k][r] = c0 + r < p.N && kk < p.K && (!p.rows || has_class(p.rows[kk], p.classes)) ? load1((const TB *)p.b + (c0 + r) * p.bc + kk * p.bk, 0) : 0.f;
        }
        __syncthreads();
        for (int k = 0; k < 16; k++)
#pragma unroll
            for (int i = 0; i < 4; i++)
#pragma unroll
                for (int j = 0; j < 4; j++) acc[i][j] = fmaf(as[k][tm * 4 + i], bs[k][tc * 4 + j], acc[i][j]);
        __syncthreads();
    }
    for (int i = 0; i < 4; i++)
        for (int j = 0; j < 4; j++) {
            const int m = m0 + tm * 4 + i, c = c0 + tc * 4 + j;
            if (m >= p.M || c >= p.N) continue;
            float v = p.alpha * acc[i][j];
            if (p.bias) v += p.bias[c];
            TO *to = (TO *)p.out + m * p.ldo + c;
            if (p.beta != 0.f) v += p.beta * load1(to, 0);
            store1(to, 0, v);
        }
}

// The largest output of a row and the sum of exponentials below it, joined with another such pair.  A pair without outputs is (-inf, 0); outputs
// of -inf add nothing; +inf and NaN leave as infinity and NaN.
struct Top { float max, sum; };
__device__ __forceinline__ Top top_of(float v) { return {v == v ? v : 0.f, v == -INFINITY ? 0.f : v == INFINITY || v != v ? v : 1.f}; }
__device__ __forceinline__ Top join(Top a, Top b)
{
    const float m = fmaxf(a.max, b.max), at = __builtin_isfinite(m) ? m : 0.f;
    return {m, a.sum * (a.max == m ? 1.f : expf(a.max - at)) + b.sum * (b.max == m ? 1.f : expf(b.max - at))};
}

// One wavefront a row: row n's pair over these columns, joined with what pieces before left, and the label's output.
__global__ void __launch_bounds__(256) piece_top_kernel(const float *z, int N, int cols, int off, const int *labels, int classes, bool first, Top *top,
                                                        float *target)
{
    const int n = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (n >= N) return;
    Top t = {-INFINITY, 0.f};
    for (int j = lane; j < cols; j += 64) {
        t = join(t, top_of(z[(size_t)n * cols + j]));
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) t = join(t, {__shfl_xor(t.max, d, 64), __shfl_xor(t.sum, d, 64)});
    if (lane == 0) {
        top[n] = first ? t : join(top[n], t);
        const int j = labels ? labels[n] - off : -1;
        if (target) {
            if (first) target[n] = -INFINITY;
            if (labels && has_class(labels[n], classes) && j >= 0 && j < cols) target[n] = z[(size_t)n * cols + j];
        }
    }
}

__device__ __forceinline__ float loss_of(float lse, float target) { return target == -INFINITY ? INFINITY : lse - target; }

__global__ void __launch_bounds__(256) lse_kernel(int N, const Top *top, const int *labels, int classes, float *lse, float *target, float *loss)
{
    const int n = blockIdx.x * 256 + threadIdx.x;
    if (n >= N) return;
    const Top t = top[n];
    float l = (__builtin_isfinite(t.max) ? t.max : 0.f) + logf(t.sum);
    if (labels && !has_class(labels[n], classes)) {
        l = 0.f;
        if (target) target[n] = 0.f;
        if (loss) loss[n] = 0.f;
    } else if (loss) loss[n] = loss_of(l, target[n]);
    lse[n] = l;
}

// outputs to their gradients, in place
__global__ void __launch_bounds__(256) piece_dz_kernel(float *z, int N, int cols, int off, const int *labels, int classes, const float *lse, const float *weight)
{
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (size_t)N * cols) return;
    const int n = (int)(i / cols), j = (int)(i % cols), label = labels[n];
    const float l = lse[n], v = z[i], p = v == -INFINITY ? 0.f : expf(v - l);
    z[i] = has_class(label, classes) ? (weight ? weight[n] : 1.f) * (p - (j == label - off ? 1.f : 0.f)) : 0.f;
}
__global__ void __launch_bounds__(256) piece_dbias_kernel(const float *dz, int N, int cols, float alpha, float beta, float *db)
{
    const int j = blockIdx.x * 256 + threadIdx.x;
    if (j >= cols) return;
    float s = 0.f;
    for (int n = 0; n < N; n++) s += dz[(size_t)n * cols + j];
    db[j] = alpha * s + (beta != 0.f ? beta * db[j] : 0.f);
}
template <class T> __global__ void __launch_bounds__(256) store_rows_kernel(const float *from, size_t n, int cols, const int *labels, int classes, T *to)
{
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i < n) store1(to, i, has_class(labels[i / cols], classes) ? from[i] : 0.f);
}

// Joins the shards' shares: lse and target of `workers` shards, worker by worker.
__global__ void __launch_bounds__(256) softmax_join_kernel(int workers, int N, int classes, const float *lses, const float *targets, const int *labels,
                                                           float *lse, float *target, float *loss)
{
    const int n = blockIdx.x * 256 + threadIdx.x;
    if (n >= N) return;
    if (!has_class(labels[n], classes)) {
        lse[n] = 0.f;
        if (target) target[n] = 0.f;
        if (loss) loss[n] = 0.f;
        return;
    }
    Top t = {-INFINITY, 0.f};
    float at = -INFINITY;
    for (int k = 0; k < workers; k++) {
        t = join(t, top_of(lses[(size_t)k * N + n]));
        at = __builtin_elementwise_maximum(at, targets[(size_t)k * N + n]);
    }
    const float l = (__builtin_isfinite(t.max) ? t.max : 0.f) + logf(t.sum);
    lse[n] = l;
    if (target) target[n] = at;
    if (loss) loss[n] = loss_of(l, at);
}

// ------------------------------------------------------------------------------------------------ host

constexpr int kMaxRows = 1 << 22;       // of x and of w

static owt_status check_softmax(const owt_fc_desc *d, int &o_local)
{
    if (!d) return fail(OWT_EINVAL, "descriptor is NULL");
    if (d->N < 0 || d->I <= 0 || d->O_total <= 0 || d->workers <= 0)
        return fail(OWT_EINVAL, "N must not be negative; I, O_total and workers must be positive");
    if (d->rank < 0 || d->rank >= d->workers) return fail(OWT_EINVAL, "need 0 <= rank < workers");
    if (d->O_total % d->workers) return fail(OWT_EINVAL, "O_total must be divisible by workers");
    if (d->dtype != OWT_F32 && d->dtype != OWT_BF16) return fail(OWT_EINVAL, "unknown dtype %d", (int)d->dtype);
    if (d->flags & ~(unsigned)OWT_BIAS) return fail(OWT_EINVAL, "flags other than OWT_BIAS (0x%x) have no meaning here", d->flags);
    o_local = d->O_total / d->workers;
    if (d->N > kMaxRows || o_local > kMaxRows) return fail(OWT_EUNSUPPORTED, "more than 2^22 rows or columns");
    if ((long)d->N * d->I > 0x7fffffffL || (long)o_local * d->I > 0x7fffffffL) return fail(OWT_EUNSUPPORTED, "more than 2^31-1 elements");
    return OWT_OK;
}
static owt_status need_ptr(const void *p, const char *what)
{
    if (!p) return fail(OWT_EINVAL, "%s is NULL", what);
    return aligned16(p) ? OWT_OK : fail(OWT_EINVAL, "%s is not 16-byte aligned", what);
}
static owt_status may_ptr(const void *p, const char *what) { return aligned16(p) ? OWT_OK : fail(OWT_EINVAL, "%s is not 16-byte aligned", what); }
static owt_status need_ws(const void *ws, size_t have, size_t need)
{
    if (have < need) return fail(OWT_EWORKSPACE, "workspace too small: need %zu bytes, got %zu", need, have);
    if (need && (!ws || !aligned16(ws))) return fail(OWT_EINVAL, "ws is NULL or misaligned");
    return OWT_OK;
}
static owt_status launched()
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? OWT_OK : fail(OWT_ELAUNCH, "HIP launch failed: %s", hipGetErrorString(e));
}

struct SoftmaxLayout {
    size_t z, top, dx, total;
    SoftmaxLayout(const owt_fc_desc *d, int ol, bool forward)
    {
        size_t at = 0;
        auto take = [&](size_t bytes) { const size_t was = at; at += (bytes + 255) / 256 * 256; return was; };
        z = take((size_t)d->N * (ol < kPiece ? ol : kPiece) * 4);
        top = take(forward ? (size_t)d->N * 12 : 0);
        dx = take(!forward ? (size_t)d->N * d->I * 4 : 0);
        total = d->N ? at : 0;
    }
};

template <class TA, class TB, class TO> static void product(const SimpleProduct &p, hipStream_t s)
{
    const dim3 grid((unsigned)((p.N + 63) / 64), (unsigned)((p.M + 63) / 64));
    hipLaunchKernelGGL((simple_product_kernel<TA, TB, TO>), grid, dim3(256), 0, s, p);
}
static unsigned groups_of(size_t n) { return (unsigned)((n + 255) / 256); }

// outputs of classes [v0, v0 + cols)
template <class T> static void outputs(const owt_fc_desc *d, const void *x, const void *w, const float *bias, int v0, int cols, float *z, hipStream_t s)
{
    const SimpleProduct p = {x, (const T *)w + (size_t)v0 * d->I, d->I, 1, d->I, 1, nullptr, 0, d->N, cols, d->I, bias ? bias + v0 : nullptr, 1.f, 0.f, z, cols};
    product<T, T, float>(p, s);
}

template <class T>
static owt_status forward(const owt_fc_desc *d, int ol, const void *x, const void *w, const float *bias, const int *labels, float *lse, float *target,
                          float *loss, char *ws, hipStream_t s)
{
    const SoftmaxLayout l(d, ol, true);
    float *z = (float *)(ws + l.z), *at = target ? target : (float *)(ws + l.top) + 2 * (size_t)d->N;
    Top *top = (Top *)(ws + l.top);
    for (int v0 = 0; v0 < ol; v0 += kPiece) {
        const int cols = ol - v0 < kPiece ? ol - v0 : kPiece;
        outputs<T>(d, x, w, bias, v0, cols, z, s);
        hipLaunchKernelGGL(piece_top_kernel, dim3((unsigned)((d->N + 3) / 4)), dim3(256), 0, s, z, d->N, cols, d->rank * ol + v0, labels, d->O_total, v0 == 0,
                           top, at);
    }
    hipLaunchKernelGGL(lse_kernel, dim3(groups_of(d->N)), dim3(256), 0, s, d->N, top, labels, d->O_total, lse, at, loss);
    return launched();
}

template <class T>
static owt_status backward(const owt_fc_desc *d, int ol, const void *x, const void *w, const float *bias, const int *labels, const float *lse,
                           const float *weight, float alpha, float beta, void *dx, float *dw, float *db, char *ws, hipStream_t s)
{
    const SoftmaxLayout l(d, ol, false);
    float *z = (float *)(ws + l.z), *dxs = (float *)(ws + l.dx);
    for (int v0 = 0; v0 < ol; v0 += kPiece) {
        const int cols = ol - v0 < kPiece ? ol - v0 : kPiece;
        if (d->N) {
            outputs<T>(d, x, w, bias, v0, cols, z, s);
            hipLaunchKernelGGL(piece_dz_kernel, dim3(groups_of((size_t)d->N * cols)), dim3(256), 0, s, z, d->N, cols, d->rank * ol + v0, labels, d->O_total, lse, weight);
        }
        if (dx && d->N)
            product<float, T, float>({z, (const T *)w + (size_t)v0 * d->I, cols, 1, 1, d->I, nullptr, 0, d->N, d->I, cols, nullptr, 1.f, v0 ? 1.f : 0.f, dxs, d->I}, s);
        product<float, T, float>({z, x, 1, cols, 1, d->I, labels, d->O_total, cols, d->I, d->N, nullptr, alpha, beta, dw + (size_t)v0 * d->I, d->I}, s);
        if (db) hipLaunchKernelGGL(piece_dbias_kernel, dim3(groups_of(cols)), dim3(256), 0, s, z, d->N, cols, alpha, beta, db + v0);
    }
    if (dx && d->N) {
        const size_t n = (size_t)d->N * d->I;
        hipLaunchKernelGGL(store_rows_kernel<T>, dim3(groups_of(n)), dim3(256), 0, s, dxs, n, d->I, labels, d->O_total, (T *)dx);
    }
    return launched();
}

}  // namespace owt

using namespace owt;
#define OWT_TRY(e) do { const owt_status st_ = (e); if (st_ != OWT_OK) return st_; } while (0)

extern "C" {

size_t owt_fc_softmax_workspace_bytes(const owt_fc_desc *d, int pass)
{
    int ol;
    if (pass < 0 || pass > 2) { fail(OWT_EINVAL, "pass must be 0, 1 or 2"); return (size_t)-1; }
    if (check_softmax(d, ol) != OWT_OK) return (size_t)-1;
    return SoftmaxLayout(d, ol, pass == OWT_PASS_FWD).total;
}

owt_status owt_fc_softmax_fwd(const owt_fc_desc *d, const void *x, const void *w, const float *bias, const int *labels_or_null, float *lse,
                              float *target_or_null, float *loss_or_null, void *ws, size_t ws_bytes, void *hip_stream)
{
    int ol;
    OWT_TRY(check_softmax(d, ol));
    if (!labels_or_null && (target_or_null || loss_or_null)) return fail(OWT_EINVAL, "target and loss need labels");
    if (loss_or_null && d->workers != 1) return fail(OWT_EINVAL, "a shard of several has no loss of its own: owt_softmax_join gives it");
    if (d->N == 0) return OWT_OK;
    OWT_TRY(need_ptr(x, "x")); OWT_TRY(need_ptr(w, "w")); OWT_TRY(need_ptr(lse, "lse"));
    if (d->flags & OWT_BIAS) OWT_TRY(need_ptr(bias, "bias"));
    OWT_TRY(may_ptr(labels_or_null, "labels")); OWT_TRY(may_ptr(target_or_null, "target")); OWT_TRY(may_ptr(loss_or_null, "loss"));
    OWT_TRY(need_ws(ws, ws_bytes, SoftmaxLayout(d, ol, true).total));
    const float *b = (d->flags & OWT_BIAS) ? bias : nullptr;
    hipStream_t s = (hipStream_t)hip_stream;
    if (d->dtype == OWT_BF16) return forward<bf16_t>(d, ol, x, w, b, labels_or_null, lse, target_or_null, loss_or_null, (char *)ws, s);
    return forward<float>(d, ol, x, w, b, labels_or_null, lse, target_or_null, loss_or_null, (char *)ws, s);
}

owt_status owt_softmax_join(int workers, int N, int classes, const float *lses, const float *targets, const int *labels, float *lse,
                            float *target_or_null, float *loss_or_null, void *hip_stream)
{
    if (workers <= 0 || N < 0 || classes <= 0) return fail(OWT_EINVAL, "workers and classes must be positive, N not negative");
    if (N == 0) return OWT_OK;
    OWT_TRY(need_ptr(lses, "lses")); OWT_TRY(need_ptr(targets, "targets")); OWT_TRY(need_ptr(labels, "labels")); OWT_TRY(need_ptr(lse, "lse"));
    OWT_TRY(may_ptr(target_or_null, "target")); OWT_TRY(may_ptr(loss_or_null, "loss"));
    hipLaunchKernelGGL(softmax_join_kernel, dim3(groups_of(N)), dim3(256), 0, (hipStream_t)hip_stream, workers, N, classes, lses, targets, labels, lse,
                       target_or_null, loss_or_null);
    return launched();
}

owt_status owt_fc_softmax_bwd(const owt_fc_desc *d, const void *x, const void *w, const float *bias, const int *labels, const float *lse,
                              const float *weight_or_null, float alpha, float beta, void *dx_partial_or_null, float *dw, float *dbias_or_null, void *ws,
                              size_t ws_bytes, void *hip_stream)
{
    int ol;
    OWT_TRY(check_softmax(d, ol));
    if (!std::isfinite(alpha) || !std::isfinite(beta)) return fail(OWT_EINVAL, "alpha and beta must be finite");
    OWT_TRY(need_ptr(dw, "dw")); OWT_TRY(may_ptr(dx_partial_or_null, "dx_partial")); OWT_TRY(may_ptr(dbias_or_null, "dbias"));
    if (d->N > 0) {
        OWT_TRY(need_ptr(x, "x")); OWT_TRY(need_ptr(w, "w")); OWT_TRY(need_ptr(labels, "labels")); OWT_TRY(need_ptr(lse, "lse"));
        if (d->flags & OWT_BIAS) OWT_TRY(need_ptr(bias, "bias"));
        OWT_TRY(may_ptr(weight_or_null, "weight"));
    }
    OWT_TRY(need_ws(ws, ws_bytes, SoftmaxLayout(d, ol, false).total));
    const float *b = (d->flags & OWT_BIAS) ? bias : nullptr;
    hipStream_t s = (hipStream_t)hip_stream;
    if (d->dtype == OWT_BF16)
        return backward<bf16_t>(d, ol, x, w, b, labels, lse, weight_or_null, alpha, beta, dx_partial_or_null, dw, dbias_or_null, (char *)ws, s);
    return backward<float>(d, ol, x, w, b, labels, lse, weight_or_null, alpha, beta, dx_partial_or_null, dw, dbias_or_null, (char *)ws, s);
}

}  // extern "C"

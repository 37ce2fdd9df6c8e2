// The norm of the gradients of many tensors together, and what is done with it: the gradients times the factor that brings the norm down to a
// bound, or the momentum / weight-decay update of Section 5 with the bounded gradients.  All three are HBM-bound passes over lists of tensors.
//
// A list is cut into chunks of 16 KB that end with their tensor; a work-group walks a run of consecutive chunks, 16 bytes an access.  Pointers
// and sizes of up to kSet tensors travel in a launch's arguments (so that a captured launch holds them, and nothing is allocated); longer lists
// take several launches.
//
// us, and TB/s of what is read and written: six blocks 2048 / 8192 in bf16 norm 86 and clip 195 (5.6 over both), eight in fp32 norm 223 and update 1130 (5.1), 123 tensors of
// 12.8 M values norm and update 76 in all; a 2 GiB copy runs at 4.9.
#include <cmath>

#include "owt_host.hpp"

namespace owt {

constexpr int kClipGroups = 2048;       // eight work-groups of 256 threads a CU: all that run at a time
constexpr int kSet = 80;                // tensors of a launch (128 at most: walk_chunks): with four pointers each 3.6 KB of arguments
constexpr int kChunkBytes = 16384;      // of gradients: 64 bytes a thread
constexpr size_t kOneGroup = 4;         // so few chunks are one work-group's, and the launch that joins the sums is saved
constexpr size_t kPastChunks = 8192;    // a list of more than 128 MB is written past the caches

// P pointers for each tensor; chunks [first[t], first[t + 1]) are tensor t's, and its last one has last[t] values.  Work-group b has each + (b < more)
// chunks.  (All in 32 bits: compared in 64, the size that is left was taken for a whole chunk by the compiler's choice between the two.)
template <int P> struct TensorSet {
    void *at[P][kSet];
    unsigned first[kSet + 1], last[kSet];
    int count;
    unsigned each, more;
};

// f(t, from, values) for each chunk of this work-group's run, `chunk` values at most.  BACK: from the run's end to its beginning.  The norm walks forwards and
// leaves the ends of the runs in the 256 MB behind the L2 caches; who reads the gradients after it begins there.
template <bool BACK, int P, class F> __device__ __forceinline__ void walk_chunks(const TensorSet<P> &s, unsigned chunk, F f)
{
    const unsigned b = blockIdx.x, begin = b * s.each + min(b, s.more), end = begin + s.each + (b < s.more ? 1 : 0);
    // the tensor of the first chunk: how many begin there or before, counted by a wavefront at once (one after the other, or by halves, took 3 us a launch)
    const unsigned from = BACK ? end - 1 : begin, lane = threadIdx.x & 63;
    const unsigned a = lane < (unsigned)s.count ? s.first[lane] : ~0u, z = lane + 64 < (unsigned)s.count ? s.first[lane + 64] : ~0u;
    int t = __builtin_amdgcn_readfirstlane(__popcll(__ballot(a <= from)) + __popcll(__ballot(z <= from)) - 1);
    for (unsigned k = begin; k < end; k++) {
        const unsigned c = BACK ? end - 1 - (k - begin) : k;
        if (BACK)
            while (c < s.first[t]) t--;
        else
            while (c >= s.first[t + 1]) t++;
        const unsigned n = c + 1 == s.first[t + 1] ? s.last[t] : chunk;
        f(t, (size_t)(c - s.first[t]) * chunk, n);
    }
}
// 16 and 8 bytes; PAST: by the caches, where there is more than they hold
typedef unsigned clip_u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned clip_u32x2 __attribute__((ext_vector_type(2)));
template <bool PAST> __device__ __forceinline__ void put(void *to, const uint4 &v)
{
    const clip_u32x4 u = {v.x, v.y, v.z, v.w};
    if (PAST) __builtin_nontemporal_store(u, (clip_u32x4 *)to);
    else *(clip_u32x4 *)to = u;
}
template <bool PAST> __device__ __forceinline__ void put(void *to, const uint2 &v)
{
    const clip_u32x2 u = {v.x, v.y};
    if (PAST) __builtin_nontemporal_store(u, (clip_u32x2 *)to);
    else *(clip_u32x2 *)to = u;
}
template <bool PAST> __device__ __forceinline__ void put(void *to, const float4 &v)
{
    put<PAST>(to, make_uint4(__float_as_uint(v.x), __float_as_uint(v.y), __float_as_uint(v.z), __float_as_uint(v.w)));
}

template <class T> constexpr int kPer = 16 / sizeof(T);             // values of an access
template <class T> __device__ __forceinline__ void widen(const uint4 &v, float (&f)[kPer<T>])
{
    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int k = 0; k < 4; k++) {
        if (sizeof(T) == 4) f[k] = __uint_as_float(u[k]);
        else {
            f[2 * k % kPer<T>] = __uint_as_float(u[k] << 16);
            f[(2 * k + 1) % kPer<T>] = __uint_as_float(u[k] & 0xffff0000u);
        }
    }
}
template <class T> __device__ __forceinline__ uint4 narrow(const float (&f)[kPer<T>])
{
    uint32_t u[4];
#pragma unroll
    for (int k = 0; k < 4; k++)
        u[k] = sizeof(T) == 4 ? __float_as_uint(f[k]) : f32x2_to_bf16x2(f[2 * k % kPer<T>], f[(2 * k + 1) % kPer<T>]);
    return make_uint4(u[0], u[1], u[2], u[3]);
}

// A work-group's sum in a fixed order: lanes in pairs, then wavefronts one by one.  The result is thread 0's.
template <int WAVES> __device__ __forceinline__ double group_sum(double v)
{
    __shared__ double part[WAVES];
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d, 64);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.;
    if (threadIdx.x == 0)
        for (int w = 0; w < WAVES; w++) v += part[w];
    return v;
}

// sqrt of the sum of g^2.  Squares are summed in 64 bits: no gradient that fp32 holds overflows or vanishes in them, and the sum is as exact as its result's 32 bits
// whatever the number of values.  (An instruction of 64 bits a value is half the fp32 rate, twenty times what memory brings.)
template <class T, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) grad_square_kernel(const TensorSet<1> s, double *partial, float *norm)
{
    constexpr int V = kPer<T>, CH = kChunkBytes / sizeof(T), U = CH / (V * 64 * WAVES);
    double sum[4] = {0., 0., 0., 0.};
    auto add = [&](const uint4 &v) __attribute__((always_inline)) {
        float f[V];
        widen<T>(v, f);
#pragma unroll
        for (int k = 0; k < V; k++) sum[k & 3] = fma((double)f[k], (double)f[k], sum[k & 3]);
    };
    walk_chunks<false>(s, CH, [&](int t, size_t from, unsigned n) __attribute__((always_inline)) {
        const T *g = (const T *)s.at[0][t] + from;
        if (n == CH) {
            uint4 v[U];
#pragma unroll
            for (int u = 0; u < U; u++) v[u] = ((const uint4 *)g)[threadIdx.x + 64 * WAVES * u];
#pragma unroll
            for (int u = 0; u < U; u++) add(v[u]);
        } else {
            for (unsigned i = threadIdx.x; i < n / V; i += 64 * WAVES) add(((const uint4 *)g)[i]);
            const unsigned i = n / V * V + threadIdx.x;
            if (i < n) {
                const double x = load1(g, (int)i);
                sum[0] = fma(x, x, sum[0]);
            }
        }
    });
    const double all = group_sum<WAVES>((sum[0] + sum[1]) + (sum[2] + sum[3]));
    if (threadIdx.x == 0) {
        if (norm) *norm = (float)sqrt(all);         // the only work-group of the only launch
        else partial[blockIdx.x] = all;
    }
}

__global__ void __launch_bounds__(1024) grad_norm_join_kernel(const double *partial, int n, float *norm)
{
    double v = 0.;
    for (int i = threadIdx.x; i < n; i += 1024) v += partial[i];
    v = group_sum<16>(v);
    if (threadIdx.x == 0) *norm = (float)sqrt(v);
}

// g times a factor is ((g * first) * second) * last.  A factor below 2^-100 (a bound of 0.001 on a norm of 1e30 is 2^-110) loses bits where fp32 has no normal number for it, though
// what comes of a large g has all of its own: it goes in three parts then, of which only the last product may leave fp32's normal numbers.
struct Factor { float first, second, last; };
__device__ __forceinline__ Factor factor_of(double f)
{
    if (fabs(f) >= 0x1p-100) return {1.f, 1.f, (float)f};
    return {0x1p-75f, (float)(f * 0x1p150), 0x1p-75f};
}

// out = g * min(1, max / norm); zeros where the norm is not finite.  Gradients that stay as they are and where they are are not touched.
template <class T, bool PAST>
__global__ void __launch_bounds__(256) grad_clip_kernel(const TensorSet<2> s, const float *norm, float max_norm)
{
    constexpr int V = kPer<T>, CH = kChunkBytes / sizeof(T), U = CH / (V * 256);
    const float all = *norm;
    const bool fine = __builtin_isfinite(all);
    const double bounded = (double)max_norm / (double)all;
    const bool whole = !(bounded < 1.);                     // (0 / 0 is no bound, either)
    const Factor factor = factor_of(whole ? 1. : bounded);
    auto scaled = [&](const uint4 &v) __attribute__((always_inline)) {
        float f[V];
        widen<T>(v, f);
#pragma unroll
        for (int k = 0; k < V; k++) f[k] = fine ? f[k] * factor.first * factor.second * factor.last : 0.f;
        return narrow<T>(f);
    };
    walk_chunks<true>(s, CH, [&](int t, size_t from, unsigned n) __attribute__((always_inline)) {
        const T *g = (const T *)s.at[0][t] + from;
        T *out = (T *)s.at[1][t] + from;
        if (fine && whole && g == out) return;
        if (n == CH) {
            uint4 v[U];
#pragma unroll
            for (int u = 0; u < U; u++) v[u] = ((const uint4 *)g)[threadIdx.x + 256 * u];
#pragma unroll
            for (int u = 0; u < U; u++) put<PAST>((uint4 *)out + threadIdx.x + 256 * u, scaled(v[u]));
        } else {
            for (unsigned i = threadIdx.x; i < n / V; i += 256) ((uint4 *)out)[i] = scaled(((const uint4 *)g)[i]);
            const unsigned i = n / V * V + threadIdx.x;
            if (i < n) store1(out, i, fine ? load1(g, (int)i) * factor.first * factor.second * factor.last : 0.f);
        }
    });
}

// vel := mu*vel + eps*(gscale*factor*g - omega*w);  w := w + vel;  factor = min(1, max / (|gscale| norm)).  A norm that is not finite: no step.
template <bool COPY, bool PAST>
__global__ void __launch_bounds__(256) sgd_clipped_kernel(const TensorSet<3 + COPY> s, float mu, float eps, float omega, float gscale,
                                                          const float *norm, float max_norm)
{
    constexpr int CH = kChunkBytes / 4, U = CH / 1024;
    const float all = *norm;
    if (!__builtin_isfinite(all)) return;
    const double bounded = (double)max_norm / ((double)fabsf(gscale) * (double)all);        // (0 / 0 is no bound, either)
    const Factor scale = bounded < 1. ? factor_of(gscale * bounded) : Factor{1.f, 1.f, gscale};
    auto upd = [&](float &wv, float &vv, float gv) __attribute__((always_inline)) {
        vv = fmaf(mu, vv, eps * fmaf(scale.last, gv * scale.first * scale.second, -omega * wv));
        wv += vv;
    };
    walk_chunks<true>(s, CH, [&](int t, size_t from, unsigned n) __attribute__((always_inline)) {
        float *w = (float *)s.at[0][t] + from, *vel = (float *)s.at[1][t] + from;
        const float *g = (const float *)s.at[2][t] + from;
        uint16_t *wb = COPY ? (uint16_t *)s.at[2 + COPY][t] + from : nullptr;
        auto step = [&](unsigned i, float4 a, float4 v, const float4 &d) __attribute__((always_inline)) {
            upd(a.x, v.x, d.x); upd(a.y, v.y, d.y); upd(a.z, v.z, d.z); upd(a.w, v.w, d.w);
            put<PAST>((float4 *)vel + i, v);
            put<PAST>((float4 *)w + i, a);
            if (COPY) put<PAST>((uint2 *)wb + i, make_uint2(f32x2_to_bf16x2(a.x, a.y), f32x2_to_bf16x2(a.z, a.w)));
        };
        if (n == CH) {
            float4 a[U], v[U], d[U];
#pragma unroll
            for (int u = 0; u < U; u++) {
                a[u] = ((const float4 *)w)[threadIdx.x + 256 * u];
                v[u] = ((const float4 *)vel)[threadIdx.x + 256 * u];
                d[u] = ((const float4 *)g)[threadIdx.x + 256 * u];
            }
#pragma unroll
            for (int u = 0; u < U; u++) step(threadIdx.x + 256 * u, a[u], v[u], d[u]);
        } else {
            for (unsigned i = threadIdx.x; i < n / 4; i += 256) step(i, ((const float4 *)w)[i], ((const float4 *)vel)[i], ((const float4 *)g)[i]);
            const unsigned i = n / 4 * 4 + threadIdx.x;
            if (i < n) {
                float a = w[i], v = vel[i];
                upd(a, v, g[i]);
                vel[i] = v; w[i] = a;
                if (COPY) wb[i] = f32_to_bf16(a);
            }
        }
    });
}

// ------------------------------------------------------------------------------------------------ host

static size_t chunks_of(size_t n, size_t chunk) { return n / chunk + (n % chunk != 0); }

// Sizes that a walk counts in 32 bits
static owt_status check_list(int count, const size_t *n, size_t &chunks, size_t chunk)
{
    if (count < 0) return fail(OWT_EINVAL, "count must not be negative");
    if (count > 0 && !n) return fail(OWT_EINVAL, "n is NULL");
    chunks = 0;
    for (int t = 0; t < count; t++) {
        if (n[t] > ((size_t)1 << 40)) return fail(OWT_EUNSUPPORTED, "tensor %d has more than 2^40 values", t);
        chunks += chunks_of(n[t], chunk);
        if (chunks > 0x7fffffffu) return fail(OWT_EUNSUPPORTED, "more than 2^31-1 chunks of 16 KB");
    }
    return OWT_OK;
}
static owt_status check_pointers(int count, const size_t *n, const void *const *p, const char *what)
{
    if (count > 0 && !p) return fail(OWT_EINVAL, "%s is NULL", what);
    for (int t = 0; t < count; t++)
        if (n[t]) {
            if (!p[t]) return fail(OWT_EINVAL, "%s[%d] is NULL", what, t);
            if (!aligned16(p[t])) return fail(OWT_EINVAL, "%s[%d] is not 16-byte aligned", what, t);
        }
    return OWT_OK;
}
static int values_of_chunk(owt_dtype dtype) { return kChunkBytes / (dtype == OWT_BF16 ? 2 : 4); }

// go(set, work-groups) for each kSet tensors that are not empty
template <int P, class F> static owt_status for_sets(int count, const size_t *n, const void *const *const (&at)[P], size_t chunk, F go)
{
    TensorSet<P> s;
    s.count = 0;
    s.first[0] = 0;
    for (int t = 0; t <= count; t++) {
        if (s.count == kSet || (t == count && s.count > 0)) {
            const unsigned chunks = s.first[s.count], groups = chunks < (unsigned)kClipGroups ? chunks : (unsigned)kClipGroups;
            s.each = chunks / groups;
            s.more = chunks % groups;
            go(s, groups);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return fail(OWT_ELAUNCH, "HIP launch failed: %s", hipGetErrorString(e));
            s.count = 0;
        }
        if (t == count || n[t] == 0) continue;
        for (int k = 0; k < P; k++) s.at[k][s.count] = const_cast<void *>(at[k][t]);
        s.last[s.count] = (unsigned)((n[t] - 1) % chunk) + 1;
        s.first[s.count + 1] = s.first[s.count] + (unsigned)chunks_of(n[t], chunk);
        s.count++;
    }
    return OWT_OK;
}
static size_t sets_of(int count, const size_t *n)
{
    size_t full = 0;
    for (int t = 0; t < count; t++) full += n[t] != 0;
    return (full + kSet - 1) / kSet;
}

}  // namespace owt

using namespace owt;
#define OWT_TRY(e) do { const owt_status st_ = (e); if (st_ != OWT_OK) return st_; } while (0)

extern "C" {

size_t owt_grad_norm_workspace_bytes(int count, const size_t *n)
{
    size_t chunks;
    if (check_list(count, n, chunks, values_of_chunk(OWT_F32)) != OWT_OK) return (size_t)-1;
    return sets_of(count, n) * kClipGroups * sizeof(double);
}

owt_status owt_grad_norm(int count, const size_t *n, const void *const *g, owt_dtype dtype, float *norm, void *ws, size_t ws_bytes, void *hip_stream)
{
    if (dtype != OWT_F32 && dtype != OWT_BF16) return fail(OWT_EINVAL, "unknown dtype %d", (int)dtype);
    const int chunk = values_of_chunk(dtype);
    size_t chunks;
    OWT_TRY(check_list(count, n, chunks, chunk));
    OWT_TRY(check_pointers(count, n, g, "g"));
    if (!norm || !aligned16(norm)) return fail(OWT_EINVAL, "norm is NULL or not 16-byte aligned");
    const size_t sets = sets_of(count, n), need = sets * kClipGroups * sizeof(double);
    if (ws_bytes < need) return fail(OWT_EWORKSPACE, "workspace too small: need %zu bytes, got %zu", need, ws_bytes);
    if (need && (!ws || !aligned16(ws))) return fail(OWT_EINVAL, "ws is NULL or misaligned");
    hipStream_t s = (hipStream_t)hip_stream;
    double *partial = (double *)ws;
    int parts = 0;
    const bool one = sets == 1 && chunks <= kOneGroup;
    OWT_TRY(for_sets<1>(count, n, {g}, chunk, [&](TensorSet<1> &set, unsigned groups) {
        if (one) {
            set.each = (unsigned)chunks;
            set.more = 0;
            groups = 1;
        }
        if (dtype == OWT_F32) hipLaunchKernelGGL((grad_square_kernel<float, 4>), dim3(groups), dim3(256), 0, s, set, partial + parts, one ? norm : nullptr);
        else hipLaunchKernelGGL((grad_square_kernel<bf16_t, 4>), dim3(groups), dim3(256), 0, s, set, partial + parts, one ? norm : nullptr);
        parts += (int)groups;
    }));
    if (one) return OWT_OK;
    hipLaunchKernelGGL(grad_norm_join_kernel, dim3(1), dim3(1024), 0, s, partial, parts, norm);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? OWT_OK : fail(OWT_ELAUNCH, "HIP launch failed: %s", hipGetErrorString(e));
}

static owt_status check_bound(const float *norm, float max_norm)
{
    if (!norm || !aligned16(norm)) return fail(OWT_EINVAL, "norm is NULL or not 16-byte aligned");
    if (!(max_norm > 0.f)) return fail(OWT_EINVAL, "max_norm must be positive");
    return OWT_OK;
}

owt_status owt_grad_clip(int count, const size_t *n, const void *const *g, void *const *out, owt_dtype dtype, const float *norm, float max_norm,
                         void *hip_stream)
{
    if (dtype != OWT_F32 && dtype != OWT_BF16) return fail(OWT_EINVAL, "unknown dtype %d", (int)dtype);
    const int chunk = values_of_chunk(dtype);
    size_t chunks;
    OWT_TRY(check_list(count, n, chunks, chunk));
    OWT_TRY(check_pointers(count, n, g, "g"));
    OWT_TRY(check_pointers(count, n, out, "out"));
    OWT_TRY(check_bound(norm, max_norm));
    hipStream_t s = (hipStream_t)hip_stream;
    return for_sets<2>(count, n, {g, out}, chunk, [&](const TensorSet<2> &set, unsigned groups) {
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(groups), dim3(256), 0, s, set, norm, max_norm); };
        const bool past = chunks > kPastChunks;
        if (dtype == OWT_F32) { if (past) go(grad_clip_kernel<float, true>); else go(grad_clip_kernel<float, false>); }
        else if (past) go(grad_clip_kernel<bf16_t, true>);
        else go(grad_clip_kernel<bf16_t, false>);
    });
}

owt_status owt_sgd_momentum_clipped(int count, const size_t *n, float *const *w, float *const *vel, const float *const *g, float mu, float eps,
                                    float omega, float gscale, const float *norm, float max_norm, void *const *w_bf16_or_null, void *hip_stream)
{
    const int chunk = values_of_chunk(OWT_F32);
    size_t chunks;
    OWT_TRY(check_list(count, n, chunks, chunk));
    OWT_TRY(check_pointers(count, n, (const void *const *)w, "w"));
    OWT_TRY(check_pointers(count, n, (const void *const *)vel, "vel"));
    OWT_TRY(check_pointers(count, n, (const void *const *)g, "g"));
    if (w_bf16_or_null) OWT_TRY(check_pointers(count, n, w_bf16_or_null, "w_bf16"));
    if (!std::isfinite(mu) || !std::isfinite(eps) || !std::isfinite(omega) || !std::isfinite(gscale))
        return fail(OWT_EINVAL, "mu, eps, omega and gscale must be finite");
    OWT_TRY(check_bound(norm, max_norm));
    hipStream_t s = (hipStream_t)hip_stream;
    const void *const *W = (const void *const *)w, *const *V = (const void *const *)vel, *const *G = (const void *const *)g;
    const bool past = chunks > kPastChunks / 2;         // (two lists are written)
    if (w_bf16_or_null)
        return for_sets<4>(count, n, {W, V, G, w_bf16_or_null}, chunk, [&](const TensorSet<4> &set, unsigned groups) {
            auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(groups), dim3(256), 0, s, set, mu, eps, omega, gscale, norm, max_norm); };
            if (past) go(sgd_clipped_kernel<true, true>);
            else go(sgd_clipped_kernel<true, false>);
        });
    return for_sets<3>(count, n, {W, V, G}, chunk, [&](const TensorSet<3> &set, unsigned groups) {
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(groups), dim3(256), 0, s, set, mu, eps, omega, gscale, norm, max_norm); };
        if (past) go(sgd_clipped_kernel<false, true>);
        else go(sgd_clipped_kernel<false, false>);
    });
}

}  // extern "C"

// Rows of 8-bit values: writing them (a checkpoint, or the RMS norm of a sum), reading them back, and the norm's backward pass.
//
//   value = q * scale, one scale a row, q = nearest whole number (ties to even) to t * 127 / max|t|, scale = max|t| / 127
//   norm: h = x + res, t = h * gain, rstd = (mean h^2 + eps)^-1/2, scale = max|t| / 127 * rstd:
// rstd is a factor of the whole row, so q does not depend on it and one pass with one reduction (the sum of squares and the largest
// magnitude together) gives everything.  All of it is bound by memory: a row is read once, stays in registers across the reduction, and is
// written once.
#pragma once
#include "owt_common.hpp"
#include "q8.hpp"
#include "q8piece.hpp"

namespace owt {

// V whole numbers of -127 .. 127, packed
template <int V> __device__ __forceinline__ void store_q(signed char *p, const int (&q)[V])
{
    uint32_t w[V / 4];
#pragma unroll
    for (int k = 0; k < V / 4; k++)
        w[k] = (q[4 * k] & 255u) | ((q[4 * k + 1] & 255u) << 8) | ((q[4 * k + 2] & 255u) << 16) | ((uint32_t)q[4 * k + 3] << 24);
    if (V == 4) *(uint32_t *)p = w[0];
    else *(uint2 *)p = make_uint2(w[0], w[V / 4 - 1]);
}

// (sum, largest of unsigned bit patterns) over the TPR threads of a row, the same in every one of them and in a fixed order.  `slot`: LDS
// of this row, two places a wavefront; its use by the next call is kept apart by the caller.
template <int TPR> __device__ __forceinline__ void row_reduce(float &s, uint32_t &m, float *slot, int lane_in_row)
{
#pragma unroll
    for (int d = (TPR < 64 ? TPR : 64) / 2; d >= 1; d >>= 1) {
        s += __shfl_xor(s, d, 64);
        m = max(m, (uint32_t)__shfl_xor((int)m, d, 64));
    }
    if (TPR > 64) {
        constexpr int W = TPR / 64;
        const int w = lane_in_row >> 6;
        if ((lane_in_row & 63) == 0) { slot[2 * w] = s; slot[2 * w + 1] = __uint_as_float(m); }
        __syncthreads();
        s = 0.f; m = 0;
#pragma unroll
        for (int k = 0; k < W; k++) { s += slot[2 * k]; m = max(m, __float_as_uint(slot[2 * k + 1])); }
    }
}

struct Q8RowParams {
    const void *x, *res;        // res: norm only, may be null
    const float *gain;          // norm only, may be null (all ones)
    void *h;                    // norm with res only, may be null; may be x or res
    signed char *q;
    float *scale, *rstd;        // rstd: norm only, may be null
    int rows, cols;
    size_t pitch;
    float eps;
};

// What a row's largest magnitude (as bits) gives.  NaN has larger bits than infinity, so it survives the maximum: a row that holds either
// has q = 0 and a scale that is not finite, and reads back as NaN everywhere instead of as numbers that look right.  Rows of magnitudes
// near the smallest of fp32, whose reciprocal would overflow, are scaled by 2^64 on the way.
struct Q8Scale {
    float up, inv, unit;
    bool fine;
    __device__ __forceinline__ Q8Scale(uint32_t bits)
    {
        const float amax = __uint_as_float(bits);
        fine = bits > 0 && bits < 0x7f800000u;
        up = amax < 0x1p-64f ? 0x1p64f : 1.f;
        inv = 127.f * (1.f / (amax * up));
        unit = amax / 127.f;
    }
    __device__ __forceinline__ int operator()(float t) const { return fine ? __float2int_rn(t * up * inv) : 0; }
};

// TPR threads a row, 16 to 1024 of a work-group's 256 or 1024, each with up to P pieces in registers.  LONG: rows of more pieces than that are read again after the
// reduction (the caches hold them).  BIG: a tensor is more than an eighth of the 256 MB behind the L2 caches.  Then h is not there any more
// when it is read again, behind the products in between, and what is read here is not read again: past the caches, 16384 x 4096 bf16 values
// are packed in 37 us (46 without) and the norm of 8192 x 4096 takes 47 (56).
template <class T, bool NORM, bool RES, int TPR, int P, bool LONG, bool BIG>
__global__ void __launch_bounds__(TPR > 256 ? TPR : 256) q8_rows_kernel(const Q8RowParams p)
{
    constexpr int V = Piece<T>::V, THREADS = TPR > 256 ? TPR : 256, RPW = THREADS / TPR;
    __shared__ float red[2 * (THREADS / 64)];
    const int sub = threadIdx.x / TPR, t0 = threadIdx.x % TPR;
    const size_t row = (size_t)blockIdx.x * RPW + sub;
    const bool in = row < (size_t)p.rows;
    const T *x = (const T *)p.x + row * p.cols, *res = RES ? (const T *)p.res + row * p.cols : nullptr;
    signed char *q = p.q + row * p.pitch;
    const int pieces = (int)(p.pitch / V), full = in ? (p.cols + V - 1) / V : 0;

    // h of a piece, and t from it
    auto fetch = [&](int j, float (&v)[V]) __attribute__((always_inline)) {
        load_piece<T, BIG && !LONG>(x, j, p.cols, v);
        if (RES) {
            float r[V];
            load_piece<T, BIG && !LONG>(res, j, p.cols, r);
#pragma unroll
            for (int i = 0; i < V; i++) v[i] += r[i];
        }
    };
    auto gained = [&](int j, float (&v)[V]) __attribute__((always_inline)) {
        if (NORM && p.gain) {
            float g[4];
#pragma unroll
            for (int k = 0; k < V / 4; k++) {
                load_piece<float>(p.gain, j * (V / 4) + k, p.cols, g);
#pragma unroll
                for (int i = 0; i < 4; i++) v[4 * k + i] *= g[i];
            }
        }
    };
    float s = 0.f;
    uint32_t m = 0;
    auto tally = [&](const float (&v)[V]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < V; i++) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
    };
    auto squares = [&](const float (&v)[V]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < V; i++) s = fmaf(v[i], v[i], s);
    };
    auto put = [&](int j, const Q8Scale &sc, const float (&v)[V]) __attribute__((always_inline)) {
        int o[V];
#pragma unroll
        for (int i = 0; i < V; i++) o[i] = sc(v[i]);
        store_q<V>(q + (size_t)j * V, o);
    };

    auto put_h = [&](int j, const float (&v)[V]) __attribute__((always_inline)) { store_piece<T, BIG>((T *)p.h + row * p.cols, j, p.cols, v); };
    if (!LONG) {
        float v[P][V];
#pragma unroll
        for (int k = 0; k < P; k++) {
            const int j = k * TPR + t0;
            if (j < full) fetch(j, v[k]);
            else
#pragma unroll
                for (int i = 0; i < V; i++) v[k][i] = 0.f;
        }
#pragma unroll
        for (int k = 0; k < P; k++) {
            const int j = k * TPR + t0;
            if (NORM) squares(v[k]);
            if (NORM && RES && p.h && j < full) put_h(j, v[k]);
            if (j < full) gained(j, v[k]);
            tally(v[k]);
        }
        row_reduce<TPR>(s, m, red, t0);
        const Q8Scale sc(m);
        if (!in) return;
#pragma unroll
        for (int k = 0; k < P; k++)
            if (k * TPR + t0 < pieces) put(k * TPR + t0, sc, v[k]);
        if (t0 == 0) {
            const float rstd = NORM ? 1.f / sqrtf(s / (float)p.cols + p.eps) : 1.f;
            p.scale[row] = NORM ? sc.unit * rstd : sc.unit;
            if (NORM && p.rstd) p.rstd[row] = rstd;
        }
    } else {
        for (int j = t0; j < full; j += TPR) {
            float v[V];
            fetch(j, v);
            if (NORM) squares(v);
            gained(j, v);
            tally(v);
        }
        row_reduce<TPR>(s, m, red, t0);
        const Q8Scale sc(m);
        if (!in) return;
        for (int j = t0; j < pieces; j += TPR) {
            float v[V];
#pragma unroll
            for (int i = 0; i < V; i++) v[i] = 0.f;
            if (j < full) {
                fetch(j, v);
                if (NORM && RES && p.h) put_h(j, v);
                gained(j, v);
            }
            put(j, sc, v);
        }
        if (t0 == 0) {
            const float rstd = NORM ? 1.f / sqrtf(s / (float)p.cols + p.eps) : 1.f;
            p.scale[row] = NORM ? sc.unit * rstd : sc.unit;
            if (NORM && p.rstd) p.rstd[row] = rstd;
        }
    }
}

// x = q * scale: a piece a thread, 2^lpr threads next to each other in a row, `segs` runs of them along it.
template <class T>
__global__ void __launch_bounds__(256) q8_unpack_kernel(const signed char *__restrict__ q, const float *__restrict__ scale, T *__restrict__ x,
                                                        int rows, int cols, size_t pitch, int lpr, unsigned segs)
{
    constexpr int V = Piece<T>::V;
    const unsigned rb = blockIdx.x / segs, seg = blockIdx.x - rb * segs;
    const size_t row = ((size_t)rb << (8 - lpr)) + (threadIdx.x >> lpr);
    const int j = (int)((seg << lpr) + (threadIdx.x & ((1u << lpr) - 1)));
    if (row >= (size_t)rows || (long)j * V >= cols) return;
    const signed char *src = q + row * pitch + (size_t)j * V;
    uint32_t w[V / 4];
    if (V == 4) w[0] = *(const uint32_t *)src;
    else {
        const uint2 u = *(const uint2 *)src;
        w[0] = u.x; w[V / 4 - 1] = u.y;
    }
    const float sc = scale[row];
    float v[V];
#pragma unroll
    for (int i = 0; i < V; i++) v[i] = (float)(signed char)(w[i / 4] >> (8 * (i & 3))) * sc;
    store_piece<T>(x + row * cols, j, cols, v);
}

// The norm's backward pass.  With xn = h * rstd and g = dy * gain:
//   dh = rstd * (g - xn * mean(g * xn)) + dres;   dgain[c] = sum over rows of dy * xn
struct Q8NormBwdParams {
    const void *dy, *h, *dres;
    const float *gain, *rstd;
    void *dh;
    float *partial;             // [strips][cols] sums of dy * xn, or null
    int rows, cols, strips;
};

// A strip of rows is every strips-th row; TPR threads walk it, each with its P pieces of the columns, whose sums for the gain stay in
// registers to the end of the strip.  BIG as above (8192 x 4096 bf16 53 us, 55 without; 515 x 9216 fp32, which the caches hold, 19 and 17).
template <class T, bool RES, int TPR, int P, bool BIG>
__global__ void __launch_bounds__(TPR > 256 ? TPR : 256) rmsnorm_bwd_kernel(const Q8NormBwdParams p)
{
    constexpr int V = Piece<T>::V, THREADS = TPR > 256 ? TPR : 256, SPW = THREADS / TPR;
    __shared__ float red[2][2 * (THREADS / 64)];
    const int sub = threadIdx.x / TPR, t0 = threadIdx.x % TPR;
    const int strip = blockIdx.x * SPW + sub;
    if (TPR <= 64 && strip >= p.strips) return;     // (wider rows have a work-group to themselves and a strip each)
    const int full = (p.cols + V - 1) / V;
    const float inv = 1.f / (float)p.cols;
    // The gain stays in registers, too, where they hold it: not for more than 16 values of each of 1024 threads.
    constexpr bool HELD = P * V <= 16 || TPR < 1024;
    float gain[HELD ? P : 1][V], sum[P][V];
    auto fetch_gain = [&](int k, float (&to)[V]) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < V / 4; c++) {
            float g[4] = {1.f, 1.f, 1.f, 1.f};
            if (p.gain) load_piece<float>(p.gain, (k * TPR + t0) * (V / 4) + c, p.cols, g);
#pragma unroll
            for (int i = 0; i < 4; i++) to[4 * c + i] = g[i];
        }
    };
#pragma unroll
    for (int k = 0; k < P; k++) {
        if (HELD) fetch_gain(k, gain[HELD ? k : 0]);
#pragma unroll
        for (int i = 0; i < V; i++) sum[k][i] = 0.f;
    }
    int turn = 0;
    for (size_t row = strip; row < (size_t)p.rows; row += p.strips, turn ^= 1) {
        const size_t at = row * p.cols;
        const float rstd = p.rstd[row];
        float h[P][V], d[P][V], dot = 0.f;
#pragma unroll
        for (int k = 0; k < P; k++) {
            const int j = k * TPR + t0;
            if (j < full) {
                load_piece<T, BIG>((const T *)p.h + at, j, p.cols, h[k]);
                load_piece<T, BIG>((const T *)p.dy + at, j, p.cols, d[k]);
            } else
#pragma unroll
                for (int i = 0; i < V; i++) h[k][i] = d[k][i] = 0.f;
        }
#pragma unroll
        for (int k = 0; k < P; k++) {
            if (!HELD) fetch_gain(k, gain[0]);
#pragma unroll
            for (int i = 0; i < V; i++) {
                h[k][i] *= rstd;
                sum[k][i] = fmaf(d[k][i], h[k][i], sum[k][i]);
                d[k][i] *= gain[HELD ? k : 0][i];
                dot = fmaf(d[k][i], h[k][i], dot);
            }
        }
        uint32_t none = 0;
        row_reduce<TPR>(dot, none, red[turn], t0);
        const float mean = dot * inv;
#pragma unroll
        for (int k = 0; k < P; k++) {
            const int j = k * TPR + t0;
            if (j >= full) continue;
            float r[V];
            if (RES) load_piece<T, BIG>((const T *)p.dres + at, j, p.cols, r);
#pragma unroll
            for (int i = 0; i < V; i++) {
                const float v = rstd * fmaf(-h[k][i], mean, d[k][i]);
                r[i] = RES ? v + r[i] : v;
            }
            store_piece<T>((T *)p.dh + at, j, p.cols, r);
        }
    }
    if (p.partial) {
        float *out = p.partial + (size_t)strip * p.cols;
#pragma unroll
        for (int k = 0; k < P; k++)
#pragma unroll
            for (int c = 0; c < V / 4; c++) {
                const int j = (k * TPR + t0) * (V / 4) + c;
                if (j * 4 >= p.cols) continue;
                float v[4];
#pragma unroll
                for (int i = 0; i < 4; i++) v[i] = sum[k][4 * c + i];
                store_piece<float>(out, j, p.cols, v);
            }
    }
}

// dgain = alpha * (the strips' sums, in order) + beta * dgain: 16 columns x 16 phases of the strips a work-group.
__global__ void __launch_bounds__(256) rmsnorm_dgain_kernel(const float *__restrict__ partial, float *dgain, int cols, int strips, float alpha, float beta)
{
    __shared__ float red[16][17];
    const int cl = threadIdx.x & 15, ph = threadIdx.x >> 4, c = blockIdx.x * 16 + cl;
    float s = 0.f;
    if (c < cols)
#pragma unroll 16
        for (int k = ph; k < strips; k += 16) s += partial[(size_t)k * cols + c];
    red[ph][cl] = s;
    __syncthreads();
    if (ph == 0 && c < cols) {
        float t = 0.f;
#pragma unroll
        for (int k = 0; k < 16; k++) t += red[k][cl];
        dgain[c] = alpha * t + (beta != 0.f ? beta * dgain[c] : 0.f);
    }
}

}  // namespace owt

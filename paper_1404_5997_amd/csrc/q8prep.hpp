// Operands of the 8-bit shard's backward products (q8gemm.hpp).
//
// With dz = dy where y > 0 (or dy), the left operands are  dw: A[o][n] = dz[n][o] xs[n],  dx: A[n][o] = dz[n][o] ws[o],  the right ones the
// whole numbers, transposed: B[i][n] = xq[n][i],  B[i][o] = wq[o][i].  Whole numbers of 8 bits are exact in f16.  A row of a left operand
// is scaled by a power of two that takes its largest finite magnitude to [2^14, 2^15), and each value is written as h + m, two f16
// values: that holds 22 bits of a value of 2^-16 of the row's largest and more, and 2^-39 of the largest below.  bf16 dx takes h alone (11
// bits, where the result keeps 8).  A value that is not finite is h by itself.
//
// First launch: dz is read once for the bias gradient's sums and the largest magnitudes of columns (times xs) and rows (times ws), in
// parts of 64 columns x a strip of rows.  Second launch: operands, 64 x 64 values a work-group, through LDS where they are transposed.
#pragma once
#include "owt_common.hpp"

namespace owt {

struct Q8PrepParams {
    const void *dy, *y;                 // y: ReLU mask, may be null
    const float *xs, *ws;
    const signed char *xq, *wq;
    int N, I, O, bf16;
    size_t xpitch;                      // of xq and wq
    int want_dx, dx_planes;
    float alpha, beta;
    float *db;                          // may be null
    // scratch
    int strips, strip_rows;             // strips of rows (multiples of 64) of the first launch
    float *colsum;                      // [strips][O]
    float *colmax;                      // [strips][O]
    float *rowmax;                      // [ceil(O/64)][N]
    int *col_exp, *row_exp;             // [O], [N]
    _Float16 *aw, *ax, *bw, *bx;        // dw: [O][Nk][2][64], dx: [N][Ok][planes][64]; [I][Nk][64], [I][Ok][64] (Nk, Ok steps of 64)
    int nk, ok;                         // steps of 64 rows (tokens), of 64 outputs
    int tiles_z, tiles_x;               // work-groups of the second launch: dz's, then xq's, then wq's
};

constexpr int kQ8PrepTile = 64;

template <class T> __device__ __forceinline__ float q8_dz(const Q8PrepParams &p, size_t at)
{
    const float v = load1((const T *)p.dy + at, 0);
    return p.y && !(load1((const T *)p.y + at, 0) > 0.f) ? 0.f : v;
}
// what a value adds to a largest finite magnitude
__device__ __forceinline__ float q8_finite_abs(float v) { return fabsf(v) < __uint_as_float(0x7f800000u) ? fabsf(v) : 0.f; }
// the power of two that takes it to [2^14, 2^15)
__device__ __forceinline__ int q8_exponent(float largest) { return largest > 0.f ? 14 - ilogbf(largest) : 0; }

// 256 threads: thread (c, r) = column c of 64, every fourth row of the strip.
template <class T> __global__ void __launch_bounds__(256) q8_stat_kernel(const Q8PrepParams p)
{
    __shared__ float red[2][4][64];
    const int c = threadIdx.x & 63, r = threadIdx.x >> 6, cb = blockIdx.x, strip = blockIdx.y, o = cb * 64 + c;
    const int n_end = min(p.N, (strip + 1) * p.strip_rows);
    const float ws = o < p.O ? p.ws[o] : 0.f;
    float sum = 0.f, cmax = 0.f;
    for (int n = strip * p.strip_rows + r; n < n_end; n += 4) {       // (a wavefront is one row of 64 columns: the loop is uniform in it)
        const float dz = o < p.O ? q8_dz<T>(p, (size_t)n * p.O + o) : 0.f;
        sum += dz;
        cmax = fmaxf(cmax, q8_finite_abs(dz * p.xs[n]));
        if (p.want_dx) {
            float v = q8_finite_abs(dz * ws);
#pragma unroll
            for (int d = 32; d >= 1; d >>= 1) v = fmaxf(v, __shfl_xor(v, d, 64));
            if (c == 0) p.rowmax[(size_t)cb * p.N + n] = v;
        }
    }
    red[0][r][c] = sum;
    red[1][r][c] = cmax;
    __syncthreads();
    if (r == 0 && o < p.O) {
        p.colsum[(size_t)strip * p.O + o] = (red[0][0][c] + red[0][1][c]) + (red[0][2][c] + red[0][3][c]);
        p.colmax[(size_t)strip * p.O + o] = fmaxf(fmaxf(red[1][0][c], red[1][1][c]), fmaxf(red[1][2][c], red[1][3][c]));
    }
}

__device__ __forceinline__ void q8_halves(float v, int e, _Float16 &h, _Float16 &m)
{
    const float t = ldexpf(v, e);
    h = (_Float16)t;
    m = fabsf(t) < __uint_as_float(0x7f800000u) ? (_Float16)(t - (float)h) : (_Float16)0.f;
}

// A 64 x 64 tile of whole numbers q[k][i], as f16 to b[i][k]
__device__ __forceinline__ void q8_turn(const signed char *q, size_t pitch, int K, int I, int kt, int it, _Float16 *b, int ksteps, unsigned char *lds)
{
    // threads 16 a row of 4 values; LDS [k][i], rows of 68 bytes
    const int tid = threadIdx.x;
#pragma unroll
    for (int s = 0; s < 4; s++) {
        const int k = s * 16 + (tid >> 4), i = (tid & 15) * 4;
        // (a row is whole multiples of 128 bytes, so the four are inside it)
        const uint32_t w = kt * 64 + k < K ? *(const uint32_t *)(q + (size_t)(kt * 64 + k) * pitch + it * 64 + i) : 0u;
        *(uint32_t *)(lds + k * 68 + i) = w;
    }
    __syncthreads();
    // threads 8 a row of 8 values
#pragma unroll
    for (int s = 0; s < 2; s++) {
        const int i = s * 32 + (tid >> 3), k = (tid & 7) * 8;
        if (it * 64 + i >= I) continue;
        union { _Float16 h[8]; uint4 u; } v;
#pragma unroll
        for (int j = 0; j < 8; j++) v.h[j] = (_Float16)(float)(signed char)lds[(k + j) * 68 + i];
        *(uint4 *)(b + ((size_t)(it * 64 + i) * ksteps + kt) * 64 + k) = v.u;
    }
}

template <class T> __global__ void __launch_bounds__(256) q8_prep_kernel(const Q8PrepParams p)
{
    __shared__ __attribute__((aligned(16))) float tile[64 * 65];
    __shared__ int ce[64], re[64];
    const int tid = threadIdx.x;
    int b = blockIdx.x;
    if (b >= p.tiles_z) {
        b -= p.tiles_z;
        const int its = (p.I + 63) / 64;
        if (b < p.tiles_x) q8_turn(p.xq, p.xpitch, p.N, p.I, b / its, b % its, p.bw, p.nk, (unsigned char *)tile);
        else {
            b -= p.tiles_x;
            q8_turn(p.wq, p.xpitch, p.O, p.I, b / its, b % its, p.bx, p.ok, (unsigned char *)tile);
        }
        return;
    }
    const int nt = b / p.ok, ot = b % p.ok, n0 = nt * 64, o0 = ot * 64;
    if (tid < 64) {                                 // exponents of the columns; the bias gradient
        const int o = o0 + tid;
        float mx = 0.f, s = 0.f;
        if (o < p.O)
            for (int k = 0; k < p.strips; k++) {
                mx = fmaxf(mx, p.colmax[(size_t)k * p.O + o]);
                if (nt == 0) s += p.colsum[(size_t)k * p.O + o];
            }
        ce[tid] = q8_exponent(mx);
        if (nt == 0 && o < p.O) {
            p.col_exp[o] = ce[tid];
            if (p.db) p.db[o] = p.alpha * s + (p.beta != 0.f ? p.beta * p.db[o] : 0.f);
        }
    } else if (tid < 128 && p.want_dx) {            // and of the rows
        const int n = n0 + tid - 64, cbs = (p.O + 63) / 64;
        float mx = 0.f;
        if (n < p.N)
            for (int k = 0; k < cbs; k++) mx = fmaxf(mx, p.rowmax[(size_t)k * p.N + n]);
        re[tid - 64] = q8_exponent(mx);
        if (ot == 0 && n < p.N) p.row_exp[n] = re[tid - 64];
    }
    const int c = tid & 63, r = tid >> 6, o = o0 + c;
    const float ws = o < p.O ? p.ws[o] : 0.f;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 16; k++) {
        const int n = n0 + 4 * k + r;
        const float dz = n < p.N && o < p.O ? q8_dz<T>(p, (size_t)n * p.O + o) : 0.f;
        tile[(4 * k + r) * 65 + c] = n < p.N ? dz * p.xs[n] : 0.f;
        if (p.want_dx && n < p.N) {
            _Float16 h, m;
            q8_halves(dz * ws, re[4 * k + r], h, m);
            _Float16 *at = p.ax + ((size_t)n * p.ok + ot) * p.dx_planes * 64 + c;
            at[0] = h;
            if (p.dx_planes == 2) at[64] = m;
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 16; k++) {                  // a wavefront writes a row of 64 tokens
        const int oc = 4 * k + r;
        if (o0 + oc >= p.O) continue;
        _Float16 h, m;
        q8_halves(tile[c * 65 + oc], ce[oc], h, m);
        _Float16 *at = p.aw + ((size_t)(o0 + oc) * p.nk + nt) * 128 + c;
        at[0] = h;
        at[64] = m;
    }
}

}  // namespace owt

// Operands of the 8-bit shard's backward products (q8gemm.hpp).
//
// With dz = dy where y > 0 (or dy), the left operands are  dw: A[o][n] = dz[n][o] xs[n],  dx: A[n][o] = dz[n][o] ws[o],  the right ones the
// whole numbers, transposed: B[i][n] = xq[n][i],  B[i][o] = wq[o][i].  Whole numbers of 8 bits are exact in f16.  A row of a left operand
// is scaled by a power of two that takes its largest finite magnitude to [2^14, 2^15), and each value is written as h + m, two f16
// values: that holds 22 bits of a value of 2^-16 of the row's largest and more, and 2^-39 of the largest below.  (bf16 dx as well: of h alone
// its sums are off by 2^-12 of their terms, which is more than the result's own rounding where they cancel.)  A value that is not finite is h by itself.
//
// First launch: the whole numbers are turned, and dz is read once for the bias gradient's sums and the largest magnitudes of columns (times
// xs) and rows (times ws), in parts of 64 columns x a strip of rows.  Second launch: the left operands, 64 x 64 values a work-group, the
// one of dw turned through LDS.  Both are bound by memory: 8192 x 4096 -> 4096 in bf16 moves 580 MB in 120 us.  (One
// launch for few rows and columns, each work-group finding the magnitudes of its own: 128 x 9216 -> 512 16 us where these two take 12.)
#pragma once
#include <type_traits>

#include "owt_common.hpp"
#include "q8piece.hpp"

namespace owt {

struct Q8PrepParams {
    const void *dy, *y;                 // y: ReLU mask, may be null
    const float *xs, *ws;
    const signed char *xq, *wq;
    int N, I, O;
    size_t xpitch;                      // of xq and wq
    int want_dx;
    float alpha, beta;
    float *db;                          // may be null
    // scratch
    int strips, strip_rows;             // strips of rows (multiples of 64) of the first launch
    float *colsum;                      // [strips][O]
    float *colmax;                      // [strips][O]
    float *rowmax;                      // [ceil(O/64)][N]
    int *col_exp, *row_exp;             // [O], [N]
    _Float16 *aw, *ax, *bw, *bx;        // dw: [O][nk][2][64], dx: [N][ok][2][64]; [I][nk][64], [I][ok][64]
    int nk, ok;                         // steps of 64 rows (tokens), of 64 outputs
    int tiles_s, tiles_x;               // work-groups of the first launch: statistics, then xq's tiles, then wq's
};

// dz of piece j of row n (zeros past the end of either).  HOW: 0 for any rows; 1 where rows are whole pieces and there are some, 2 where they
// have a mask besides: then no load is behind a branch, and as many are on their way as a loop is unrolled to (behind branches they
// wait for each other).
template <class T, int HOW> __device__ __forceinline__ void q8_dz(const Q8PrepParams &p, int n, int j, float (&v)[Piece<T>::V])
{
    constexpr int V = Piece<T>::V;
    const bool in = n < p.N && j * V < p.O;
    if (HOW) {
        const size_t at = (size_t)min(n, p.N - 1) * p.O + min(j, p.O / V - 1) * V;
        Piece<T>::load((const T *)p.dy + at, v);
        float y[V];
        if (HOW == 2) Piece<T>::load((const T *)p.y + at, y);
#pragma unroll
        for (int i = 0; i < V; i++) v[i] = in && (HOW == 1 || y[i] > 0.f) ? v[i] : 0.f;
        return;
    }
#pragma unroll
    for (int i = 0; i < V; i++) v[i] = 0.f;
    if (!in) return;
    load_piece_at_once<T>((const T *)p.dy + (size_t)n * p.O, j, p.O, v);
    if (p.y) {
        float y[V];
        load_piece_at_once<T>((const T *)p.y + (size_t)n * p.O, j, p.O, y);
#pragma unroll
        for (int i = 0; i < V; i++) v[i] = y[i] > 0.f ? v[i] : 0.f;
    }
}
template <class T, class F> __device__ __forceinline__ void q8_rows_are(const Q8PrepParams &p, F f)
{
    if (p.N <= 0 || p.O % Piece<T>::V) f(std::integral_constant<int, 0>{});
    else if (p.y) f(std::integral_constant<int, 2>{});
    else f(std::integral_constant<int, 1>{});
}
// what a value adds to a largest finite magnitude
__device__ __forceinline__ float q8_finite_abs(float v) { return fabsf(v) < __uint_as_float(0x7f800000u) ? fabsf(v) : 0.f; }
// the power of two that takes it to [2^14, 2^15)
__device__ __forceinline__ int q8_exponent(float largest) { return largest > 0.f ? 15 - __builtin_amdgcn_frexp_expf(largest) : 0; }
// v 2^e as two f16 values, the first in the low half
__device__ __forceinline__ uint32_t q8_halves(float v, int e)
{
    const float t = ldexpf(v, e);
    const _Float16 h = (_Float16)t, m = fabsf(t) < __uint_as_float(0x7f800000u) ? (_Float16)(t - (float)h) : (_Float16)0.f;
    return (uint32_t)__builtin_bit_cast(uint16_t, h) | ((uint32_t)__builtin_bit_cast(uint16_t, m) << 16);
}

// The first launch's statistics: 64 columns of a strip of rows.  A wavefront reads 64 / LPR rows at a time, LPR lanes a row.
template <class T, int HOW> __device__ __forceinline__ void q8_stat(const Q8PrepParams &p, int cb, int strip, float *lds)
{
    constexpr int V = Piece<T>::V, LPR = 64 / V, RPW = 64 / LPR, AT = 4;      // AT pieces of a thread on their way at a time
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lc = lane % LPR, lr = lane / LPR, j = cb * LPR + lc;
    const int n_end = min(p.N, (strip + 1) * p.strip_rows);
    float ws[V], sum[V], cmax[V];
#pragma unroll
    for (int i = 0; i < V; i++) {
        ws[i] = j * V + i < p.O ? p.ws[j * V + i] : 0.f;
        sum[i] = cmax[i] = 0.f;
    }
    for (int n0 = strip * p.strip_rows + wave * RPW * AT; n0 < n_end; n0 += 4 * RPW * AT) {
        float dz[AT][V], xs[AT];
#pragma unroll
        for (int a = 0; a < AT; a++) {
            const int n = n0 + a * RPW + lr;
            xs[a] = p.xs[min(n, n_end - 1)];
            q8_dz<T, HOW>(p, n < n_end ? n : p.N, j, dz[a]);
        }
#pragma unroll
        for (int a = 0; a < AT; a++) {
            float r = 0.f;
#pragma unroll
            for (int i = 0; i < V; i++) {
                sum[i] += dz[a][i];
                cmax[i] = fmaxf(cmax[i], q8_finite_abs(dz[a][i] * xs[a]));
                r = fmaxf(r, q8_finite_abs(dz[a][i] * ws[i]));
            }
            if (p.want_dx) {
#pragma unroll
                for (int d = LPR / 2; d >= 1; d >>= 1) r = fmaxf(r, __shfl_xor(r, d, 64));
                const int n = n0 + a * RPW + lr;
                if (lc == 0 && n < n_end) p.rowmax[(size_t)cb * p.N + n] = r;
            }
        }
    }
#pragma unroll
    for (int i = 0; i < V; i++) {
#pragma unroll
        for (int d = LPR; d < 64; d <<= 1) {
            sum[i] += __shfl_xor(sum[i], d, 64);
            cmax[i] = fmaxf(cmax[i], __shfl_xor(cmax[i], d, 64));
        }
        if (lr == 0) {
            lds[wave * 64 + lc * V + i] = sum[i];
            lds[256 + wave * 64 + lc * V + i] = cmax[i];
        }
    }
    __syncthreads();
    const int c = threadIdx.x, o = cb * 64 + c;
    if (c < 64 && o < p.O) {
        p.colsum[(size_t)strip * p.O + o] = (lds[c] + lds[64 + c]) + (lds[128 + c] + lds[192 + c]);
        p.colmax[(size_t)strip * p.O + o] = fmaxf(fmaxf(lds[256 + c], lds[320 + c]), fmaxf(lds[384 + c], lds[448 + c]));
    }
}

// Whole numbers q[k][i], 64 k x 128 i, as f16 to b[i][k].  The rows are whole multiples of 128 bytes, so a tile's 128 are inside them.
typedef _Float16 q8_f16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void q8_turn(const signed char *q, size_t pitch, int K, int I, int kt, int it, _Float16 *b, int ksteps, unsigned *lds)
{
    constexpr int P = 33;                           // words of a row in LDS: the eight rows and eight words that lanes read lie in 64 banks
    const int tid = threadIdx.x;
    uint4 w[2];
#pragma unroll
    for (int s = 0; s < 2; s++) {
        const int k = s * 32 + (tid >> 3);
        w[s] = kt * 64 + k < K ? *(const uint4 *)(q + (size_t)(kt * 64 + k) * pitch + it * 128 + (tid & 7) * 16) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int s = 0; s < 2; s++) {
        unsigned *at = lds + (s * 32 + (tid >> 3)) * P + (tid & 7) * 4;
        at[0] = w[s].x; at[1] = w[s].y; at[2] = w[s].z; at[3] = w[s].w;
    }
    __syncthreads();
    const int ko = tid & 7, i4 = tid >> 3;          // eight k, four i
    unsigned r[8];
#pragma unroll
    for (int j = 0; j < 8; j++) r[j] = lds[(ko * 8 + j) * P + i4] ^ 0x80808080u;        // 128 added to each
#pragma unroll
    for (int t = 0; t < 4; t++) {
        const int i = it * 128 + i4 * 4 + t;
        unsigned h[4];
#pragma unroll
        for (int j = 0; j < 4; j++) {
            // 0x64uu is 1024 + uu in f16
            const unsigned two = __builtin_amdgcn_perm(r[2 * j + 1], r[2 * j], 0x0c000c00u | (unsigned)t | ((unsigned)(4 + t) << 16)) | 0x64006400u;
            const q8_f16x2 v = __builtin_bit_cast(q8_f16x2, two) - (q8_f16x2){1152.f, 1152.f};
            h[j] = __builtin_bit_cast(unsigned, v);
        }
        if (i < I) *(uint4 *)(b + ((size_t)i * ksteps + kt) * 64 + ko * 8) = make_uint4(h[0], h[1], h[2], h[3]);
    }
}

template <class T> __global__ void __launch_bounds__(256) q8_stat_kernel(const Q8PrepParams p)
{
    __shared__ __attribute__((aligned(16))) unsigned lds[64 * 33];
    int b = blockIdx.x;
    const int its = (p.I + 127) / 128;
    if (b < p.tiles_s) q8_rows_are<T>(p, [&](auto how) __attribute__((always_inline)) { q8_stat<T, decltype(how)::value>(p, b % p.ok, b / p.ok, (float *)lds); });
    else if ((b -= p.tiles_s) < p.tiles_x) q8_turn(p.xq, p.xpitch, p.N, p.I, b / its, b % its, p.bw, p.nk, lds);
    else {
        b -= p.tiles_x;
        q8_turn(p.wq, p.xpitch, p.O, p.I, b / its, b % its, p.bx, p.ok, lds);
    }
}

// A 64 x 64 tile of dz.  DX: dx's operand, too.
template <class T, bool DX, int HOW> __device__ __forceinline__ void q8_split(const Q8PrepParams &p, uint32_t *tile, int *ce, int *re)
{
    constexpr int V = Piece<T>::V, LPR = 64 / V, RPP = 256 / LPR, PASSES = 64 / RPP;       // lanes a row, rows a pass
    const int tid = threadIdx.x, nt = blockIdx.x / p.ok, ot = blockIdx.x % p.ok, n0 = nt * 64, o0 = ot * 64;
    const int lc = tid % LPR, lr = tid / LPR;
    float dz[PASSES][V], ws[V], xs[PASSES];
#pragma unroll
    for (int s = 0; s < PASSES; s++) {
        const int n = n0 + s * RPP + lr;
        q8_dz<T, HOW>(p, n, ot * LPR + lc, dz[s]);
        xs[s] = n < p.N ? p.xs[n] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < V; i++) ws[i] = o0 + lc * V + i < p.O ? p.ws[o0 + lc * V + i] : 0.f;
    {   // largest magnitudes of the tile's columns and rows, and the bias gradient: each by four threads, every fourth part
        float *red = (float *)tile;                 // [3][4][64], before the tile
        const int i = tid & 63, part = tid >> 6, o = o0 + i, n = n0 + i;
        float cmax = 0.f, sum = 0.f, rmax = 0.f;
        if (o < p.O) {
#pragma unroll 8
            for (int k = part; k < p.strips; k += 4) cmax = fmaxf(cmax, p.colmax[(size_t)k * p.O + o]);
            if (nt == 0)
#pragma unroll 8
                for (int k = part; k < p.strips; k += 4) sum += p.colsum[(size_t)k * p.O + o];
        }
        if (DX && n < p.N)
#pragma unroll 8
            for (int k = part; k < p.ok; k += 4) rmax = fmaxf(rmax, p.rowmax[(size_t)k * p.N + n]);
        red[tid] = cmax; red[256 + tid] = sum; red[512 + tid] = rmax;
        __syncthreads();
        if (tid < 64) {
            const int e = q8_exponent(fmaxf(fmaxf(red[i], red[64 + i]), fmaxf(red[128 + i], red[192 + i])));
            ce[i] = e;
            if (nt == 0 && o < p.O) {
                p.col_exp[o] = e;
                const float s = (red[256 + i] + red[320 + i]) + (red[384 + i] + red[448 + i]);
                if (p.db) p.db[o] = p.alpha * s + (p.beta != 0.f ? p.beta * p.db[o] : 0.f);
            }
        } else if (DX && tid < 128) {
            const int e = q8_exponent(fmaxf(fmaxf(red[512 + i], red[576 + i]), fmaxf(red[640 + i], red[704 + i])));
            re[i] = e;
            if (ot == 0 && n < p.N) p.row_exp[n] = e;
        }
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < PASSES; s++) {
        const int r = s * RPP + lr, n = n0 + r;
#pragma unroll
        for (int i = 0; i < V; i++) tile[r * 65 + lc * V + i] = n < p.N ? q8_halves(dz[s][i] * xs[s], ce[lc * V + i]) : 0u;
        if (DX && n < p.N) {
            uint32_t both[V], h[V / 2], m[V / 2];
            const int e = re[r];
#pragma unroll
            for (int i = 0; i < V; i++) both[i] = q8_halves(dz[s][i] * ws[i], e);
#pragma unroll
            for (int i = 0; i < V / 2; i++) {
                h[i] = __builtin_amdgcn_perm(both[2 * i + 1], both[2 * i], 0x05040100u);
                m[i] = __builtin_amdgcn_perm(both[2 * i + 1], both[2 * i], 0x07060302u);
            }
            _Float16 *at = p.ax + ((size_t)n * p.ok + ot) * 128 + lc * V;
            if (V == 8) {
                *(uint4 *)at = make_uint4(h[0], h[1], h[V / 2 - 2], h[V / 2 - 1]);
                *(uint4 *)(at + 64) = make_uint4(m[0], m[1], m[V / 2 - 2], m[V / 2 - 1]);
            } else {
                *(uint2 *)at = make_uint2(h[0], h[1]);
                *(uint2 *)(at + 64) = make_uint2(m[0], m[1]);
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int at = 0; at < 512; at += 256) {         // eight tokens of an output a thread, eight threads a row of 64
        const int oc = (at + tid) >> 3, ko = tid & 7;
        if (o0 + oc >= p.O) continue;
        uint32_t both[8];
#pragma unroll
        for (int j = 0; j < 8; j++) both[j] = tile[(ko * 8 + j) * 65 + oc];
        uint32_t h[4], m[4];
#pragma unroll
        for (int j = 0; j < 4; j++) {
            h[j] = __builtin_amdgcn_perm(both[2 * j + 1], both[2 * j], 0x05040100u);
            m[j] = __builtin_amdgcn_perm(both[2 * j + 1], both[2 * j], 0x07060302u);
        }
        _Float16 *to = p.aw + ((size_t)(o0 + oc) * p.nk + nt) * 128 + ko * 8;
        *(uint4 *)to = make_uint4(h[0], h[1], h[2], h[3]);
        *(uint4 *)(to + 64) = make_uint4(m[0], m[1], m[2], m[3]);
    }
}

template <class T, bool DX> __global__ void __launch_bounds__(256) q8_prep_kernel(const Q8PrepParams p)
{
    __shared__ uint32_t tile[64 * 65];              // [n][o], both halves of a value in a word
    __shared__ int ce[64], re[64];
    q8_rows_are<T>(p, [&](auto how) __attribute__((always_inline)) { q8_split<T, DX, decltype(how)::value>(p, tile, ce, re); });
}

}  // namespace owt

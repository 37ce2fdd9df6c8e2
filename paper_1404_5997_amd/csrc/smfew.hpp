// Softmax cross-entropy of few fp32 rows: the weights are what it costs, so they are read as they lie, once for the outputs and once for the gradients.
//
//   z[n][o] = bias[o] + sum_i x[n][i] w[o][i]                               leaves as each row's largest value and sum for 16 classes, or as dz in fp32
//   dx[n][i] = sum_o dz[n][o] w[o][i],  dw[o][i] = sum_n dz[n][o] x[n][i]   in one walk over w: a step reads 16 rows of w and writes 16 of dw
//
// v_mfma_f32_16x16x4_f32 takes one value of either operand a lane (lane l: row l % 16, k = l / 16) and gives four results (rows 4 (l / 16) + r of the first
// operand, column l % 16 of the second), so that operands come straight from memory, 16 bytes a lane, and k is in any order that both agree on.  All is fp32.
//
// HBM bounds few rows, the matrix unit many: 64 rows are 16 instructions of 32 clocks a KB of weights (32 for the gradients), 157 TFLOP/s at best.  Measured, outputs | gradients' walk:
//    1 x 2048 -> 65536    99 us, 5.4 TB/s of w     265 us, 4.1 TB/s of w and dw
//    3 x  513 -> 50000    22 us, 4.7 TB/s           59 us, 3.5 TB/s
//   24 x 1024 -> 65536    69 us, 3.9 TB/s          179 us, 3.0 TB/s
//   48 x 1024 -> 65536    90 us, 71 TFLOP/s        203 us, 63 TFLOP/s
//   64 x 1024 -> 65536   105 us, 82 TFLOP/s        229 us, 75 TFLOP/s
#pragma once
#include <type_traits>

#include "smgemm.hpp"

namespace owt {

typedef float sm_f32x4 __attribute__((ext_vector_type(4)));

// 16 bytes from where rows begin anywhere; WHOLE: of a wavefront whose columns are all there
template <bool WHOLE> __device__ __forceinline__ float4 sm_loose4(const float *row, int c, int cols)
{
    if (WHOLE || c + 4 <= cols) {
        const SmLoose l = *(const SmLoose *)(row + c);
        return make_float4(__uint_as_float(l.u[0]), __uint_as_float(l.u[1]), __uint_as_float(l.u[2]), __uint_as_float(l.u[3]));
    }
    return make_float4(c < cols ? row[c] : 0.f, c + 1 < cols ? row[c + 1] : 0.f, c + 2 < cols ? row[c + 2] : 0.f, 0.f);
}
__device__ __forceinline__ void sm_put_loose4(float *to, const float (&u)[4])
{
    SmLoose l;
#pragma unroll
    for (int t = 0; t < 4; t++) l.u[t] = __float_as_uint(u[t]);
    *(SmLoose *)to = l;
}
__device__ __forceinline__ float sm_at(const float4 &v, int k) { return k == 0 ? v.x : k == 1 ? v.y : k == 2 ? v.z : v.w; }

struct SmFewParams {
    const float *x, *w;         // [M][I], [N][I]
    int I;
    float *dz;                  // [M][pitch], zeros from N on
    int pitch;
    SmParams p;                 // M rows, N classes; bias, labels, lse, weight, top, target; dw: out, alpha, beta, big, db; dx: partial
    int strip, strips;          // classes of a work-group, a multiple of 16
};

// 16 CB classes a work-group, 16 NB rows, a quarter of k a wavefront: their sums meet in LDS.
template <int NB, int CB, bool DZ> __global__ void __launch_bounds__(256) sm_few_kernel(const SmFewParams f)
{
    __shared__ float part[4][CB * NB][4][64];
    const SmParams &p = f.p;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r16 = lane & 15, k4 = lane >> 4, v0 = blockIdx.x * 16 * CB;
    const float *wr[CB], *xr[NB];
#pragma unroll
    for (int c = 0; c < CB; c++) wr[c] = f.w + (size_t)min(v0 + 16 * c + r16, p.N - 1) * f.I;
#pragma unroll
    for (int n = 0; n < NB; n++) xr[n] = f.x + (size_t)min(16 * n + r16, p.M - 1) * f.I;
    sm_f32x4 acc[CB][NB];
#pragma unroll
    for (int c = 0; c < CB; c++)
#pragma unroll
        for (int n = 0; n < NB; n++) acc[c][n] = {0.f, 0.f, 0.f, 0.f};
    // A step is 32 values of k: 32 bytes of a row a lane, so that four lanes take a line.  Its products have a sum of their own: chains of 32 and I / 128
    // roundings where one chain of I / 4 was eight times as far off (6 x 2048 -> 1833: dbias 3.5e-6, 4.3e-7 so), in no more time.
    auto step = [&](auto whole, int k) {
        sm_f32x4 sum[CB][NB];
#pragma unroll
        for (int h = 0; h < 2; h++) {
            float4 a[CB], b[NB];
#pragma unroll
            for (int c = 0; c < CB; c++) a[c] = sm_loose4<decltype(whole)::value>(wr[c], k + 4 * h, f.I);
#pragma unroll
            for (int n = 0; n < NB; n++) b[n] = sm_loose4<decltype(whole)::value>(xr[n], k + 4 * h, f.I);
#pragma unroll
            for (int e = 0; e < 4; e++)
#pragma unroll
                for (int c = 0; c < CB; c++)
#pragma unroll
                    for (int n = 0; n < NB; n++) {
                        const sm_f32x4 none = {0.f, 0.f, 0.f, 0.f};
                        sum[c][n] = __builtin_amdgcn_mfma_f32_16x16x4f32(sm_at(a[c], e), sm_at(b[n], e), h || e ? sum[c][n] : none, 0, 0, 0);
                    }
        }
#pragma unroll
        for (int c = 0; c < CB; c++)
#pragma unroll
            for (int n = 0; n < NB; n++) acc[c][n] += sum[c][n];
    };
    int k = 32 * wave;
    for (; k + 32 <= f.I; k += 128) step(std::true_type(), k + 8 * k4);
    if (k < f.I) step(std::false_type(), k + 8 * k4);
#pragma unroll
    for (int c = 0; c < CB; c++)
#pragma unroll
        for (int n = 0; n < NB; n++)
#pragma unroll
            for (int r = 0; r < 4; r++) part[wave][c * NB + n][r][lane] = acc[c][n][r];
    __syncthreads();
    // sums of 16 classes (four of them this lane's) by 16 rows (one of them)
    for (int b = wave; b < CB * NB; b += 4) {
        const int c = v0 + 16 * (b / NB) + 4 * k4, m = 16 * (b % NB) + r16;
        float z[4];
#pragma unroll
        for (int r = 0; r < 4; r++) {
            z[r] = (part[0][b][r][lane] + part[1][b][r][lane]) + (part[2][b][r][lane] + part[3][b][r][lane]);
            z[r] = c + r < p.N ? z[r] + (p.bias ? p.bias[c + r] : 0.f) : -INFINITY;
        }
        if (DZ) {
            const SmDzRow w = sm_dz_row<false>(p, m);
            float d[4];
#pragma unroll
            for (int r = 0; r < 4; r++) {
                const float e = w.weight == 0.f ? 0.f : exp_of(z[r] - w.lse);
                d[r] = w.weight * (w.label == c + r ? e - 1.f : e);
            }
            if (m < p.M && c < f.pitch) *(float4 *)(f.dz + (size_t)m * f.pitch + c) = make_float4(d[0], d[1], d[2], d[3]);
        } else {
            float most = fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3]));
            most = fmaxf(most, __shfl_xor(most, 16, 64));
            most = fmaxf(most, __shfl_xor(most, 32, 64));
            const float at = __builtin_isfinite(most) ? most : 0.f;
            float sum = (exp_of(z[0] - at) + exp_of(z[1] - at)) + (exp_of(z[2] - at) + exp_of(z[3] - at));
            sum += __shfl_xor(sum, 16, 64);
            sum += __shfl_xor(sum, 32, 64);
            if (m < p.M) {
                if (k4 == 0) p.top[(size_t)(blockIdx.x * CB + b / NB) * p.M + m] = {most, sum};
                const int mine = p.labels && has_class(p.labels[m], p.classes) ? p.labels[m] - p.off - c : -1;
#pragma unroll
                for (int r = 0; r < 4; r++)
                    if (mine == r && c + r < p.N) p.target[m] = z[r];
            }
        }
    }
}

// 64 columns a wavefront, `strip` classes a work-group, its rows of x in registers: its rows of dw, its part of dx, and of the first columns' work-groups its classes of dbias.
template <int NB> __global__ void __launch_bounds__(256) sm_few_back_kernel(const SmFewParams f)
{
    constexpr int ROWS = 16 * NB;
    __shared__ float dz[64][ROWS + 1];              // of 64 classes at a time
    const SmParams &p = f.p;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r16 = lane & 15, k4 = lane >> 4;
    const int i0 = blockIdx.x * 256 + wave * 64, strip = blockIdx.y, v_beg = strip * f.strip, v_end = min(p.N, v_beg + f.strip);
    const bool want_dx = p.partial != nullptr;
    // x of dw's products: row 4 s + k4, column i0 + 16 t + r16; rows without a class are zeros
    float xa[4][4 * NB];
#pragma unroll
    for (int s = 0; s < 4 * NB; s++) {
        const int m = 4 * s + k4;
        const bool real = m < p.M && has_class(p.labels[m], p.classes);
#pragma unroll
        for (int t = 0; t < 4; t++) xa[t][s] = real && i0 + 16 * t + r16 < f.I ? f.x[(size_t)m * f.I + i0 + 16 * t + r16] : 0.f;
    }
    sm_f32x4 dx[4][NB];                             // [column of four][row block]: rows 4 k4 + r, column i0 + 4 r16 + j
#pragma unroll
    for (int j = 0; j < 4; j++)
#pragma unroll
        for (int n = 0; n < NB; n++) dx[j][n] = {0.f, 0.f, 0.f, 0.f};
    // four rows of w a lane, read a block of 16 classes ahead (of the last rows again at the end, so that none is read that is not there)
    auto rows_of = [&](int v, float4 (&w)[4]) __attribute__((always_inline)) {
#pragma unroll
        for (int q = 0; q < 4; q++) {
            const float *row = f.w + (size_t)min(v + 4 * q + k4, v_end - 1) * f.I;
            w[q] = i0 + 64 <= f.I ? sm_loose4<true>(row, i0 + 4 * r16, f.I) : sm_loose4<false>(row, i0 + 4 * r16, f.I);
        }
    };
    float4 now[4], next[4];
    if (want_dx && i0 < f.I) rows_of(v_beg, now);
    for (int v0 = v_beg; v0 < v_end; v0 += 16) {
        const int v = (v0 - v_beg) & 63;
        if (v == 0) {
            __syncthreads();
            for (int e = threadIdx.x; e < 64 * ROWS; e += 256) {
                const int m = e >> 6, at = v0 + (e & 63);
                dz[e & 63][m] = m < p.M && at < v_end ? f.dz[(size_t)m * f.pitch + at] : 0.f;
            }
            __syncthreads();
            if (p.db && blockIdx.x == 0 && threadIdx.x < 64 && v0 + (int)threadIdx.x < v_end) {
                float sum = 0.f;
                for (int m = 0; m < p.M; m++) sum += dz[threadIdx.x][m];
                float *db = p.db + v0 + threadIdx.x;
                *db = p.alpha * sum + (p.beta != 0.f ? p.beta * *db : 0.f);
            }
        }
        if (i0 >= f.I) continue;                    // (whole wavefronts; the barriers are in front of it)
        if (want_dx) {
            rows_of(v0 + 16, next);
#pragma unroll
            for (int q = 0; q < 4; q++)
#pragma unroll
                for (int n = 0; n < NB; n++) {
                    const float a = dz[v + 4 * q + k4][16 * n + r16];
#pragma unroll
                    for (int j = 0; j < 4; j++) dx[j][n] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, sm_at(now[q], j), dx[j][n], 0, 0, 0);
                }
#pragma unroll
            for (int q = 0; q < 4; q++) now[q] = next[q];
        }
        sm_f32x4 dw[4];                             // columns i0 + 16 t + 4 k4 + r, class r16
#pragma unroll
        for (int t = 0; t < 4; t++) dw[t] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < 4 * NB; s++) {
            const float b = dz[v + r16][4 * s + k4];
#pragma unroll
            for (int t = 0; t < 4; t++) dw[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(xa[t][s], b, dw[t], 0, 0, 0);
        }
        const int o = v0 + r16;
        if (o >= v_end) continue;
        float *row = (float *)p.out + (size_t)o * f.I;
#pragma unroll
        for (int t = 0; t < 4; t++) {
            const int c = i0 + 16 * t + 4 * k4;
            float u[4] = {p.alpha * dw[t][0], p.alpha * dw[t][1], p.alpha * dw[t][2], p.alpha * dw[t][3]};
            if (c + 4 <= f.I) {
                if (p.beta != 0.f) {
                    const float4 old = sm_loose4<true>(row, c, f.I);
                    u[0] += p.beta * old.x; u[1] += p.beta * old.y; u[2] += p.beta * old.z; u[3] += p.beta * old.w;
                }
                if (p.big) {
                    const sm_f32x4 to = {u[0], u[1], u[2], u[3]};
                    __builtin_nontemporal_store(to, (sm_f32x4 *)(row + c));
                } else sm_put_loose4(row + c, u);
            } else
#pragma unroll
                for (int r = 0; r < 4; r++)
                    if (c + r < f.I) row[c + r] = u[r] + (p.beta != 0.f ? p.beta * row[c + r] : 0.f);
        }
    }
    if (!want_dx || i0 >= f.I) return;
    float *to = p.partial + (size_t)strip * p.M * f.I;
#pragma unroll
    for (int n = 0; n < NB; n++)
#pragma unroll
        for (int r = 0; r < 4; r++) {
            const int m = 16 * n + 4 * k4 + r, c = i0 + 4 * r16;
            if (m >= p.M) continue;
            const float u[4] = {dx[0][n][r], dx[1][n][r], dx[2][n][r], dx[3][n][r]};
            if (c + 4 <= f.I) sm_put_loose4(to + (size_t)m * f.I + c, u);
            else
#pragma unroll
                for (int j = 0; j < 4; j++)
                    if (c + j < f.I) to[(size_t)m * f.I + c + j] = u[j];
        }
}

// dx from the strips' parts, in an order that does not change: 64 x 4 values a work-group, every sixteenth strip a wavefront
__global__ void __launch_bounds__(1024) sm_few_join_kernel(const SmFewParams f)
{
    __shared__ float4 part[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const size_t n = (size_t)f.p.M * f.I, at = ((size_t)blockIdx.x * 64 + lane) * 4;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    if (at < n) {
        const int left = n - at < 4 ? (int)(n - at) : 4;
#pragma unroll 8
        for (int k = wave; k < f.strips; k += 16) {
            const float4 v = sm_loose4<false>(f.p.partial + k * n + at, 0, left);
            sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
        }
    }
    part[wave][lane] = sum;
    __syncthreads();
    if (wave || at >= n) return;
#pragma unroll
    for (int k = 1; k < 16; k++) { sum.x += part[k][lane].x; sum.y += part[k][lane].y; sum.z += part[k][lane].z; sum.w += part[k][lane].w; }
    // (a row without a class is zeros whatever w holds: its zeros of dz times an infinity are not)
    float u[4];
#pragma unroll
    for (int t = 0; t < 4; t++) u[t] = at + t < n && has_class(f.p.labels[(unsigned)(at + t) / (unsigned)f.I], f.p.classes) ? sm_at(sum, t) : 0.f;
    float *to = (float *)f.p.out + at;
    if (at + 4 <= n) *(float4 *)to = make_float4(u[0], u[1], u[2], u[3]);
    else
        for (int t = 0; t < (int)(n - at); t++) to[t] = sm_at(make_float4(u[0], u[1], u[2], u[3]), t);
}

}  // namespace owt

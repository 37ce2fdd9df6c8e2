// Matrix products of the dense shard in 8 bits.
//
//   forward    y[n][o]  = act(xs[n] ws[o] sum_i xq[n][i] wq[o][i] + bias[o])         whole numbers in 8 bits, the sum exact in 32
//   backward   dw[o][i] = alpha sum_n (dz[n][o] xs[n]) xq[n][i] + beta dw            real by whole numbers, on the f16 instruction
//              dx[n][i] = sum_o (dz[n][o] ws[o]) wq[o][i]
//
// All three are C[m][c] = sum_k A[m][k] B[c][k] with k contiguous in both operands (the backward pass lays its operands out so first,
// q8prep.hpp) in rows of whole 128-byte steps, zeros behind the last value: 128 whole numbers or 64 f16 values a step.  A step's
// fragments are 16 consecutive bytes of a row for both instructions (v_mfma_i32_32x32x32_i8: 16 values of a row a lane;
// v_mfma_f32_32x32x16_f16: 8), so one kernel serves both and they differ in the instruction alone.
//
// A work-group's operand tiles go from memory straight into LDS, 1 KB an instruction (8 rows of 128 bytes), into a ring of NS stages;
// 16-byte piece c of row r sits in slot c ^ ((r >> 1) & 7), which spreads a fragment's 32 rows over all banks.  Rows past the end of an
// operand re-read its last one; their results are not stored.
#pragma once
#include "owt_common.hpp"

namespace owt {

typedef float q8_f32x16 __attribute__((ext_vector_type(16)));
typedef int q8_i32x16 __attribute__((ext_vector_type(16)));
typedef int q8_i32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 q8_f16x8 __attribute__((ext_vector_type(8)));

struct Q8Int {
    typedef q8_i32x16 Acc;
    static __device__ __forceinline__ Acc mul(q8_i32x4 a, q8_i32x4 b, Acc c) { return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0); }
};
struct Q8Half {
    typedef q8_f32x16 Acc;
    static __device__ __forceinline__ Acc mul(q8_i32x4 a, q8_i32x4 b, Acc c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(q8_f16x8, a), __builtin_bit_cast(q8_f16x8, b), c, 0, 0, 0);
    }
};

// Results of the forward pass: both scales, bias, ReLU, storage type
struct Q8FwdOut {
    const float *xs, *ws, *bias;        // bias may be null
    void *y;
    int relu, bf16;
};
// Results of a backward product: row m was scaled by 2^exps[m]
struct Q8BwdOut {
    const int *exps;
    float alpha, beta;
    void *out;
    int bf16;
};

struct Q8GemmParams {
    const unsigned char *a, *b;
    size_t lda, ldb;                    // bytes from row to row, multiples of 128
    int M, N, ksteps;                   // rows of C, columns of C, steps of A's rows
    int planes;                         // consecutive steps of A that meet the same step of B
    int tiles_n, splits, ksteps_per_split;
    int tiles;                          // tiles_m * tiles_n
    void *partial;                      // [splits][M][N], 32 bits each (splits > 1)
    Q8FwdOut f;
    Q8BwdOut d;
};

// The value of C[m][c] from its whole sum
__device__ __forceinline__ void q8_finish(const Q8GemmParams &p, int m, int c, int sum)
{
    float v = (float)sum * (p.f.xs[m] * p.f.ws[c]);
    if (p.f.bias) v += p.f.bias[c];
    if (p.f.relu) v = fmaxf(v, 0.f);
    const size_t o = (size_t)m * p.N + c;
    if (p.f.bf16) store1((bf16_t *)p.f.y, o, v);
    else store1((float *)p.f.y, o, v);
}
__device__ __forceinline__ void q8_finish(const Q8GemmParams &p, int m, int c, float sum)
{
    float v = ldexpf(sum, -p.d.exps[m]) * p.d.alpha;
    const size_t o = (size_t)m * p.N + c;
    if (p.d.bf16) store1((bf16_t *)p.d.out, o, v);
    else {
        if (p.d.beta != 0.f) v += p.d.beta * ((const float *)p.d.out)[o];
        store1((float *)p.d.out, o, v);
    }
}

// A wave-uniform address, in scalar registers
__device__ __forceinline__ const unsigned char *q8_uniform(const unsigned char *p)
{
    const unsigned long long a = (unsigned long long)p;
    const unsigned lo = (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)a), hi = (unsigned)__builtin_amdgcn_readfirstlane((int)(a >> 32));
    return (const unsigned char *)(((unsigned long long)hi << 32) | lo);
}

// One tile of C over the steps of `split`: WM x WN wavefronts of MB x NB blocks of 32 x 32; lds: NS stages.
template <class Op, int WM, int WN, int MB, int NB, int NS>
__device__ __forceinline__ void q8gemm_tile(const Q8GemmParams &p, int tile, int split, unsigned char *lds)
{
    constexpr int NW = WM * WN, BM = 32 * MB * WM, BN = 32 * NB * WN;
    constexpr int AI = BM / 8 / NW, BI = BN / 8 / NW, L = AI + BI;       // loads of a wavefront and stage
    static_assert((BM / 8) % NW == 0 && (BN / 8) % NW == 0, "every wavefront issues the same number of loads");
    static_assert(NS >= 2 && NS <= 4 && (NS - 2) * L <= 63, "the wait counter has six bits");
    constexpr int STAGE = (BM + BN) * 128;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int li = lane & 31, lh = lane >> 5;
    const int wm0 = (wave / WN) * 32 * MB, wn0 = (wave % WN) * 32 * NB;
    const int tm = tile / p.tiles_n, tn = tile - tm * p.tiles_n;
    const int m0 = tm * BM, n0 = tn * BN;
    const int ks_beg = split * p.ksteps_per_split;
    const int nst = min(p.ksteps, ks_beg + p.ksteps_per_split) - ks_beg;

    // byte offsets of this lane's pieces of a step from the tile's first row (rows of up to 2^23 bytes: the host sees to it)
    unsigned asrc[AI], bsrc[BI];
#pragma unroll
    for (int i = 0; i < AI; i++) {
        const int row = 8 * (wave + NW * i) + (lane >> 3), piece = (lane & 7) ^ ((row >> 1) & 7);
        asrc[i] = (unsigned)min(row, p.M - 1 - m0) * (unsigned)p.lda + 16 * piece;
    }
#pragma unroll
    for (int i = 0; i < BI; i++) {
        const int row = 8 * (wave + NW * i) + (lane >> 3), piece = (lane & 7) ^ ((row >> 1) & 7);
        bsrc[i] = (unsigned)min(row, p.N - 1 - n0) * (unsigned)p.ldb + 16 * piece;
    }
    const unsigned char *ag = q8_uniform(p.a + (size_t)m0 * p.lda), *bg = q8_uniform(p.b + (size_t)n0 * p.ldb);

    // lane l's 16 bytes land at LDS byte address `dst` (wave-uniform, in m0) + 16 l; the s_nop is the wait state that the hardware wants
    // between a scalar write of m0 and a load into LDS
    auto dma16 = [&](unsigned off, const unsigned char *base, unsigned dst) __attribute__((always_inline)) {
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(off), "s"(base), "s"(__builtin_amdgcn_readfirstlane(dst)) : "memory", "m0");
    };
    const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char *)lds + wave * 1024;
    auto issue = [&](int ks, int buf) __attribute__((always_inline)) {
        ks = __builtin_amdgcn_readfirstlane(ks);
        const unsigned char *ap = ag + (size_t)ks * 128, *bp = bg + (size_t)(p.planes == 2 ? ks >> 1 : ks) * 128;
        const unsigned da = lds0 + buf * STAGE, db = da + BM * 128;
#pragma unroll
        for (int i = 0; i < AI; i++) dma16(asrc[i], ap, da + NW * i * 1024);
#pragma unroll
        for (int i = 0; i < BI; i++) dma16(bsrc[i], bp, db + NW * i * 1024);
    };

    unsigned fr[4];                                 // this lane's piece of a fragment's row, for each quarter of a step
#pragma unroll
    for (int kc = 0; kc < 4; kc++) fr[kc] = li * 128 + 16 * ((2 * kc + lh) ^ ((li >> 1) & 7));

    typename Op::Acc acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; i++)
#pragma unroll
        for (int j = 0; j < NB; j++)
#pragma unroll
            for (int r = 0; r < 16; r++) acc[i][j][r] = 0;

    auto compute = [&](const unsigned char *sa, const unsigned char *sb) __attribute__((always_inline)) {
#pragma unroll
        for (int kc = 0; kc < 4; kc++) {
            q8_i32x4 af[MB], bf[NB];
#pragma unroll
            for (int i = 0; i < MB; i++) af[i] = *(const q8_i32x4 *)(sa + fr[kc] + (wm0 + 32 * i) * 128);
#pragma unroll
            for (int j = 0; j < NB; j++) bf[j] = *(const q8_i32x4 *)(sb + fr[kc] + (wn0 + 32 * j) * 128);
#pragma unroll
            for (int i = 0; i < MB; i++)
#pragma unroll
                for (int j = 0; j < NB; j++) acc[i][j] = Op::mul(af[i], bf[j], acc[i][j]);
        }
    };

    // s_waitcnt vmcnt(k stages' loads) lgkmcnt(0), expcnt untouched
#define OWT_WAIT_STAGES(k) __builtin_amdgcn_s_waitcnt((((k) * L) & 15) | ((((k) * L) >> 4) << 14) | (7 << 4))
#pragma unroll
    for (int i = 0; i < NS - 1; i++)
        if (i < nst) issue(ks_beg + i, i);
    int cur = 0, fill = NS - 1;                     // stage s lives in buffer s % NS; `fill` is the buffer of stage s + NS - 1
    for (int s = 0; s < nst; s++) {
        // this wavefront's pieces of stage s have landed and its reads of stage s - 1 are done; behind the barrier that holds for all
        const int ahead = min(NS - 2, nst - 1 - s);
        if (ahead == 0) OWT_WAIT_STAGES(0);
        else if (ahead == 1) OWT_WAIT_STAGES(1);
        else OWT_WAIT_STAGES(NS >= 4 ? 2 : 1);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (s + NS - 1 < nst) issue(ks_beg + s + NS - 1, fill);
        compute(lds + cur * STAGE, lds + cur * STAGE + BM * 128);
        cur = cur == NS - 1 ? 0 : cur + 1;
        fill = fill == NS - 1 ? 0 : fill + 1;
    }
#undef OWT_WAIT_STAGES

    // accumulator register r of lane (li, lh): row 8 (r / 4) + 4 lh + r % 4, column li of its block
#pragma unroll
    for (int i = 0; i < MB; i++)
#pragma unroll
        for (int r = 0; r < 16; r++) {
            const int row = m0 + wm0 + 32 * i + 8 * (r / 4) + 4 * lh + r % 4;
            if (row >= p.M) continue;
#pragma unroll
            for (int j = 0; j < NB; j++) {
                const int col = n0 + wn0 + 32 * j + li;
                if (col >= p.N) continue;
                if (p.splits > 1) {
                    auto *out = (decltype(acc[0][0][0] + 0) *)p.partial;
                    out[((size_t)split * p.M + row) * p.N + col] = acc[i][j][r];
                } else q8_finish(p, row, col, acc[i][j][r]);
            }
        }
}

template <class Op, int WM, int WN, int MB, int NB, int NS, int OCC>
__global__ void __launch_bounds__(64 * WM * WN, (OCC * WM * WN + 3) / 4) q8gemm_kernel(const Q8GemmParams p)
{
    __shared__ __attribute__((aligned(16))) unsigned char lds[NS * 32 * (MB * WM + NB * WN) * 128];
    int tile, split;
    if (!owt_split_major_wg(p.tiles, p.splits, tile, split)) return;
    q8gemm_tile<Op, WM, WN, MB, NB, NS>(p, tile, split, lds);
}

// Adds up the parts of a split sum, in order.
template <class S>
__global__ void __launch_bounds__(256) q8_join_kernel(const Q8GemmParams p)
{
    const size_t n = (size_t)p.M * p.N, stride = (size_t)gridDim.x * 256;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += stride) {
        S s = 0;
        for (int k = 0; k < p.splits; k++) s += ((const S *)p.partial)[(size_t)k * n + i];
        q8_finish(p, (int)(i / p.N), (int)(i % p.N), s);
    }
}

}  // namespace owt

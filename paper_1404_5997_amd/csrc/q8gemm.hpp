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
#include <type_traits>

#include "owt_common.hpp"
#include "q8piece.hpp"

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
    float least;                        // 0 with ReLU, else minus infinity
};
// Results of a backward product: row m was scaled by 2^exps[m]
struct Q8BwdOut {
    const int *exps;
    float alpha, beta;                  // beta only where results are fp32
};

struct Q8GemmParams {
    const unsigned char *a, *b;
    size_t lda, ldb;                    // bytes from row to row, multiples of 128
    int M, N, ksteps;                   // rows of C, columns of C, steps of A's rows
    int planes;                         // consecutive steps of A that meet the same step of B
    int tiles_n, splits, ksteps_per_split;
    int tiles;                          // tiles_m * tiles_n
    void *out;                          // C
    int bf16;                           // its type
    int big;                            // it is more than an eighth of the 256 MB behind the L2 caches
    void *partial;                      // [splits][M][N], 32 bits each (splits > 1)
    Q8FwdOut f;
    Q8BwdOut d;
};

// Four results C[m][c .. c + 3] of a row of N.  VEC: N is a multiple of four (then c is, too, and rows are aligned to four values).  Without
// it rows begin anywhere, which memory takes as well, and the last of them may be past the row.
struct __attribute__((packed, aligned(2))) Q8FourHalves { uint32_t lo, hi; };
template <bool VEC, class T> __device__ __forceinline__ void q8_store4(T *row, int c, int N, const float (&v)[4])
{
    if (VEC) {
        if (c >= N) return;
        if (sizeof(T) == 4) *(float4 *)((float *)row + c) = make_float4(v[0], v[1], v[2], v[3]);
        else *(uint2 *)((uint16_t *)row + c) = make_uint2(f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3]));
    } else if (c + 4 <= N) {
        if (sizeof(T) == 4) Piece<float>::store((float *)row + c, v);
        else {
            Q8FourHalves *to = (Q8FourHalves *)((uint16_t *)row + c);
            to->lo = f32x2_to_bf16x2(v[0], v[1]);
            to->hi = f32x2_to_bf16x2(v[2], v[3]);
        }
    } else {
#pragma unroll
        for (int t = 0; t < 3; t++)
            if (c + t < N) store1(row, (size_t)(c + t), v[t]);
    }
}
template <bool VEC> __device__ __forceinline__ void q8_load4(const float *row, int c, int N, float (&v)[4])
{
    if (VEC) {
        const float4 u = c < N ? *(const float4 *)(row + c) : make_float4(0.f, 0.f, 0.f, 0.f);
        v[0] = u.x; v[1] = u.y; v[2] = u.z; v[3] = u.w;
    } else load_piece<float>(row, c / 4, N, v);
}
// What four columns have in common for all rows, and a row for all columns: its scale, or its exponent.
struct Q8Cols { float ws[4], bias[4]; };
__device__ __forceinline__ Q8Cols q8_cols(const Q8GemmParams &p, int c, q8_i32x16)
{
    Q8Cols k = {};
    q8_load4<false>(p.f.ws, c, p.N, k.ws);
    if (p.f.bias) q8_load4<false>(p.f.bias, c, p.N, k.bias);
    return k;
}
__device__ __forceinline__ Q8Cols q8_cols(const Q8GemmParams &, int, q8_f32x16) { return {}; }
__device__ __forceinline__ int q8_row(const Q8GemmParams &p, int m, q8_i32x16) { return m < p.M ? __float_as_int(p.f.xs[m]) : 0; }
__device__ __forceinline__ int q8_row(const Q8GemmParams &p, int m, q8_f32x16) { return m < p.M ? p.d.exps[m] : 0; }

// Results from whole sums
__device__ __forceinline__ void q8_values(const Q8GemmParams &p, const Q8Cols &k, int row, const int (&sum)[4], float (&v)[4])
{
#pragma unroll
    for (int t = 0; t < 4; t++) {
        v[t] = (float)sum[t] * (__int_as_float(row) * k.ws[t]) + k.bias[t];
        v[t] = __builtin_elementwise_maximum(v[t], p.f.least);  // (NaN stays)
    }
}
__device__ __forceinline__ void q8_values(const Q8GemmParams &p, const Q8Cols &, int row, const float (&sum)[4], float (&v)[4])
{
#pragma unroll
    for (int t = 0; t < 4; t++) v[t] = ldexpf(sum[t], -row) * p.d.alpha;
}
// How results are written: at row + c
enum { Q8_PARTIAL, Q8_F32, Q8_F32_ADD, Q8_BF16, Q8_F32_ONCE, Q8_BF16_ONCE };     // ONCE: past the caches, where rows are whole fours
template <int HOW, bool VEC> __device__ __forceinline__ void q8_put(const Q8GemmParams &p, void *row, int c, float (&v)[4])
{
    if (HOW == Q8_BF16 || HOW == Q8_BF16_ONCE) q8_store4<VEC>((bf16_t *)row, c, p.N, v);
    else {
        if (HOW == Q8_F32_ADD) {
            float old[4];
            q8_load4<VEC>((float *)row, c, p.N, old);
#pragma unroll
            for (int t = 0; t < 4; t++) v[t] += p.d.beta * old[t];
        }
        q8_store4<VEC>((float *)row, c, p.N, v);
    }
}
// calls f(how, vec) with the constants of this product
template <class F> __device__ __forceinline__ void q8_how(const Q8GemmParams &p, bool partial, F f)
{
    using std::integral_constant;
    auto with = [&](auto vec) __attribute__((always_inline)) {
        if (decltype(vec)::value && p.big && !partial && (p.bf16 || p.d.beta == 0.f)) {
            if (p.bf16) f(integral_constant<int, Q8_BF16_ONCE>{}, vec);
            else f(integral_constant<int, Q8_F32_ONCE>{}, vec);
        } else if (partial) f(integral_constant<int, Q8_PARTIAL>{}, vec);
        else if (p.bf16) f(integral_constant<int, Q8_BF16>{}, vec);
        else if (p.d.beta != 0.f) f(integral_constant<int, Q8_F32_ADD>{}, vec);
        else f(integral_constant<int, Q8_F32>{}, vec);
    };
    if ((p.N & 3) == 0) with(integral_constant<bool, true>{});
    else with(integral_constant<bool, false>{});
}

// A wave-uniform address, in scalar registers
__device__ __forceinline__ const unsigned char *q8_uniform(const unsigned char *p)
{
    const unsigned long long a = (unsigned long long)p;
    const unsigned lo = (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)a), hi = (unsigned)__builtin_amdgcn_readfirstlane((int)(a >> 32));
    return (const unsigned char *)(((unsigned long long)hi << 32) | lo);
}

// 16 bytes a lane from base + off straight into LDS: lane l's land at byte address `dst` (wave-uniform, in m0) + 16 l; the s_nop is the wait
// state that the hardware wants between a scalar write of m0 and a load into LDS
__device__ __forceinline__ void q8_load_lds(unsigned off, const unsigned char *base, unsigned dst)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(off), "s"(base), "s"(__builtin_amdgcn_readfirstlane(dst)) : "memory", "m0");
}

// One tile of C over the steps of `split`: WM x WN wavefronts of MB x NB blocks of 32 x 32; lds: NS stages of both operands' tiles of a step.
//
// PAIRS: the steps of A go in pairs that meet the same step of B, and lds holds NS tiles of one operand, filled one by one in the order they
// are used.  256 x 256 results take 32 KB of either operand a step, so that two stages are all that LDS holds; this way B is loaded once for a
// pair, its fragments, read from LDS with the first plane, stay in registers for the second, and with five tiles a load has two products of
// a step to arrive in instead of less than one (dw of 8192 x 4096 -> 4096 432 us, 466 by stages, which are the faster ones where sums are short).
template <class Op, int WM, int WN, int MB, int NB, int NS, bool PAIRS>
__device__ __forceinline__ void q8gemm_tile(const Q8GemmParams &p, int tile, int split, unsigned char *lds)
{
    constexpr int NW = WM * WN, BM = 32 * MB * WM, BN = 32 * NB * WN;
    constexpr int AI = BM / 8 / NW, BI = BN / 8 / NW, L = AI + BI;     // loads of a wavefront and stage
    static_assert((BM / 8) % NW == 0 && (BN / 8) % NW == 0, "every wavefront issues the same number of loads");
    static_assert(NS >= 2 && (PAIRS ? 3 * AI : (NS - 1) * L) <= 63, "the wait counter has six bits");
    static_assert(!PAIRS || (BM == BN && NS == 5), "tiles of one size, five of them");
    constexpr int STAGE = PAIRS ? BM * 128 : (BM + BN) * 128;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int li = lane & 31, lh = lane >> 5;
    const int wm0 = (wave / WN) * 32 * MB, wn0 = (wave % WN) * 32 * NB;
    // tiles run down groups of 8 tile rows: the ones that are computed at a time then share rows and columns (of 1024 tiles of 256 x 256, an
    // XCD's 32 at a time read 12 tiles of operands from beyond its L2, row by row they would read 33)
    const int tiles_m = (p.M + BM - 1) / BM, first = tile / (8 * p.tiles_n) * 8, high = min(8, tiles_m - first);
    const int in_group = tile - first * p.tiles_n, tm = first + in_group % high, tn = in_group / high;
    const int m0 = tm * BM, n0 = tn * BN;
    const int ks_beg = split * p.ksteps_per_split;
    const int nst = min(p.ksteps, ks_beg + p.ksteps_per_split) - ks_beg;

    // byte offsets of this lane's pieces of a step from the tile's first row, in 32 bits (255 rows of up to 2^24 bytes: the host sees to it)
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

    const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char *)lds + wave * 1024;
    // the loads of step `ks` (past the last one: that again) into buffer `buf`: where from, and the i-th of them
    const unsigned char *ap, *bp;
    unsigned to;
    const int ks_end = ks_beg + nst - 1;
    auto aim = [&](int ks, int buf) __attribute__((always_inline)) {
        ks = __builtin_amdgcn_readfirstlane(min(ks, ks_end));
        ap = q8_uniform(ag + (size_t)ks * 128);
        bp = q8_uniform(bg + (size_t)(p.planes == 2 ? ks >> 1 : ks) * 128);
        to = lds0 + buf * STAGE;
    };
    auto load = [&](int i) __attribute__((always_inline)) {
        if (i < AI) q8_load_lds(asrc[i < AI ? i : 0], ap, to + NW * i * 1024);
        else q8_load_lds(bsrc[i < AI ? 0 : i - AI], bp, to + BM * 128 + NW * (i - AI) * 1024);
    };

    unsigned fr[4];                                 // this lane's piece of a fragment's row, for each slice of 32 bytes
#pragma unroll
    for (int kc = 0; kc < 4; kc++) fr[kc] = li * 128 + 16 * ((2 * kc + lh) ^ ((li >> 1) & 7));

    // what the results need besides the sums is on its way from the start
    constexpr int QW = 8 * NB, RT = (BM + 64 * NW - 1) / (64 * NW);     // 16-byte pieces of a wavefront's row of results; rows' scales of a thread
    const int q = lane % QW, c = n0 + wn0 + 4 * q;
    const Q8Cols k = q8_cols(p, c, typename Op::Acc());
    int scale[RT];
#pragma unroll
    for (int i = 0; i < RT; i++) scale[i] = q8_row(p, m0 + tid + i * 64 * NW, typename Op::Acc());

    typename Op::Acc acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; i++)
#pragma unroll
        for (int j = 0; j < NB; j++)
#pragma unroll
            for (int r = 0; r < 16; r++) acc[i][j][r] = 0;

    // A slice of 32 bytes: its products, and between them the reads of the next slice's fragments and, in a step's last one, loads.  The order is
    // kept as written: the compiler would gather the reads in front of the products that wait for them.
    constexpr int P = MB * NB;
    q8_i32x4 af[2][MB], bf[PAIRS ? 4 : 2][NB];
    auto read = [&](q8_i32x4 &to, int tile_at, int row, int kc) __attribute__((always_inline)) { to = *(const q8_i32x4 *)(lds + tile_at + row * 128 + fr[kc]); };
    // products of af[a] and bf[b]; reads f = 0 .. reads - 1 by `reader`, loads i = 0 .. loads - 1 by `loader`
    auto slice = [&](int a, int b, int reads, auto reader, int loads, auto loader) __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < P; t++) {
#pragma unroll
            for (int f = 0; f < MB + NB; f++)
                if (f < reads && f * P / reads == t) reader(f);
            acc[t / NB][t % NB] = Op::mul(bf[b][t % NB], af[a][t / NB], acc[t / NB][t % NB]);
#pragma unroll
            for (int i = 0; i < L; i++)
                if (i < loads && i * P / loads == t) loader(i);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto nothing = [](int) __attribute__((always_inline)) {};
    // s_waitcnt vmcnt(n) lgkmcnt(0), expcnt untouched; then the same of all wavefronts
#define OWT_ARRIVED(n) do { asm volatile("" ::: "memory"); __builtin_amdgcn_s_waitcnt(((n) & 15) | (((n) >> 4) << 14) | (7 << 4)); \
                            __builtin_amdgcn_s_barrier(); asm volatile("" ::: "memory"); } while (0)
    if constexpr (PAIRS) {
        const int pairs = nst / 2;
        auto place = [](int slot) __attribute__((always_inline)) { return slot * STAGE; };
        auto turn = [](int slot, int by) __attribute__((always_inline)) { slot += by; return slot >= 5 ? slot - 5 : slot; };
        auto a_from = [&](int ks) __attribute__((always_inline)) { return q8_uniform(ag + (size_t)__builtin_amdgcn_readfirstlane(min(ks, ks_beg + nst - 2 + (ks & 1))) * 128); };
        auto b_from = [&](int t) __attribute__((always_inline)) { return q8_uniform(bg + (size_t)__builtin_amdgcn_readfirstlane(ks_beg / 2 + min(t, pairs - 1)) * 128); };
        auto load_a = [&](const unsigned char *from, int slot, int i) __attribute__((always_inline)) { q8_load_lds(asrc[i], from, lds0 + place(slot) + NW * i * 1024); };
        auto load_b = [&](const unsigned char *from, int slot, int i) __attribute__((always_inline)) { q8_load_lds(bsrc[i], from, lds0 + place(slot) + NW * i * 1024); };
        if (nst > 0) {
            // B of pair t lies in slot 3 t, the two planes of A in 3 t + 1 and 3 t + 2 (modulo five).  Behind the first plane the first two of them
            // are the second plane of pair t + 1 and B of pair t + 2, behind the second the third is the first plane of pair t + 2.
            int sb = 0;
#pragma unroll
            for (int id = 0; id < 5; id++)
#pragma unroll
                for (int i = 0; i < AI; i++) {
                    if (id % 3 == 0) load_b(b_from(id / 3), id, i);
                    else load_a(a_from(ks_beg + 2 * (id / 3) + id % 3 - 1), id, i);
                }
            OWT_ARRIVED(3 * AI);
#pragma unroll
            for (int f = 0; f < MB; f++) read(af[0][f], place(1), wm0 + 32 * f, 0);
#pragma unroll
            for (int f = 0; f < NB; f++) read(bf[0][f], place(0), wn0 + 32 * f, 0);
            for (int t = 0; t < pairs; t++) {
                const int sh = turn(sb, 1), sm = turn(sb, 2), nb = turn(sb, 3), nh = turn(sb, 4);
#pragma unroll
                for (int kc = 0; kc < 3; kc++)
                    slice(kc & 1, kc, MB + NB, [&](int f) __attribute__((always_inline)) {
                        if (f < MB) read(af[(kc & 1) ^ 1][f < MB ? f : 0], place(sh), wm0 + 32 * f, kc + 1);
                        else read(bf[PAIRS ? kc + 1 : 0][f < MB ? 0 : f - MB], place(sb), wn0 + 32 * (f - MB), kc + 1);
                    }, 0, nothing);
                // The second plane is there, and everybody has the last fragments of the first and of B.  (The last pairs load the last one again, and
                // the very last reads fragments that nothing uses: a second copy of this code would take longer to arrive than that does.)
                OWT_ARRIVED(2 * AI);
                const unsigned char *fm = a_from(ks_beg + 2 * t + 3), *fb = b_from(t + 2), *fh = a_from(ks_beg + 2 * t + 4);
                slice(1, PAIRS ? 3 : 0, MB, [&](int f) __attribute__((always_inline)) { read(af[0][f < MB ? f : 0], place(sm), wm0 + 32 * f, 0); },
                      L, [&](int i) __attribute__((always_inline)) {
                          if (i < AI) load_a(fm, sb, i < AI ? i : 0);
                          else load_b(fb, sh, i < AI ? 0 : i - AI);
                      });
#pragma unroll
                for (int kc = 0; kc < 3; kc++)
                    slice(kc & 1, kc, MB, [&](int f) __attribute__((always_inline)) { read(af[(kc & 1) ^ 1][f < MB ? f : 0], place(sm), wm0 + 32 * f, kc + 1); }, 0, nothing);
                OWT_ARRIVED(2 * AI);
                slice(1, PAIRS ? 3 : 0, MB + NB, [&](int f) __attribute__((always_inline)) {
                    if (f < MB) read(af[0][f < MB ? f : 0], place(nh), wm0 + 32 * f, 0);
                    else read(bf[0][f < MB ? 0 : f - MB], place(nb), wn0 + 32 * (f - MB), 0);
                }, AI, [&](int i) __attribute__((always_inline)) { load_a(fh, sm, i < AI ? i : 0); });
                sb = nb;
            }
        }
    } else if (nst > 0) {
#pragma unroll
        for (int s = 0; s < NS; s++) {
            aim(ks_beg + s, s);
#pragma unroll
            for (int i = 0; i < L; i++) load(i);
        }
        OWT_ARRIVED((NS - 1) * L);
        auto reads = [&](int side, int kc, int buf) __attribute__((always_inline)) {
            return [&, side, kc, buf](int f) __attribute__((always_inline)) {
                if (f < MB) read(af[side][f < MB ? f : 0], buf * STAGE, wm0 + 32 * f, kc);
                else read(bf[side][f < MB ? 0 : f - MB], buf * STAGE, BM + wn0 + 32 * (f - MB), kc);
            };
        };
#pragma unroll
        for (int f = 0; f < MB + NB; f++) reads(0, 0, 0)(f);
        int cur = 0;                                // stage s lives in buffer s % NS
        for (int s = 0; s < nst; s++) {
            const int next = cur == NS - 1 ? 0 : cur + 1;
#pragma unroll
            for (int kc = 0; kc < 3; kc++) slice(kc & 1, kc & 1, MB + NB, reads((kc & 1) ^ 1, kc + 1, cur), 0, nothing);
            // stage s + 1 has landed and everybody has this stage's last fragments: its buffer is filled anew (the last ones as above)
            OWT_ARRIVED((NS - 2) * L);
            aim(ks_beg + s + NS, cur);
            slice(1, 1, MB + NB, reads(0, 0, next), L, load);
            cur = next;
        }
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);             // vmcnt(0): the last loads into LDS have landed, too
#undef OWT_ARRIVED

    // Accumulator register r of lane (li, lh): column 8 (r / 4) + 4 lh + r % 4 of C, row li of its block (the operands change places in the
    // instruction): four neighbouring results a lane.  They go through LDS, 32 rows of a wavefront at a time, so that rows are written as
    // runs of 32 NB values; 16-byte piece q of row r sits in slot q ^ (r % 16) (or % 8).  The rows' scales come from LDS, too: a scale read
    // from memory would wait for the stores before it.  A wavefront has its SIMD to itself here and an instruction
    // takes it 8 clocks, so they are few: no branch, no 64-bit address (the first form took 30000 clocks of the end of a 256 x 256 tile).
    typedef decltype(typename Op::Acc()[0] + 0) S;
    constexpr int SW = QW < 16 ? QW - 1 : 15;       // the bits of a row's swizzle
    static_assert(NS * STAGE >= NW * 32 * QW * 16 + BM * 4, "32 rows of each wavefront and the rows' scales fit the stages");
    unsigned char *mine = lds + wave * (32 * QW * 16);
    int *rows = (int *)(lds + NW * (32 * QW * 16));
    __syncthreads();                                // everybody has read the last stage
#pragma unroll
    for (int i = 0; i < RT; i++)
        if (tid + i * 64 * NW < BM) rows[tid + i * 64 * NW] = scale[i];
    __syncthreads();
    const unsigned width = (unsigned)p.N * (p.splits == 1 && p.bf16 ? 2 : 4);       // (rows of up to 2^24 bytes: 128 of them are addressed with 32 bits)
    char *base = (p.splits > 1 ? (char *)p.partial + (size_t)split * p.M * width : (char *)p.out) + (size_t)(m0 + wm0) * width;
    const int m_end = __builtin_amdgcn_readfirstlane(max(0, min(32 * MB, p.M - m0 - wm0)));     // rows of this wavefront that exist
    const unsigned char *src = mine + lane / QW * (QW * 16);
    const int *factor = rows + wm0 + lane / QW;
    // Lanes read what others of their wavefront wrote, and write where others read.  LDS takes a wavefront's accesses in order; this keeps the
    // compiler to that order, too, and is no instruction.
    auto in_order = [] __attribute__((always_inline)) () {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    };
#pragma unroll
    for (int i = 0; i < MB; i++) {
        if (i > 0) in_order();
#pragma unroll
        for (int j = 0; j < NB; j++)
#pragma unroll
            for (int g = 0; g < 4; g++) {
                q8_i32x4 v;
#pragma unroll
                for (int t = 0; t < 4; t++) {
                    const S u = acc[i][j][4 * g + t];       // (a bit cast of the element in place takes the vector's first)
                    v[t] = __builtin_bit_cast(int, u);
                }
                *(q8_i32x4 *)(mine + (li * QW + ((8 * j + 2 * g + lh) ^ (li & SW))) * 16) = v;
            }
        in_order();
        q8_how(p, p.splits > 1, [&](auto how, auto vec) __attribute__((always_inline)) {
            constexpr int HOW = decltype(how)::value;
            constexpr bool HALF = HOW == Q8_BF16 || HOW == Q8_BF16_ONCE;
            constexpr int PAST = HOW == Q8_BF16_ONCE || HOW == Q8_F32_ONCE ? 2 : 0;       // (the operands are read again and stay in the caches: 8192 x 4096 -> 8192 in bf16 239 us, 246 without)
            // whole fours: through a descriptor that ends with the last row, where what lies outside is not written
            const __amdgpu_buffer_rsrc_t rs = owt_make_rsrc(q8_uniform((const unsigned char *)base), (unsigned)m_end * width);
            unsigned at = c < p.N ? (unsigned)(32 * i + lane / QW) * width + (unsigned)c * (HALF ? 2 : 4) : 0x80000000u;
            const unsigned step = c < p.N ? (64 / QW) * width : 0;
#pragma nounroll
            for (int it = 0; it < QW / 2; it += 4) {        // four rows' reads at a time, then their results
                q8_i32x4 w[4];
                int f[4];
#pragma unroll
                for (int u = 0; u < 4; u++) {
                    const int r = (it + u) * (64 / QW);
                    w[u] = *(const q8_i32x4 *)(src + r * (QW * 16) + (q ^ ((r + lane / QW) & SW)) * 16);
                    f[u] = factor[32 * i + r];
                }
#pragma unroll
                for (int u = 0; u < 4; u++) {
                    float v[4];
                    S sum[4];
#pragma unroll
                    for (int t = 0; t < 4; t++) {
                        const int e = w[u][t];
                        sum[t] = __builtin_bit_cast(S, e);
                        v[t] = __int_as_float(e);           // (a part of a sum: 32 bits as they are)
                    }
                    if (HOW != Q8_PARTIAL) q8_values(p, k, f[u], sum, v);
                    if (decltype(vec)::value) {
                        if (HOW == Q8_F32_ADD) {
                            const float4 old = buffer_load4(rs, at);
                            v[0] += p.d.beta * old.x; v[1] += p.d.beta * old.y; v[2] += p.d.beta * old.z; v[3] += p.d.beta * old.w;
                        }
                        if (HALF) {
                            const owt_u32x2 o = {f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3])};
                            __builtin_amdgcn_raw_buffer_store_b64(o, rs, (int)at, 0, PAST);
                        } else {
                            const owt_u32x4 o = {__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
                            __builtin_amdgcn_raw_buffer_store_b128(o, rs, (int)at, 0, PAST);
                        }
                        at += step;
                    } else {
                        const int m = 32 * i + (it + u) * (64 / QW) + lane / QW;
                        if (m < m_end) q8_put<HOW, false>(p, base + (size_t)m * width, c, v);
                    }
                }
            }
        });
    }
}

template <class Op, int WM, int WN, int MB, int NB, int NS, bool PAIRS, int OCC>
__global__ void __launch_bounds__(64 * WM * WN, (OCC * WM * WN + 3) / 4) q8gemm_kernel(const Q8GemmParams p)
{
    __shared__ __attribute__((aligned(16))) unsigned char lds[NS * 32 * (MB * WM + (PAIRS ? 0 : NB * WN)) * 128];
    int tile, split;
    if (!owt_split_major_wg(p.tiles, p.splits, tile, split)) return;
    q8gemm_tile<Op, WM, WN, MB, NB, NS, PAIRS>(p, tile, split, lds);
}

// Both backward products in one launch, neither split: the one of longer sums first.
template <int WM, int WN, int MB, int NB, int NS, int OCC>
__global__ void __launch_bounds__(64 * WM * WN, (OCC * WM * WN + 3) / 4) q8gemm_pair_kernel(const Q8GemmParams p0, const Q8GemmParams p1)
{
    __shared__ __attribute__((aligned(16))) unsigned char lds[NS * 32 * (MB * WM + NB * WN) * 128];
    const int first = owt_split_major_grid(p0.tiles, 1), b = (int)blockIdx.x;
    // (the numbering of owt_split_major_wg, within a product's work-groups: their number is a multiple of 8)
    auto run = [&](const Q8GemmParams &p, int l) __attribute__((always_inline)) {
        const int xcd = l & 7, jx = l >> 3, each = p.tiles >> 3, more = p.tiles & 7;
        if (jx < each + (xcd < more ? 1 : 0)) q8gemm_tile<Q8Half, WM, WN, MB, NB, NS, false>(p, xcd * each + min(xcd, more) + jx, 0, lds);
    };
    if (b < first) run(p0, b);
    else run(p1, b - first);
}

// Adds up the parts of a split sum, in order: four columns a thread.
template <class Op>
__global__ void __launch_bounds__(256) q8_join_kernel(const Q8GemmParams p)
{
    typedef decltype(typename Op::Acc()[0] + 0) S;
    const unsigned quads = (unsigned)(p.N + 3) / 4;
    const size_t n = (size_t)p.M * quads, stride = (size_t)gridDim.x * 256, whole = (size_t)p.M * p.N;
    q8_how(p, false, [&](auto how, auto vec) __attribute__((always_inline)) {
        constexpr bool VEC = decltype(vec)::value;
        for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += stride) {
            const int m = (int)(i / quads), c = (int)(i % quads) * 4;
            const float *part = (const float *)p.partial + (size_t)m * p.N;
            S s[4] = {};
#pragma unroll 4
            for (int k = 0; k < p.splits; k++) {
                float v[4];
                q8_load4<VEC>(part + k * whole, c, p.N, v);
#pragma unroll
                for (int t = 0; t < 4; t++) s[t] += __builtin_bit_cast(S, v[t]);
            }
            float v[4];
            q8_values(p, q8_cols(p, c, typename Op::Acc()), q8_row(p, m, typename Op::Acc()), s, v);
            q8_put<decltype(how)::value, VEC>(p, (char *)p.out + (size_t)m * p.N * (p.bf16 ? 2 : 4), c, v);
        }
    });
}

}  // namespace owt

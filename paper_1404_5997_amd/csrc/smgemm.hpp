// Matrix products of softmax cross-entropy on the 16-bit matrix instructions, and what happens to their results before they leave the chip.
//
//   outputs   z[n][o]  = sum_i x[n][i] w[o][i]       leave as each row's largest value and sum of exponentials, or as gradients dz
//   dx[n][i]  = sum_o dz[n][o] w[o][i]
//   dw[o][i]  = sum_n dz[n][o] x[n][i]
//
// A softmax needs of its outputs, forward, the running maximum m of a row and sum s of exp(z - m): two such pairs join as (max, s1 exp(m1 - max) + s2 exp(m2 - max)), so that
// a tile's 256 outputs of a row leave as 16 bytes.  Backward dz comes from the outputs and the joined log of the sum alone, element by element.
//
// All three are C[m][c] = sum_k A[m][k] B[c][k] with operands as they lie in memory: "along" where k is contiguous (x and w of the outputs, dz of
// dx), "across" where rows of memory are k and m or c is contiguous (w of dx; dz and x of dw).  A step is 64 values of k.  Of an operand along it takes 128
// bytes of each row, across it 64 rows: 128 bytes for each of a tile's rows of C either way, which go straight into LDS, 1 KB an instruction, into a ring of NS
// stages.  Fragments of v_mfma_f32_32x32x16_{bf16,f16} are 8 values of k of a row a lane: 16 consecutive bytes along (16-byte piece c of row r sits in slot
// c ^ ((r >> 1) & 7), which spreads 32 rows over all banks), two transposing reads across (four rows of k by 16 columns each; piece c of row k
// sits in slot c ^ 4 (k % 4), so that those four rows lie in different banks).
//
// An operand may have planes, in rows of [step][plane][64 values]: values as sums of two.  A step of memory is then several steps here.
//
// Operands end anywhere: rows of memory past the end re-read the last one, columns the last piece of eight.  What is multiplied wrongly by
// that is not stored, or meets zeros: along k, x and w have them up to a whole step, and dz; across, x has rows of them up to a whole step (and w meets dz's).
//
// fp32 values are two f16 ones, of the value times 2^e, e of its row: the row's largest magnitude then lies in [2^14, 2^15).  A result's sums are of values
// times 2^(e of its row + e of its column).
// What bounds it: power on large products, 1.22 to 1.31 PFLOP/s with the forward pass's end (8192 rows 4096 -> 32768 in 1680 to 1800 us, the library's product alone
// runs at 1.31), 1.39 for dw's pairs, 1.30 for dx's, 1.15 where outputs leave as dz (a tenth of a tile's time is its end: 16 K exponentials a wavefront, two bf16 values each).  Few
// rows: memory (one row 4096 -> 65536 104 us, 5.4 TB/s of weights).  256 x 256 results a work-group of four wavefronts read 64 bytes a clock from LDS for 512 clocks of
// the matrix unit a slice, half of what LDS gives; smaller tiles read more and serve sizes with few tiles.
#pragma once
#include <type_traits>

#include "owt_common.hpp"

namespace owt {

typedef float sm_f32x16 __attribute__((ext_vector_type(16)));
typedef int sm_i32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 sm_f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 sm_bf16x8 __attribute__((ext_vector_type(8)));
typedef short sm_i16x4 __attribute__((ext_vector_type(4)));

struct SmBf16 {
    static __device__ __forceinline__ sm_f32x16 mul(sm_i32x4 a, sm_i32x4 b, sm_f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(sm_bf16x8, a), __builtin_bit_cast(sm_bf16x8, b), c, 0, 0, 0);
    }
};
struct SmHalf {
    static __device__ __forceinline__ sm_f32x16 mul(sm_i32x4 a, sm_i32x4 b, sm_f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(sm_f16x8, a), __builtin_bit_cast(sm_f16x8, b), c, 0, 0, 0);
    }
};

__device__ __forceinline__ bool has_class(int label, int classes) { return (unsigned)label < (unsigned)classes; }

// The largest output of a row and the sum of exponentials below it, joined with another such pair.  A pair without outputs is (-inf, 0); outputs
// of -inf add nothing; +inf and NaN leave as infinity and NaN.
struct Top { float max, sum; };
__device__ __forceinline__ Top top_of(float v) { return {v == v ? v : 0.f, v == -INFINITY ? 0.f : v == INFINITY || v != v ? v : 1.f}; }
__device__ __forceinline__ float exp_of(float v) { return __builtin_amdgcn_exp2f(v * 1.44269504088896341f); }
__device__ __forceinline__ Top join(Top a, Top b)
{
    const float m = fmaxf(a.max, b.max), at = __builtin_isfinite(m) ? m : 0.f;
    return {m, a.sum * (a.max == m ? 1.f : exp_of(a.max - at)) + b.sum * (b.max == m ? 1.f : exp_of(b.max - at))};
}

struct SmOperand {
    const unsigned char *at;
    size_t ld;              // bytes from row to row of memory
    size_t step;            // bytes from step to step: along 128 a plane, across 64 rows
    int rows;               // rows of memory, of m or c (along) or of k (across)
    int pieces;             // across: pieces of eight values of a row
    int planes;
};

// products of a step of memory: one; two planes of A with B; three planes of A with B, or where A has two the three larger of both planes of both
enum { SM_ONE = 1, SM_PAIR = 2, SM_THREE = 3 };

// Rows of x or w laid out for the products: whole steps of 64 values, zeros behind the last one, and zeros for rows without a class (labels null: all have one).
struct SmPrep {
    const void *from;           // [rows][cols]
    unsigned char *to;          // out_rows rows of `steps` steps
    int rows, out_rows, cols, steps;
    const int *labels;
    int classes;
    const float *weight;        // of the rows, or null
    int *exps, *lows;           // fp32: each row's exponent, and the least of a work-group's rows, less those of their weights
};

struct SmParams {
    SmOperand a, b;
    int M, N;               // C
    int products, steps;    // steps here: products times those of memory
    int tiles_n, tiles, splits, steps_per_split;
    // outputs: bias of a column, or null; exponents of rows and columns (f16 values)
    const float *bias;
    const int *row_exp, *col_exp;
    const int *labels;      // of row m (null: every row counts); column `label - off` is its own, classes [0, classes) exist
    int off, classes;
    // forward: pairs [tiles_n * wavefronts along c][M], the labels' outputs
    Top *top;
    float *target;
    // backward: the whole layer's lse, weights or null; dz [M][step][2][64] (f16 values: one for dw and one for dx, with the least exponent of x's rows with their
    // weights and that of w's rows)
    const float *lse, *weight;
    unsigned char *dz, *dz_dx;
    size_t dz_ld;
    int dz_step;            // bytes of 64 classes: 128 a plane
    const int *lows_x, *lows_w; // what the least exponents are the least of
    int num_x, num_w;
    int *least;                 // [0] of x, [1] of w: for the products that follow
    SmPrep copy;                // bf16: x for dw, by work-groups behind the tiles' (out_rows 0: none)
    float *dbias;               // sums over the rows of each wavefront [..][N]; dw: [strips][M], summed up to db
    int strips;
    float *db;
    // results
    void *out;              // C, rows of N values
    int bf16;               // its type
    int big;                // it is more than an eighth of the 256 MB behind the L2 caches
    float alpha, beta;      // beta only where results are fp32
    const float *add;       // fp32 [M][N] that is added to alpha times the sum (may be out), or null
    const int *under;       // (f16 values) results are the sums times 2^-(*under + kSmDzTop)
    float *partial;         // [splits][M][N] (splits > 1)
};
constexpr int kSmTop = 14;          // a row's largest magnitude is scaled to [2^14, 2^15)
constexpr int kSmDzTop = 15;        // and dz to 2^15 for what is 1 with its factors
// f16 values end at 65504: an exponential counts as this at most.  It is 1 at most but for the outputs' errors, which are that large for outputs from some 2^22 on.
constexpr float kSmDzMost = 65504.f / 32768.f;
constexpr int kSmNone = 1 << 20;    // the exponent of a row of zeros

// What a row of dx is multiplied by: 0 without a class; with f16 values dz came without its weight
template <bool HALF> __device__ __forceinline__ float sm_row_factor(const SmParams &p, int m)
{
    if (!p.labels) return 1.f;
    if (m >= p.M || !has_class(p.labels[m], p.classes)) return 0.f;
    return HALF && p.weight ? p.weight[m] : 1.f;
}

// A wave-uniform address, in scalar registers
__device__ __forceinline__ const unsigned char *sm_uniform(const unsigned char *p)
{
    const unsigned long long a = (unsigned long long)p;
    const unsigned lo = (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)a), hi = (unsigned)__builtin_amdgcn_readfirstlane((int)(a >> 32));
    return (const unsigned char *)(((unsigned long long)hi << 32) | lo);
}
// 16 bytes a lane from base + off straight into LDS: lane l's land at byte address `dst` (wave-uniform, in m0) + 16 l; the s_nop is the wait
// state that the hardware wants between a scalar write of m0 and a load into LDS
__device__ __forceinline__ void sm_load_lds(unsigned off, const unsigned char *base, unsigned dst)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(off), "s"(base), "s"(__builtin_amdgcn_readfirstlane(dst)) : "memory", "m0");
}

enum { SM_TOP, SM_DZ, SM_OUT };

// RING: 0, NS stages of both operands' tiles of a step.  SM_PAIR, SM_THREE: the products of a step of memory go together, and LDS holds five tiles of one
// operand, filled one by one in the order they are used.  256 x 256 results take 32 KB of either operand a step, so that two stages are all that LDS holds; this way a
// step of memory loads three tiles for two products, or four for three, instead of four and six, a tile that two products use is read from LDS once and stays in
// registers for the other, and a load has two products to arrive in.
template <int WM_, int WN_, int MB_, int NB_, int NS_, int OCC_, int RING_ = 0> struct SmShape {
    static constexpr int WM = WM_, WN = WN_, MB = MB_, NB = NB_, NS = NS_, OCC = OCC_, RING = RING_, NW = WM * WN, BM = 32 * MB * WM, BN = 32 * NB * WN;
    static constexpr int STAGE = RING_ ? BM * 128 : (BM + BN) * 128, TILES = NS * STAGE, LDS = TILES + (RING_ ? 0 : (BM + BN) * 4);
};

// The pieces of a tile of R rows of C that a lane loads, and where a fragment's lane reads.
template <bool ACROSS, int R, int NW> struct SmTile {
    static constexpr int LOADS = R / 8 / NW, PIECES = R / 8;       // pieces of a row across
    static_assert((R / 8) % NW == 0, "every wavefront issues the same number of loads");
    static __device__ __forceinline__ int turned(int k) { return R >= 128 ? 4 * (k & 3) : R == 64 ? 4 * ((k >> 1) & 1) : 0; }
    // offset of this lane's piece of load i from the first byte of the tile's step; `left`: rows of memory that exist from there on; c0: first column
    static __device__ __forceinline__ unsigned from(const SmOperand &o, int wave, int lane, int i, int c0, int left)
    {
        if (ACROSS) {
            const int q = 64 * (wave + NW * i) + lane, k = q / PIECES, piece = min(c0 / 8 + ((q % PIECES) ^ turned(k)), o.pieces - 1);
            return (unsigned)min(k, left - 1) * (unsigned)o.ld + (unsigned)(piece >> 3) * (unsigned)(o.planes * 128) + 16 * (piece & 7);
        }
        const int row = 8 * (wave + NW * i) + (lane >> 3), piece = (lane & 7) ^ ((row >> 1) & 7);
        return (unsigned)min(row, left - 1) * (unsigned)o.ld + 16 * piece;
    }
};

// dz = weight (exp(z - lse) - [label]): what a row and four columns bring to it, and what is kept.  Rows without a class are zeros (they have no weight), and so are
// columns past the last up to a whole step: a bias of -infinity takes exponentials to zero.  (Rows all of whose outputs are -infinity
// have an lse of -infinity: any other number will do in its place.)
struct SmDzRow { float lse, weight; int label, exp; };      // exp: of x's row
struct SmDzColumns { float bias[4]; int exp[4]; };          // exp: of w's rows
template <bool SCALED> __device__ __forceinline__ SmDzRow sm_dz_row(const SmParams &p, int m)
{
    const int at = m < p.M ? p.labels[m] : -1;
    if (m >= p.M || !has_class(at, p.classes)) return {INFINITY, 0.f, -1, 0};
    const float lse = p.lse[m];
    // (a label behind these columns is no column of the last step's zeros, either)
    return {lse == -INFINITY ? 0.f : lse, p.weight ? p.weight[m] : 1.f, at - p.off < p.N ? at - p.off : -1, SCALED ? p.row_exp[m] : 0};
}
template <bool SCALED> __device__ __forceinline__ SmDzColumns sm_dz_columns(const SmParams &p, int c)
{
    SmDzColumns k;
#pragma unroll
    for (int t = 0; t < 4; t++) {
        k.bias[t] = c + t < p.N ? (p.bias ? p.bias[c + t] : 0.f) : -INFINITY;
        k.exp[t] = !SCALED ? 0 : c + t < p.N ? p.col_exp[c + t] : kSmNone;
    }
    return k;
}
__device__ __forceinline__ uint32_t sm_halves(float lo, float hi)
{
    typedef _Float16 Two __attribute__((ext_vector_type(2)));
    const Two v = {(_Float16)lo, (_Float16)hi};
    return __builtin_bit_cast(uint32_t, v);
}
// four values as two f16 ones each, 128 bytes apart
__device__ __forceinline__ void sm_put_halves(unsigned char *to, const float (&v)[4])
{
    float lo[4];
#pragma unroll
    for (int t = 0; t < 4; t++) lo[t] = v[t] - (float)(_Float16)v[t];
    *(uint2 *)to = make_uint2(sm_halves(v[0], v[1]), sm_halves(v[2], v[3]));
    *(uint2 *)(to + 128) = make_uint2(sm_halves(lo[0], lo[1]), sm_halves(lo[2], lo[3]));
}
// and as two bf16 ones, or three
__device__ __forceinline__ void sm_put_bf16s(unsigned char *to, const float (&v)[4], bool three)
{
    const uint2 hi = make_uint2(f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3]));
    const float lo[4] = {v[0] - __uint_as_float(hi.x << 16), v[1] - __uint_as_float(hi.x & 0xffff0000u), v[2] - __uint_as_float(hi.y << 16),
                         v[3] - __uint_as_float(hi.y & 0xffff0000u)};
    *(uint2 *)to = hi;
    const uint2 second = make_uint2(f32x2_to_bf16x2(lo[0], lo[1]), f32x2_to_bf16x2(lo[2], lo[3]));
    *(uint2 *)(to + 128) = second;
    if (three)
        *(uint2 *)(to + 256) = make_uint2(f32x2_to_bf16x2(lo[0] - __uint_as_float(second.x << 16), lo[1] - __uint_as_float(second.x & 0xffff0000u)),
                                          f32x2_to_bf16x2(lo[2] - __uint_as_float(second.y << 16), lo[3] - __uint_as_float(second.y & 0xffff0000u)));
}
// The least exponents of x's rows with their weights and of w's, found by the work-group for itself; `first` leaves them to the products that follow.
// two: eight words of LDS that nothing else is in.
__device__ __forceinline__ int2 sm_leasts(const SmParams &p, int *two, bool first)
{
    int x = kSmNone, w = kSmNone;
    for (int i = threadIdx.x; i < p.num_x; i += 256) x = min(x, p.lows_x[i]);
    for (int i = threadIdx.x; i < p.num_w; i += 256) w = min(w, p.lows_w[i]);
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
        x = min(x, __shfl_xor(x, d, 64));
        w = min(w, __shfl_xor(w, d, 64));
    }
    if ((threadIdx.x & 63) == 0) {
        two[threadIdx.x >> 6] = x;
        two[4 + (threadIdx.x >> 6)] = w;
    }
    __syncthreads();
    const int2 v = make_int2(min(min(two[0], two[1]), min(two[2], two[3])), min(min(two[4], two[5]), min(two[6], two[7])));
    if (first && threadIdx.x == 0) {
        p.least[0] = v.x;
        p.least[1] = v.y;
    }
    return v;
}

// STARTED: sums that began at bias - lse / 2.  All lanes of a wavefront come here together.
template <bool SCALED, bool STARTED>
__device__ __forceinline__ void sm_dz(const SmParams &p, int2 least, int m, int c, const float4 &sum, const SmDzRow &w, const SmDzColumns &k, float (&sums)[4])
{
    const float u[4] = {sum.x, sum.y, sum.z, sum.w};
    float d[4], e[4];
#pragma unroll
    for (int t = 0; t < 4; t++) {
        const float from_lse = STARTED ? u[t] - 0.5f * w.lse : (SCALED ? ldexpf(u[t], -(w.exp + k.exp[t])) : u[t]) + k.bias[t] - w.lse;
        e[t] = w.weight == 0.f ? 0.f : exp_of(from_lse);        // (a row without a class may hold anything, and bf16 outputs are of x as it lies)
        if (SCALED) e[t] = e[t] > kSmDzMost ? kSmDzMost : e[t];  // (NaN stays)
    }
    if (__any((unsigned)(w.label - c) < 4u))        // (of many classes hardly ever)
#pragma unroll
        for (int t = 0; t < 4; t++) e[t] = w.label == c + t ? e[t] - 1.f : e[t];
#pragma unroll
    for (int t = 0; t < 4; t++) {
        d[t] = w.weight * e[t];
        sums[t] += d[t];
    }
    if (m >= p.M || c >= (p.N + 63) / 64 * 64) return;
    const size_t at = (size_t)m * p.dz_ld + (size_t)(c >> 6) * (SCALED ? 256 : p.dz_step) + 2 * (c & 63);
    if (SCALED) {
        const int ex = kSmDzTop - (w.exp - least.x), lw = least.y + kSmDzTop;
#pragma unroll
        for (int t = 0; t < 4; t++) {
            d[t] = ldexpf(d[t], ex);
            e[t] = ldexpf(e[t], lw - k.exp[t]);
        }
        sm_put_halves(p.dz + at, d);
        sm_put_halves(p.dz_dx + at, e);
    } else sm_put_bf16s(p.dz + at, d, p.dz_step == 384);
}

struct __attribute__((packed, aligned(2))) SmFourHalves { uint32_t lo, hi; };

// A result from its sum
template <bool SCALED> __device__ __forceinline__ void sm_result(float (&v)[4], int shift, float factor, float alpha)
{
#pragma unroll
    for (int t = 0; t < 4; t++) {
        const float u = SCALED ? ldexpf(v[t], shift) : v[t];
        v[t] = factor == 0.f ? 0.f : u * (factor * alpha);
    }
}

template <class Op, bool TA, bool TB, class S, int END>
__device__ __forceinline__ void sm_tile(const SmParams &p, int tile, int split, unsigned char *lds)
{
    constexpr int WN = S::WN, MB = S::MB, NB = S::NB, NS = S::NS, NW = S::NW, BM = S::BM, BN = S::BN, STAGE = S::STAGE;
    typedef SmTile<TA, BM, NW> LoadA;
    typedef SmTile<TB, BN, NW> LoadB;
    constexpr int AI = LoadA::LOADS, BI = LoadB::LOADS, L = AI + BI;
    static_assert(NW == 4, "256 threads");
    static_assert(S::RING || (NS >= 2 && (NS - 1) * L <= 63), "the wait counter has six bits");
    static_assert(!S::RING || (BM == BN && NS == 5 && 3 * AI <= 63), "tiles of one size, five of them");

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int li = lane & 31, lh = lane >> 5;
    const int wm = wave / WN, wn = wave % WN, wm0 = wm * 32 * MB, wn0 = wn * 32 * NB;
    // tiles run down groups of 8 tile rows: the ones that are computed at a time then share rows and columns
    const int tiles_m = (p.M + BM - 1) / BM, first = tile / (8 * p.tiles_n) * 8, high = min(8, tiles_m - first);
    const int in_group = tile - first * p.tiles_n, tm = first + in_group % high, tn = in_group / high;
    const int m0 = tm * BM, n0 = tn * BN;
    const int s_beg = split * p.steps_per_split, nst = min(p.steps, s_beg + p.steps_per_split) - s_beg, s_end = s_beg + nst - 1;

    unsigned asrc[AI], bsrc[BI];
    const unsigned char *ag, *bg;
    if (TA) ag = p.a.at; else ag = sm_uniform(p.a.at + (size_t)m0 * p.a.ld);
    if (TB) bg = p.b.at; else bg = sm_uniform(p.b.at + (size_t)n0 * p.b.ld);
#pragma unroll
    for (int i = 0; i < AI; i++) asrc[i] = LoadA::from(p.a, wave, lane, i, m0, TA ? 64 : p.a.rows - m0);
#pragma unroll
    for (int i = 0; i < BI; i++) bsrc[i] = LoadB::from(p.b, wave, lane, i, n0, TB ? 64 : p.b.rows - n0);

    const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char *)lds + wave * 1024;
    // the loads of step `s` (past the last one: that again) into buffer `buf`: where from, and the i-th of them
    const unsigned char *ap, *bp;
    unsigned to;
    auto aim = [&](int s, int buf) __attribute__((always_inline)) {
        s = __builtin_amdgcn_readfirstlane(min(s, s_end));
        int t = s, pa = 0, pb = 0;
        if (p.products == SM_PAIR) {
            t = s >> 1;
            pa = s & 1;
        } else if (p.products == SM_THREE) {
            t = s / 3;
            const int i = s - 3 * t;
            pa = p.a.planes == 3 ? i : i == 2;
            pb = p.a.planes == 3 ? 0 : i == 1;
        }
        // the last rows of k: what is loaded behind them is the same step's
        if (TA && 64 * t + 64 > p.a.rows) {
#pragma unroll
            for (int i = 0; i < AI; i++) asrc[i] = LoadA::from(p.a, wave, lane, i, m0, p.a.rows - 64 * t);
        }
        if (TB && 64 * t + 64 > p.b.rows) {
#pragma unroll
            for (int i = 0; i < BI; i++) bsrc[i] = LoadB::from(p.b, wave, lane, i, n0, p.b.rows - 64 * t);
        }
        ap = sm_uniform(ag + (size_t)t * p.a.step + 128 * pa);
        bp = sm_uniform(bg + (size_t)t * p.b.step + 128 * pb);
        to = lds0 + buf * STAGE;
    };
    auto load = [&](int i) __attribute__((always_inline)) {
        if (i < AI) sm_load_lds(asrc[i < AI ? i : 0], ap, to + NW * i * 1024);
        else sm_load_lds(bsrc[i < AI ? 0 : i - AI], bp, to + BM * 128 + NW * (i - AI) * 1024);
    };

    // where this lane reads a fragment: along its piece of a row for each slice of 16 k, across its quarter of a row for each 32 rows of C
    unsigned along[4], acrossA[MB], acrossB[NB];
#pragma unroll
    for (int kc = 0; kc < 4; kc++) along[kc] = li * 128 + 16 * ((2 * kc + lh) ^ ((li >> 1) & 7));
    const int l16 = lane & 15, k4 = l16 >> 2;
    auto cross = [&](int c, int rows) __attribute__((always_inline)) {      // column c, a multiple of 32, of a tile of `rows` columns
        const int turned = rows >= 128 ? 4 * k4 : rows == 64 ? 4 * (k4 >> 1) : 0;
        return (unsigned)((8 * lh + k4) * rows * 2 + (((c >> 3) + 2 * ((lane >> 4) & 1) + ((l16 & 3) >> 1)) ^ turned) * 16 + 8 * (l16 & 1));
    };
#pragma unroll
    for (int f = 0; f < MB; f++) acrossA[f] = cross(wm0 + 32 * f, BM);
#pragma unroll
    for (int f = 0; f < NB; f++) acrossB[f] = cross(wn0 + 32 * f, BN);
    auto read_across = [&](unsigned at, int pitch) __attribute__((always_inline)) {
        typedef __attribute__((address_space(3))) sm_i16x4 Local;
        const sm_i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Local *)(lds + at)), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Local *)(lds + at + 4 * pitch));
        typedef int Two __attribute__((ext_vector_type(2)));
        const Two l = __builtin_bit_cast(Two, lo), h = __builtin_bit_cast(Two, hi);
        return sm_i32x4{l[0], l[1], h[0], h[1]};
    };

    const bool some = END != SM_OUT || nst > 0;     // (split sums alone may have none here)
    if (!S::RING && some)
#pragma unroll
        for (int s = 0; s < NS; s++) {
            aim(s_beg + s, s);
#pragma unroll
            for (int i = 0; i < L; i++) load(i);
        }

    // Sums of outputs in bf16 start at what is added to them anyhow, while the first operands are on their way: the columns' bias (-infinity for those that
    // do not exist), and for dz less half of the rows' lse.  A sum's roundings go by its size on the way: of an output near lse, whose dz is a small difference, it
    // runs from -lse / 2 to lse / 2 then and is rounded half as coarsely.
    constexpr bool SCALED = std::is_same<Op, SmHalf>::value, STARTED = !SCALED && END != SM_OUT;
    sm_f32x16 acc[MB][NB];
    if (STARTED) {
        float *bias = (float *)(lds + S::TILES), *half = bias + BN;      // (each read from memory once, and not by every lane for itself: 45 us of 250 in a launch of 512 tiles)
        for (int c = tid; c < BN; c += 64 * NW) bias[c] = n0 + c < p.N ? (p.bias ? p.bias[n0 + c] : 0.f) : -INFINITY;
        if (END == SM_DZ)
            for (int r = tid; r < BM; r += 64 * NW) half[r] = 0.5f * sm_dz_row<false>(p, m0 + r).lse;
        __syncthreads();
        float less[MB];
#pragma unroll
        for (int i = 0; i < MB; i++) less[i] = END == SM_DZ ? half[wm0 + 32 * i + li] : 0.f;
#pragma unroll
        for (int j = 0; j < NB; j++)
#pragma unroll
            for (int g = 0; g < 4; g++) {
                const float4 b = *(const float4 *)(bias + wn0 + 32 * j + 8 * g + 4 * lh);
#pragma unroll
                for (int i = 0; i < MB; i++) {
                    acc[i][j][4 * g] = b.x - less[i];
                    acc[i][j][4 * g + 1] = b.y - less[i];
                    acc[i][j][4 * g + 2] = b.z - less[i];
                    acc[i][j][4 * g + 3] = b.w - less[i];
                }
            }
    } else {
#pragma unroll
        for (int i = 0; i < MB; i++)
#pragma unroll
            for (int j = 0; j < NB; j++)
#pragma unroll
                for (int r = 0; r < 16; r++) acc[i][j][r] = 0;
    }

    // A slice of 16 k: its products, and between them the reads of the next slice's fragments and, in a step's last one, loads.  The order is
    // kept as written: the compiler would gather the reads in front of the products that wait for them.
    constexpr int P = MB * NB;
    sm_i32x4 af[2][MB], bf[2][NB];
    auto read = [&](int side, int kc, int buf, int f) __attribute__((always_inline)) {
        if (f < MB) {
            const int g = f < MB ? f : 0;
            if (TA) af[side][g] = read_across(buf * STAGE + kc * 32 * BM + acrossA[g], 2 * BM);
            else af[side][g] = *(const sm_i32x4 *)(lds + buf * STAGE + (wm0 + 32 * g) * 128 + along[kc]);
        } else {
            const int g = f < MB ? 0 : f - MB;
            if (TB) bf[side][g] = read_across(buf * STAGE + BM * 128 + kc * 32 * BN + acrossB[g], 2 * BN);
            else bf[side][g] = *(const sm_i32x4 *)(lds + buf * STAGE + (BM + wn0 + 32 * g) * 128 + along[kc]);
        }
    };
    auto slice = [&](int side, int kc, int buf, int loads) __attribute__((always_inline)) {     // products of `side`, reads of slice kc of buf into the other
#pragma unroll
        for (int t = 0; t < P; t++) {
#pragma unroll
            for (int f = 0; f < MB + NB; f++)
                if (f * P / (MB + NB) == t) read(side ^ 1, kc, buf, f);
            acc[t / NB][t % NB] = Op::mul(bf[side][t % NB], af[side][t / NB], acc[t / NB][t % NB]);
#pragma unroll
            for (int i = 0; i < L; i++)
                if (i < loads && i * P / L == t) load(i);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // s_waitcnt vmcnt(n) lgkmcnt(0), expcnt untouched; then the same of all wavefronts
#define OWT_ARRIVED(n) do { asm volatile("" ::: "memory"); __builtin_amdgcn_s_waitcnt(((n) & 15) | (((n) >> 4) << 14) | (7 << 4)); \
                            __builtin_amdgcn_s_barrier(); asm volatile("" ::: "memory"); } while (0)
    if constexpr (S::RING != 0) {
        // Tile n of the order in which they are used lies in slot n % 5.  Two products: B, A0, A1 of a step of memory; three: A1, B0, A0, B1 for A1 B0, A0 B0 and A0 B1.
        // A product reads the fragments of the next slice between the instructions of one, its last slice the first ones of the next product; before that slice everybody has
        // read the product's tiles, and those that no later product reads are filled anew.
        constexpr bool THREE = S::RING == SM_THREE;
        constexpr int PER = THREE ? 4 : 3, PRODUCTS = THREE ? 3 : 2;
        const int t_beg = s_beg / PRODUCTS, t_end = t_beg + nst / PRODUCTS - 1;
        sm_i32x4 keep_a[THREE ? 4 : 1][MB], keep_b[4][NB], roll[2][MB > NB ? MB : NB];      // (rolling: those of A1, or of the tile that one product uses)
        int slot = 0;                               // of the step's first tile
        auto place = [&](int j) __attribute__((always_inline)) { const int at = slot + j; return (at >= 5 ? at - 5 : at) * STAGE; };
        const unsigned char *from_a, *from_b;       // where the tiles that are being loaded lie
        auto aim_a = [&](int t, int plane) __attribute__((always_inline)) {
            t = __builtin_amdgcn_readfirstlane(min(t, t_end));
            if (TA && 64 * t + 64 > p.a.rows) {
#pragma unroll
                for (int i = 0; i < AI; i++) asrc[i] = LoadA::from(p.a, wave, lane, i, m0, p.a.rows - 64 * t);
            }
            from_a = sm_uniform(ag + (size_t)t * p.a.step + 128 * plane);
        };
        auto aim_b = [&](int t, int plane) __attribute__((always_inline)) {
            t = __builtin_amdgcn_readfirstlane(min(t, t_end));
            if (TB && 64 * t + 64 > p.b.rows) {
#pragma unroll
                for (int i = 0; i < BI; i++) bsrc[i] = LoadB::from(p.b, wave, lane, i, n0, p.b.rows - 64 * t);
            }
            from_b = sm_uniform(bg + (size_t)t * p.b.step + 128 * plane);
        };
        auto load_a = [&](int i, int at) __attribute__((always_inline)) { sm_load_lds(asrc[i < AI ? i : 0], from_a, lds0 + at + NW * i * 1024); };
        auto load_b = [&](int i, int at) __attribute__((always_inline)) { sm_load_lds(bsrc[i < BI ? i : 0], from_b, lds0 + at + NW * i * 1024); };
        auto read_a = [&](sm_i32x4 &to, int at, int kc, int f) __attribute__((always_inline)) {
            if (TA) to = read_across(at + kc * 32 * BM + acrossA[f], 2 * BM);
            else to = *(const sm_i32x4 *)(lds + at + (wm0 + 32 * f) * 128 + along[kc]);
        };
        auto read_b = [&](sm_i32x4 &to, int at, int kc, int f) __attribute__((always_inline)) {
            if (TB) to = read_across(at + kc * 32 * BN + acrossB[f], 2 * BN);
            else to = *(const sm_i32x4 *)(lds + at + (wn0 + 32 * f) * 128 + along[kc]);
        };
        // products of a and b; reads f = 0 .. reads - 1, loads i = 0 .. loads - 1
        auto together = [&](const sm_i32x4 (&a)[MB], const sm_i32x4 (&b)[NB], int reads, auto reader, int loads, auto loader) __attribute__((always_inline)) {
#pragma unroll
            for (int t = 0; t < P; t++) {
#pragma unroll
                for (int f = 0; f < MB + NB; f++)
                    if (f < reads && f * P / reads == t) reader(f);
                acc[t / NB][t % NB] = Op::mul(b[t % NB], a[t / NB], acc[t / NB][t % NB]);
#pragma unroll
                for (int i = 0; i < 2 * AI; i++)
                    if (i < loads && i * P / loads == t) loader(i);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        auto nothing = [](int) __attribute__((always_inline)) {};
        if (some) {
#pragma unroll
            for (int n = 0; n < 5; n++) {
                const int t = t_beg + n / PER, j = n % PER;
                const bool of_b = THREE ? (j & 1) : j == 0;
                if (of_b) aim_b(t, THREE && j == 3);
                else aim_a(t, THREE ? j == 0 : j - 1);
#pragma unroll
                for (int i = 0; i < AI; i++) {
                    if (of_b) load_b(i, n * STAGE);
                    else load_a(i, n * STAGE);
                }
            }
            OWT_ARRIVED(3 * AI);
            if constexpr (THREE) {
#pragma unroll
                for (int f = 0; f < MB; f++) read_a(roll[0][f], place(0), 0, f);
#pragma unroll
                for (int f = 0; f < NB; f++) read_b(keep_b[0][f], place(1), 0, f);
                int t = t_beg;
                do {
                    // A1 B0
#pragma unroll
                    for (int kc = 0; kc < 3; kc++)
                        together(roll[kc & 1], keep_b[kc], MB + NB, [&](int f) __attribute__((always_inline)) {
                            if (f < MB) read_a(roll[(kc & 1) ^ 1][f < MB ? f : 0], place(0), kc + 1, f < MB ? f : 0);
                            else read_b(keep_b[kc + 1][f < MB ? 0 : f - MB], place(1), kc + 1, f < MB ? 0 : f - MB);
                        }, 0, nothing);
                    OWT_ARRIVED(2 * AI);            // A0 is there; A1 and B0 have been read: B0 and A0 of the next step come in their places
                    aim_b(t + 1, 0);
                    aim_a(t + 1, 0);
                    together(roll[1], keep_b[3], MB, [&](int f) __attribute__((always_inline)) { read_a(keep_a[0][f < MB ? f : 0], place(2), 0, f < MB ? f : 0); },
                             2 * AI, [&](int i) __attribute__((always_inline)) {
                                 if (i < BI) load_b(i, place(0));
                                 else load_a(i - BI, place(1));
                             });
                    // A0 B0
#pragma unroll
                    for (int kc = 0; kc < 3; kc++)
                        together(keep_a[kc], keep_b[kc], MB, [&](int f) __attribute__((always_inline)) { read_a(keep_a[kc + 1][f < MB ? f : 0], place(2), kc + 1, f < MB ? f : 0); }, 0, nothing);
                    OWT_ARRIVED(3 * AI);            // B1 is there; A0 has been read: B1 of the next step
                    aim_b(t + 1, 1);
                    together(keep_a[3], keep_b[3], NB, [&](int f) __attribute__((always_inline)) { read_b(roll[0][f < NB ? f : 0], place(3), 0, f < NB ? f : 0); },
                             BI, [&](int i) __attribute__((always_inline)) { load_b(i, place(2)); });
                    // A0 B1
#pragma unroll
                    for (int kc = 0; kc < 3; kc++)
                        together(keep_a[kc], roll[kc & 1], NB, [&](int f) __attribute__((always_inline)) { read_b(roll[(kc & 1) ^ 1][f < NB ? f : 0], place(3), kc + 1, f < NB ? f : 0); }, 0, nothing);
                    OWT_ARRIVED(2 * AI);            // the next step's A1 and B0 are there; B1 has been read: A1 of the step after that
                    aim_a(t + 2, 1);
                    together(keep_a[3], roll[1], MB + NB, [&](int f) __attribute__((always_inline)) {
                        if (f < MB) read_a(roll[0][f < MB ? f : 0], place(4), 0, f < MB ? f : 0);
                        else read_b(keep_b[0][f < MB ? 0 : f - MB], place(0), 0, f < MB ? 0 : f - MB);
                    }, AI, [&](int i) __attribute__((always_inline)) { load_a(i, place(3)); });
                    slot = slot + 4 >= 5 ? slot - 1 : slot + 4;
                } while (++t <= t_end);
            } else {
#pragma unroll
                for (int f = 0; f < MB; f++) read_a(roll[0][f], place(1), 0, f);
#pragma unroll
                for (int f = 0; f < NB; f++) read_b(keep_b[0][f], place(0), 0, f);
                int t = t_beg;
                do {
                    // A0 B
#pragma unroll
                    for (int kc = 0; kc < 3; kc++)
                        together(roll[kc & 1], keep_b[kc], MB + NB, [&](int f) __attribute__((always_inline)) {
                            if (f < MB) read_a(roll[(kc & 1) ^ 1][f < MB ? f : 0], place(1), kc + 1, f < MB ? f : 0);
                            else read_b(keep_b[kc + 1][f < MB ? 0 : f - MB], place(0), kc + 1, f < MB ? 0 : f - MB);
                        }, 0, nothing);
                    OWT_ARRIVED(2 * AI);            // A1 is there; A0 and B have been read: A1 of the next step and B of the one after that come in the places of B and A0
                    aim_a(t + 1, 1);
                    aim_b(t + 2, 0);
                    together(roll[1], keep_b[3], MB, [&](int f) __attribute__((always_inline)) { read_a(roll[0][f < MB ? f : 0], place(2), 0, f < MB ? f : 0); },
                             2 * AI, [&](int i) __attribute__((always_inline)) {
                                 if (i < AI) load_a(i, place(0));
                                 else load_b(i - AI, place(1));
                             });
                    // A1 B
#pragma unroll
                    for (int kc = 0; kc < 3; kc++)
                        together(roll[kc & 1], keep_b[kc], MB, [&](int f) __attribute__((always_inline)) { read_a(roll[(kc & 1) ^ 1][f < MB ? f : 0], place(2), kc + 1, f < MB ? f : 0); }, 0, nothing);
                    OWT_ARRIVED(2 * AI);            // the next step's B and A0 are there; A1 has been read: A0 of the step after that
                    aim_a(t + 2, 0);
                    together(roll[1], keep_b[3], MB + NB, [&](int f) __attribute__((always_inline)) {
                        if (f < MB) read_a(roll[0][f < MB ? f : 0], place(4), 0, f < MB ? f : 0);
                        else read_b(keep_b[0][f < MB ? 0 : f - MB], place(3), 0, f < MB ? 0 : f - MB);
                    }, AI, [&](int i) __attribute__((always_inline)) { load_a(i, place(2)); });
                    slot = slot + 3 >= 5 ? slot - 2 : slot + 3;
                } while (++t <= t_end);
            }
        }
    } else if (some) {
        OWT_ARRIVED(STARTED ? 0 : (NS - 1) * L);    // (with what the sums started from, everything)
#pragma unroll
        for (int f = 0; f < MB + NB; f++) read(0, 0, 0, f);
        int cur = 0;                                // stage s lives in buffer s % NS
        int s = 0;
        do {
            const int next = cur == NS - 1 ? 0 : cur + 1;
#pragma unroll
            for (int kc = 0; kc < 3; kc++) slice(kc & 1, kc + 1, cur, 0);
            // stage s + 1 has landed and everybody has this stage's last fragments: its buffer is filled anew (the last stages load the last one again,
            // and the very last reads fragments that nothing uses: a second copy of this code would take longer to arrive than that does)
            OWT_ARRIVED((NS - 2) * L);
            aim(s_beg + s + NS, cur);
            slice(1, 0, next, L);
            cur = next;
        } while (++s < nst);
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);             // vmcnt(0): the last loads into LDS have landed, too
#undef OWT_ARRIVED
    __syncthreads();                                // everybody has read the last stage

    // Accumulator register r of lane (li, lh): column 8 (r / 4) + 4 lh + r % 4 of C, row li of its block (the operands change places in the
    // instruction): four neighbouring results a lane.
    if constexpr (END == SM_TOP) {
        // Columns that do not exist have a bias of -infinity.  A lane has half of a row's values of its wavefront, the lane 32 away the other half.
        float *bias = (float *)lds;
        int *label = (int *)(bias + BN), *cexp = label + BM, *rexp = cexp + BN;
        if (SCALED) for (int c = tid; c < BN; c += 64 * NW) {
            bias[c] = n0 + c < p.N ? (p.bias ? p.bias[n0 + c] : 0.f) : -INFINITY;
            cexp[c] = n0 + c < p.N ? -p.col_exp[n0 + c] : -kSmNone;      // (what is there is a copy of the last column)
        }
        for (int r = tid; r < BM; r += 64 * NW) {
            label[r] = m0 + r < p.M && p.labels && has_class(p.labels[m0 + r], p.classes) ? p.labels[m0 + r] - p.off - n0 : -1;
            if (SCALED) rexp[r] = m0 + r < p.M ? -p.row_exp[m0 + r] : 0;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < MB; i++) {
            const int re = SCALED ? rexp[wm0 + 32 * i + li] : 0;
            // f(column, output) of this lane's outputs, four columns at a time
            auto outputs = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
                for (int j = 0; j < NB; j++)
#pragma unroll
                    for (int g = 0; g < 4; g++) {
                        const int c = 32 * j + 8 * g;
                        if (SCALED) {
                            const float4 b4 = *(const float4 *)(bias + wn0 + c + 4 * lh);
                            const int4 e4 = *(const int4 *)(cexp + wn0 + c + 4 * lh);
                            const float b[4] = {b4.x, b4.y, b4.z, b4.w};
                            const int e[4] = {e4.x, e4.y, e4.z, e4.w};
#pragma unroll
                            for (int t = 0; t < 4; t++) f(c + t, ldexpf(acc[i][j][4 * g + t], re + e[t]) + b[t]);
                        } else
#pragma unroll
                            for (int t = 0; t < 4; t++) f(c + t, acc[i][j][4 * g + t]);
                    }
            };
            // (both walks read the accumulators where they are: the compiler would keep copies of 256 of them in between)
            auto stay = [&] __attribute__((always_inline)) () {
#pragma unroll
                for (int j = 0; j < NB; j++) asm volatile("" : "+a"(acc[i][j]));
            };
            float most = -INFINITY, sum[4] = {0.f, 0.f, 0.f, 0.f};
            stay();
            outputs([&](int, float z) __attribute__((always_inline)) { most = fmaxf(most, z); });
            most = fmaxf(most, __shfl_xor(most, 32, 64));
            const float at = __builtin_isfinite(most) ? most : 0.f;
            stay();
            outputs([&](int c, float z) __attribute__((always_inline)) { sum[c & 3] += exp_of(z - at); });
            float all = (sum[0] + sum[1]) + (sum[2] + sum[3]);
            all += __shfl_xor(all, 32, 64);
            const int m = m0 + wm0 + 32 * i + li;
            if (lh == 0 && m < p.M) p.top[(size_t)(tn * WN + wn) * p.M + m] = {most, all};
            // the label's output, where it is among these (of many classes hardly ever)
            const int mine = label[wm0 + 32 * i + li] - wn0;
            if (__any(mine >= 0 && mine < 32 * NB)) {
                float v = 0.f;
                stay();
                outputs([&](int c, float z) __attribute__((always_inline)) { v = mine - 4 * lh == c ? z : v; });
                if (mine >= 0 && mine < 32 * NB && ((mine >> 2) & 1) == lh) p.target[m] = v;
            }
        }
        return;
    }

    // Results go through LDS, 32 rows of a wavefront at a time, so that rows are written as runs of 32 NB values; 16-byte piece q of row r sits in
    // slot q ^ (r % 16) (or % 8).  What a row has to itself comes from LDS, too: read from memory it would wait for the stores before it.
    constexpr int QW = 8 * NB, SW = QW < 16 ? QW - 1 : 15, RI = 64 / QW;        // pieces of a wavefront's row, the bits of a row's swizzle, rows of an access
    static_assert(NS * STAGE >= NW * 32 * QW * 16 + BM * 16 + 32, "32 rows of each wavefront and what rows have to themselves fit the stages");
    unsigned char *mine = lds + wave * (32 * QW * 16);
    const int q = lane % QW, c = n0 + wn0 + 4 * q;
    auto in_order = [] __attribute__((always_inline)) () {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    };
    auto put_rows = [&](int i) __attribute__((always_inline)) {
        if (i > 0) in_order();
#pragma unroll
        for (int j = 0; j < NB; j++)
#pragma unroll
            for (int g = 0; g < 4; g++) {
                const float4 v = make_float4(acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]);
                *(float4 *)(mine + (li * QW + ((8 * j + 2 * g + lh) ^ (li & SW))) * 16) = v;
            }
        in_order();
    };
    auto get_row = [&](int r) __attribute__((always_inline)) {      // this lane's piece of row r + lane / QW, r a multiple of RI
        return *(const float4 *)(mine + ((r + lane / QW) * QW + (q ^ ((r + lane / QW) & SW))) * 16);
    };

    if constexpr (END == SM_DZ) {
        float *lses = (float *)(lds + NW * (32 * QW * 16)), *weights = lses + BM;
        int *label = (int *)(weights + BM), *rexp = label + BM;
        for (int r = tid; r < BM; r += 64 * NW) {
            const SmDzRow w = sm_dz_row<SCALED>(p, m0 + r);
            lses[r] = w.lse;
            weights[r] = w.weight;
            label[r] = w.label;
            if (SCALED) rexp[r] = w.exp;
        }
        const int2 least = SCALED ? sm_leasts(p, rexp + BM, tile == 0) : make_int2(0, 0);
        __syncthreads();
        const SmDzColumns k = sm_dz_columns<SCALED>(p, c);
        float sums[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < MB; i++) {
            put_rows(i);
#pragma unroll 4
            for (int r = 0; r < 32; r += RI) {
                const int row = 32 * i + r + lane / QW;
                const SmDzRow w = {lses[wm0 + row], weights[wm0 + row], label[wm0 + row], SCALED ? rexp[wm0 + row] : 0};
                sm_dz<SCALED, STARTED>(p, least, m0 + wm0 + row, c, get_row(r), w, k, sums);
            }
        }
        if (p.dbias) {
#pragma unroll
            for (int t = 0; t < 4; t++)
#pragma unroll
                for (int d = QW; d < 64; d *= 2) sums[t] += __shfl_xor(sums[t], d, 64);
            float *db = p.dbias + (size_t)(tm * S::WM + wm) * p.N;
            if (lane < QW)
#pragma unroll
                for (int t = 0; t < 4; t++)
                    if (c + t < p.N) db[c + t] = sums[t];
        }
    }

    if constexpr (END == SM_OUT) {
        const bool parts = p.splits > 1;
        const unsigned width = (unsigned)p.N * (!parts && p.bf16 ? 2 : 4);
        float *factor = (float *)(lds + NW * (32 * QW * 16));
        for (int r = tid; r < BM; r += 64 * NW) factor[r] = sm_row_factor<SCALED>(p, m0 + r);
        const int shift = SCALED && !parts ? -(*p.under + kSmDzTop) : 0;
        __syncthreads();
        char *base = (parts ? (char *)(p.partial + (size_t)split * p.M * p.N) : (char *)p.out) + (size_t)(m0 + wm0) * width;
        const int m_end = __builtin_amdgcn_readfirstlane(max(0, min(32 * MB, p.M - m0 - wm0)));     // rows of this wavefront that exist
        const float *add = p.add ? p.add + (size_t)(m0 + wm0) * p.N : nullptr;
        auto ends = [&](auto how, auto vec) __attribute__((always_inline)) {
            constexpr int HOW = decltype(how)::value;       // 0: parts, 1: fp32, 2: fp32 with beta, 3: bf16; 4, 5: something is added; 6: fp32, past the caches
            constexpr bool VEC = decltype(vec)::value, HALF = HOW == 3 || HOW == 5, ADD = HOW == 4 || HOW == 5;
            constexpr int PAST = HOW == 6 ? 2 : 0;
            // whole fours: through a descriptor that ends with the last row, where what lies outside is not written
            const __amdgpu_buffer_rsrc_t rs = owt_make_rsrc(sm_uniform((const unsigned char *)base), (unsigned)m_end * width);
            const __amdgpu_buffer_rsrc_t as = owt_make_rsrc(sm_uniform((const unsigned char *)add), ADD ? (unsigned)m_end * (unsigned)p.N * 4u : 0u);
#pragma unroll
            for (int i = 0; i < MB; i++) {
                put_rows(i);
#pragma unroll 4
                for (int r = 0; r < 32; r += RI) {
                    const float4 u = get_row(r);
                    const int row = 32 * i + r + lane / QW;
                    float v[4] = {u.x, u.y, u.z, u.w};
                    if (HOW != 0) sm_result<SCALED>(v, shift, factor[wm0 + row], p.alpha);
                    // (rows that begin anywhere are written by fours, too, but for the last of them; memory takes them on any 4 bytes, and bf16 ones on any 2)
                    const bool whole = VEC ? c < p.N : c + 4 <= p.N;
                    const unsigned at = whole ? (unsigned)row * width + (unsigned)c * (HALF ? 2 : 4) : 0x80000000u;
                    if (HOW == 2) {
                        const float4 old = buffer_load4(rs, at);
                        v[0] += p.beta * old.x; v[1] += p.beta * old.y; v[2] += p.beta * old.z; v[3] += p.beta * old.w;
                    }
                    if (ADD) {
                        const float4 old = buffer_load4(as, whole ? (unsigned)row * (unsigned)p.N * 4u + (unsigned)c * 4u : 0x80000000u);
                        v[0] += old.x; v[1] += old.y; v[2] += old.z; v[3] += old.w;
                    }
                    const owt_u32x2 h = {f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3])};
                    if (!HALF) {
                        const owt_u32x4 o = {__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
                        __builtin_amdgcn_raw_buffer_store_b128(o, rs, (int)at, 0, PAST);
                    } else if (VEC) __builtin_amdgcn_raw_buffer_store_b64(h, rs, (int)at, 0, 0);
                    else if (whole && row < m_end) *(SmFourHalves *)(base + (size_t)row * width + 2 * c) = {h[0], h[1]};
                    if (!VEC && !whole && row < m_end) {
                        char *w = base + (size_t)row * width;
#pragma unroll
                        for (int t = 0; t < 3; t++)
                            if (c + t < p.N) {
                                if (HOW == 2) v[t] += p.beta * ((float *)w)[c + t];
                                if (ADD) v[t] += add[(size_t)row * p.N + c + t];
                                if (HALF) store1((bf16_t *)w, c + t, v[t]);
                                else store1((float *)w, c + t, v[t]);
                            }
                    }
                }
            }
        };
        auto with = [&](auto vec) __attribute__((always_inline)) {
            using std::integral_constant;
            if (parts) ends(integral_constant<int, 0>{}, vec);
            else if (p.add) {
                if (p.bf16) ends(integral_constant<int, 5>{}, vec);
                else ends(integral_constant<int, 4>{}, vec);
            } else if (p.bf16) ends(integral_constant<int, 3>{}, vec);
            else if (p.beta != 0.f) ends(integral_constant<int, 2>{}, vec);
            else if (p.big) ends(integral_constant<int, 6>{}, vec);
            else ends(integral_constant<int, 1>{}, vec);
        };
        if ((p.N & 3) == 0) with(std::true_type{});
        else with(std::false_type{});
        if (TA && p.db && n0 == 0 && split == 0)         // dw: rows are classes, and their bias has a gradient, too
            for (int m = m0 + tid; m < min(m0 + BM, p.M); m += 64 * NW) {
                float sum = 0.f;
#pragma unroll 8
                for (int k = 0; k < p.strips; k++) sum += p.dbias[(size_t)k * p.M + m];
                p.db[m] = p.alpha * sum + (p.beta != 0.f ? p.beta * p.db[m] : 0.f);
            }
    }
}

// 16 bytes from where rows begin anywhere
struct __attribute__((packed, aligned(2))) SmLoose { uint32_t u[4]; };

// bf16 rows, eight values a thread: work-group `at` of `of`
__device__ __forceinline__ void sm_copy_rows(const SmPrep &p, int at, int of)
{
    const int pieces = p.steps * 8, blocks = (pieces + 255) / 256;      // work-groups of a row
    for (int b = at; b < p.out_rows * blocks; b += of) {
        const int m = b / blocks, i = (b - m * blocks) * 256 + threadIdx.x, c = 8 * i;
        if (i >= pieces) continue;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (m < p.rows && c < p.cols && (!p.labels || has_class(p.labels[m], p.classes))) {
            const uint16_t *row = (const uint16_t *)p.from + (size_t)m * p.cols;
            if (c + 8 <= p.cols) {
                const SmLoose l = *(const SmLoose *)(row + c);
                v = make_uint4(l.u[0], l.u[1], l.u[2], l.u[3]);
            } else {
                uint32_t u[4];
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    const int e = c + 2 * k;
                    u[k] = (e < p.cols ? row[e] : 0u) | ((e + 1 < p.cols ? (uint32_t)row[e + 1] : 0u) << 16);
                }
                v = make_uint4(u[0], u[1], u[2], u[3]);
            }
        }
        *(uint4 *)(p.to + (size_t)m * pieces * 16 + 16 * i) = v;
    }
}
constexpr int kSmCopyGroups = 512;      // behind the tiles

template <class Op, bool TA, bool TB, class S, int END>
__global__ void __launch_bounds__(64 * S::NW, (S::OCC * S::NW + 3) / 4) sm_kernel(const SmParams p)
{
    __shared__ __attribute__((aligned(16))) unsigned char lds[S::LDS];
    if (!TA && !TB && END != SM_TOP && p.copy.out_rows) {
        const int tiles = owt_split_major_grid(p.tiles, p.splits);
        if ((int)blockIdx.x >= tiles) {
            sm_copy_rows(p.copy, blockIdx.x - tiles, gridDim.x - tiles);
            return;
        }
    }
    int tile, split;
    if (!owt_split_major_wg(p.tiles, p.splits, tile, split)) return;
    sm_tile<Op, TA, TB, S, END>(p, tile, split, lds);
}

// dx and dw in one launch, the one of longer sums first (dw is not split)
template <class Op, class S>
__global__ void __launch_bounds__(64 * S::NW, (S::OCC * S::NW + 3) / 4) sm_pair_kernel(const SmParams x, const SmParams w, bool x_first)
{
    __shared__ __attribute__((aligned(16))) unsigned char lds[S::LDS];
    const int gx = owt_split_major_grid(x.tiles, x.splits), gw = owt_split_major_grid(w.tiles, 1), b = (int)blockIdx.x;
    const bool of_x = x_first ? b < gx : b >= gw;
    // (the numbering of owt_split_major_wg, within a product's work-groups: their number is a multiple of 8)
    const int l = of_x ? (x_first ? b : b - gw) : (x_first ? b - gx : b), total = of_x ? x.tiles * x.splits : w.tiles;
    const int xcd = l & 7, jx = l >> 3, each = total >> 3, more = total & 7;
    if (jx >= each + (xcd < more ? 1 : 0)) return;
    const int one = xcd * each + min(xcd, more) + jx;
    if (of_x) sm_tile<Op, false, true, S, SM_OUT>(x, one % x.tiles, one / x.tiles, lds);
    else sm_tile<Op, true, true, S, SM_OUT>(w, one, 0, lds);
}

}  // namespace owt

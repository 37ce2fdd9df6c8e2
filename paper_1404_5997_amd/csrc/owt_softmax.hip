// Softmax cross-entropy on a dense shard's outputs, without the outputs: entry points, and the passes around the products of smgemm.hpp.
//
//   z[n][o] = bias[o] + sum_i x[n][i] w[o][i],   lse[n] = log sum_o exp z[n][o]
//   dz[n][o] = weight[n] (exp(z[n][o] - lse[n]) - [o is n's label]),   dx = dz w,   dw = alpha dz^T x + beta dw,   dbias likewise
//
// Forward, a product's work-groups leave each row's largest output and sum of exponentials over their columns, and one launch joins those.  Backward,
// the classes are taken in pieces: the outputs of a piece are computed again and leave as dz, its part of dx is added up and its rows of dw
// are done.  Where a product has few tiles its sums are split over work-groups, and the launch that joins them does the same to the outputs.
//
// bf16 weights whose rows are whole steps of 64 values are read as they lie; others, and fp32 operands, are laid out for the products first, fp32
// values as two f16 ones.
#include <cmath>

#include "smfew.hpp"
#include "softmax.hpp"

namespace owt {

// ------------------------------------------------------------------------------------------------ layout of operands

// Rows of x (a) and of w (b), either of which may be none, in one launch.
__global__ void __launch_bounds__(256) sm_rows_kernel(const SmPrep a, const SmPrep b, int groups_a)
{
    if ((int)blockIdx.x < groups_a) sm_copy_rows(a, blockIdx.x, groups_a);
    else sm_copy_rows(b, blockIdx.x - groups_a, gridDim.x - groups_a);
}

// fp32 rows as two f16 values under the power of two that brings a row's largest magnitude to [2^14, 2^15), ROWS rows a work-group.  What a
// thread does not keep of a row (1024 values of it, or 4096) is read twice, the second time from the caches.  Four rows a work-group for many rows, one for few.
template <int ROWS> __global__ void __launch_bounds__(256) sm_halves_kernel(const SmPrep a, const SmPrep b, int groups_a)
{
    constexpr int EACH = 256 / ROWS;        // threads of a row
    __shared__ float part[4];
    __shared__ int low[4];
    const bool of_a = (int)blockIdx.x < groups_a;
    const SmPrep &p = of_a ? a : b;
    const int group = of_a ? blockIdx.x : blockIdx.x - groups_a;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, at = threadIdx.x % EACH;
    const int m = group * ROWS + threadIdx.x / EACH;
    const bool real = m < p.rows && (!p.labels || has_class(p.labels[m], p.classes));
    const float *row = (const float *)p.from + (size_t)m * p.cols;
    auto four = [&](int c) __attribute__((always_inline)) {
        if (!real || c >= p.cols) return make_float4(0.f, 0.f, 0.f, 0.f);
        if (c + 4 <= p.cols) {
            const SmLoose l = *(const SmLoose *)(row + c);
            return make_float4(__uint_as_float(l.u[0]), __uint_as_float(l.u[1]), __uint_as_float(l.u[2]), __uint_as_float(l.u[3]));
        }
        return make_float4(row[c], c + 1 < p.cols ? row[c + 1] : 0.f, c + 2 < p.cols ? row[c + 2] : 0.f, 0.f);
    };
    constexpr int HELD = 4;                 // pieces of four that a thread keeps
    float4 held[HELD];
    float most = 0.f;
    auto size = [&](const float4 &v) __attribute__((always_inline)) {
        most = fmaxf(fmaxf(fmaxf(most, fabsf(v.x)), fmaxf(fabsf(v.y), fabsf(v.z))), fabsf(v.w));
    };
#pragma unroll
    for (int k = 0; k < HELD; k++) held[k] = four(4 * at + 4 * EACH * k);
#pragma unroll
    for (int k = 0; k < HELD; k++) size(held[k]);
    if (real)
#pragma unroll 4
        for (int c = 4 * at + 4 * EACH * HELD; c < p.cols; c += 4 * EACH) size(four(c));
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) most = fmaxf(most, __shfl_xor(most, d, 64));
    if (ROWS == 1) {
        if (lane == 0) part[wave] = most;
        __syncthreads();
        most = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
    }
    // (a row of infinities stays as it is: they are infinite in f16, too; NaN alone has no largest magnitude, and stays NaN)
    const int exp = !(most > 0.f) ? kSmNone : __builtin_isfinite(most) ? kSmTop - ilogbf(most) : 0, shift = exp == kSmNone ? 0 : exp;
    if (m < p.out_rows) {
        unsigned char *to = p.to + (size_t)m * p.steps * 256;
        auto write = [&](int c, const float4 &v) __attribute__((always_inline)) {
            const float s[4] = {ldexpf(v.x, shift), ldexpf(v.y, shift), ldexpf(v.z, shift), ldexpf(v.w, shift)};
            sm_put_halves(to + (size_t)(c >> 6) * 256 + 2 * (c & 63), s);
        };
#pragma unroll
        for (int k = 0; k < HELD; k++)
            if (4 * at + 4 * EACH * k < p.steps * 64) write(4 * at + 4 * EACH * k, held[k]);
#pragma unroll 4
        for (int c = 4 * at + 4 * EACH * HELD; c < p.steps * 64; c += 4 * EACH) write(c, four(c));
        if (at == 0 && m < p.rows) p.exps[m] = exp;
    }
    if (!p.lows) return;                    // (of all threads, or of none)
    // a weight is below 2^k (a row whose weight is zero or not finite says nothing)
    const float g = p.weight && m < p.rows ? fabsf(p.weight[m]) : 1.f;
    const int mine = m < p.rows && exp != kSmNone && g > 0.f && __builtin_isfinite(g) ? exp - (p.weight ? ilogbf(g) + 1 : 0) : kSmNone;
    if (ROWS > 1) {
        if (lane == 0) low[wave] = mine;
        __syncthreads();
    }
    if (threadIdx.x == 0) p.lows[group] = ROWS == 1 ? mine : min(min(low[0], low[1]), min(low[2], low[3]));
}

// ------------------------------------------------------------------------------------------------ after the products

__device__ __forceinline__ float lse_of(Top t) { return (__builtin_isfinite(t.max) ? t.max : 0.f) + logf(t.sum); }
// lse - target without lse's own rounding, which is what is left of a small loss: a label whose output is the largest, 10, and a loss of 0.05 lose five digits in 10.05 - 10
__device__ __forceinline__ float loss_of(Top t, float target)
{
    if (target == -INFINITY) return INFINITY;
    return __builtin_isfinite(t.max) ? (t.max - target) + logf(t.sum) : lse_of(t) - target;
}

struct SmRows {                 // what is known of rows of outputs, and where it goes
    const Top *top;             // [parts][N]
    int parts, N;
    const float *label_out;     // outputs of the labels that these columns hold
    const int *labels;
    int classes, off, cols;     // this worker's columns
    float *lse, *target, *loss;
};
__device__ __forceinline__ void finish_row(const SmRows &p, int n, Top t, const float *label_out)
{
    float lse = lse_of(t), target = -INFINITY, loss = 0.f;
    if (p.labels) {
        const int label = p.labels[n];
        if (!has_class(label, p.classes)) lse = target = 0.f;
        else {
            if (label >= p.off && label - p.off < p.cols) target = *label_out;
            loss = loss_of(t, target);
        }
        if (p.target) p.target[n] = target;
        if (p.loss) p.loss[n] = loss;
    }
    p.lse[n] = lse;
}
// Joins the parts of 256 / EACH rows in a work-group, EACH threads a row
template <int EACH> __global__ void __launch_bounds__(256) sm_finish_kernel(const SmRows p)
{
    constexpr int ROWS = 256 / EACH;
    __shared__ Top part[EACH][ROWS];
    const int r = threadIdx.x % ROWS, e = threadIdx.x / ROWS, n = blockIdx.x * ROWS + r;
    Top t = {-INFINITY, 0.f};
    if (n < p.N)
        for (int k = e; k < p.parts; k += EACH) t = join(t, p.top[(size_t)k * p.N + n]);
    part[e][r] = t;
    __syncthreads();
    for (int half = EACH / 2; half >= 1; half /= 2) {
        if (e < half) part[e][r] = join(part[e][r], part[e + half][r]);
        __syncthreads();
    }
    if (e == 0 && n < p.N) finish_row(p, n, part[0][r], p.label_out + n);
}

// Outputs whose sums were split: a work-group a row joins them and is done with it.
template <bool SCALED> __global__ void __launch_bounds__(256) sm_split_top_kernel(const SmParams p, const SmRows r)
{
    __shared__ Top part[4];
    __shared__ float label_out;
    const int m = blockIdx.x, at = p.labels ? p.labels[m] - p.off : -1;
    const size_t whole = (size_t)p.M * p.N;
    const float *row = p.partial + (size_t)m * p.N;
    const int re = SCALED ? p.row_exp[m] : 0;
    Top t = {-INFINITY, 0.f};
    const bool vec = (p.N & 3) == 0;
    for (int c = 4 * threadIdx.x; c < p.N; c += 1024) {
        float z[4] = {0.f, 0.f, 0.f, 0.f};
        if (vec) {
#pragma unroll 8
            for (int k = 0; k < p.splits; k++) {
                const float4 v = *(const float4 *)(row + k * whole + c);
                z[0] += v.x; z[1] += v.y; z[2] += v.z; z[3] += v.w;
            }
        } else
#pragma unroll 4
            for (int k = 0; k < p.splits; k++)
#pragma unroll
                for (int i = 0; i < 4; i++) z[i] += c + i < p.N ? row[k * whole + c + i] : 0.f;
#pragma unroll
        for (int i = 0; i < 4; i++)
            if (c + i < p.N) {
                if (SCALED) z[i] = ldexpf(z[i], -(re + p.col_exp[c + i]));
                if (p.bias) z[i] += p.bias[c + i];
                if (c + i == at) label_out = z[i];
                t = join(t, top_of(z[i]));
            }
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) t = join(t, {__shfl_xor(t.max, d, 64), __shfl_xor(t.sum, d, 64)});
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = t;
    __syncthreads();
    if (threadIdx.x == 0) finish_row(r, m, join(join(part[0], part[1]), join(part[2], part[3])), &label_out);
}

// dz of outputs whose sums were split: 32 rows by 64 columns a work-group, 16 threads a row
template <bool SCALED> __global__ void __launch_bounds__(256) sm_split_dz_kernel(const SmParams p)
{
    __shared__ float4 part[16][16];
    __shared__ int two[8];
    const int2 least = SCALED ? sm_leasts(p, two, blockIdx.x == 0 && blockIdx.y == 0) : make_int2(0, 0);
    const int q = threadIdx.x & 15, r = threadIdx.x >> 4, c = blockIdx.x * 64 + 4 * q;
    const size_t whole = (size_t)p.M * p.N;
    const SmDzColumns k = sm_dz_columns<SCALED>(p, c);
    float sums[4] = {0.f, 0.f, 0.f, 0.f};
    for (int m = blockIdx.y * 32 + r; m < (int)blockIdx.y * 32 + 32; m += 16) {      // (rows past the last are zeros; nothing is read or written of them)
        float z[4] = {0.f, 0.f, 0.f, 0.f};
        const float *row = p.partial + (size_t)m * p.N + c;
        if ((p.N & 3) == 0) {
            if (c < p.N && m < p.M)
#pragma unroll 8
                for (int s = 0; s < p.splits; s++) {
                    const float4 v = *(const float4 *)(row + s * whole);
                    z[0] += v.x; z[1] += v.y; z[2] += v.z; z[3] += v.w;
                }
        } else
            for (int s = 0; s < p.splits; s++)
#pragma unroll
                for (int t = 0; t < 4; t++)
                    if (c + t < p.N && m < p.M) z[t] += row[s * whole + t];
        sm_dz<SCALED, false>(p, least, m, c, make_float4(z[0], z[1], z[2], z[3]), sm_dz_row<SCALED>(p, m), k, sums);
    }
    if (!p.dbias) return;
    part[r][q] = make_float4(sums[0], sums[1], sums[2], sums[3]);
    __syncthreads();
    if (threadIdx.x < 64 && blockIdx.x * 64 + threadIdx.x < p.N) {
        float s = 0.f;
        for (int k2 = 0; k2 < 16; k2++) s += ((const float *)&part[k2][threadIdx.x >> 2])[threadIdx.x & 3];
        p.dbias[(size_t)blockIdx.y * p.N + blockIdx.x * 64 + threadIdx.x] = s;
    }
}

// Adds up the parts of a split sum, in order: four columns a thread.  No parts: a sum of nothing.
template <bool SCALED> __global__ void __launch_bounds__(256) sm_join_kernel(const SmParams p)
{
    const unsigned quads = (unsigned)(p.N + 3) / 4;
    const size_t n = (size_t)p.M * quads, stride = (size_t)gridDim.x * 256, whole = (size_t)p.M * p.N;
    const int shift = SCALED && p.splits ? -(*p.under + kSmDzTop) : 0;
    const bool vec = (p.N & 3) == 0;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += stride) {
        const int m = (int)(i / quads), c = (int)(i % quads) * 4;
        const size_t at = (size_t)m * p.N + c;
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        auto four = [&](const float *from, float (&u)[4]) __attribute__((always_inline)) {
            if (vec) {
                const float4 w = *(const float4 *)from;
                u[0] = w.x; u[1] = w.y; u[2] = w.z; u[3] = w.w;
            } else
#pragma unroll
                for (int t = 0; t < 4; t++) u[t] = c + t < p.N ? from[t] : 0.f;
        };
#pragma unroll 4
        for (int k = 0; k < p.splits; k++) {
            float u[4];
            four(p.partial + k * whole + at, u);
#pragma unroll
            for (int t = 0; t < 4; t++) v[t] += u[t];
        }
        sm_result<SCALED>(v, shift, sm_row_factor<SCALED>(p, m), p.alpha);
        float u[4];
        if (p.add) {
            four(p.add + at, u);
#pragma unroll
            for (int t = 0; t < 4; t++) v[t] += u[t];
        }
        if (!p.bf16 && p.beta != 0.f) {
            four((const float *)p.out + at, u);
#pragma unroll
            for (int t = 0; t < 4; t++) v[t] += p.beta * u[t];
        }
        if (vec && !p.bf16) *(float4 *)((float *)p.out + at) = make_float4(v[0], v[1], v[2], v[3]);
        else if (vec) *(uint2 *)((uint16_t *)p.out + at) = make_uint2(f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3]));
        else
#pragma unroll
            for (int t = 0; t < 4; t++)
                if (c + t < p.N) {
                    if (p.bf16) store1((bf16_t *)p.out, at + t, v[t]);
                    else store1((float *)p.out, at + t, v[t]);
                }
    }
}

// Joins the shards' shares: lse and target of `workers` shards, worker by worker.
__global__ void __launch_bounds__(256) softmax_join_kernel(int workers, int N, int classes, const float *lses, const float *targets, const int *labels,
                                                           float *lse, float *target, float *loss)
{
    const unsigned n = blockIdx.x * 256 + threadIdx.x;      // (2^31 threads at most)
    if (n >= (unsigned)N) return;
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
    const float l = lse_of(t);
    lse[n] = l;
    if (target) target[n] = at;
    if (loss) loss[n] = loss_of(t, at);
}

// ------------------------------------------------------------------------------------------------ host

constexpr int kMaxRows = 1 << 22;       // of x and of w, and values of a row: 256 rows of 2^24 bytes are addressed with 32 bits

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
    if (d->N > kMaxRows || o_local > kMaxRows || d->I > kMaxRows) return fail(OWT_EUNSUPPORTED, "more than 2^22 rows, columns or inputs");
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

// What a work-group takes: `start` for its beginning and end (`dz` more where outputs leave as dz), `step` for a step on a quiet chip, `busy` where most CUs have one.
// us, fitted to outputs, dz, dx and dw of 16 x 2048 -> 65536, 128 x 4096 -> 32768, 777 x 1536 -> 20000, 2048 x 2048 -> 16384 (bf16) and 1003 x 1024 -> 16384 (fp32)
// with every tile.  Two work-groups a CU take turns, so that what counts is how many there are, not how many rounds.
struct SmTileCost { int bm, bn, wm, wn; float start, dz, step, busy; int together; };
static const SmTileCost kSmTiles[SM_TILES] = {{256, 256, 2, 2, 11.f, 8.f, 1.05f, 1.5f, 1}, {128, 128, 2, 2, 3.f, 2.f, 0.4f, 0.55f, 1},
                                              {128, 128, 2, 2, 2.f, 1.5f, 0.6f, 0.5f, 2}, {64, 64, 2, 2, 1.2f, 0.5f, 0.21f, 0.21f, 1}};
constexpr int SM_NOTHING = -1;          // more work-groups than a launch holds
struct SmPlan { int tile, splits; float us; };
static int up(int n, int to) { return (n + to - 1) / to; }

// A product of M x N results and `steps` steps, `products` of which stay together; end: how they leave
static SmPlan sm_plan(long M, long N, int steps, int products, int end)
{
    SmPlan best{SM_NOTHING, 1, 1e30f};
    const int want = forced_tile() - kSmFirstTile, want_split = forced_split(), most = steps / products;
    for (int t = 0; t < SM_TILES; t++) {
        if (want >= 0 && want < SM_TILES && t != want) continue;
        const SmTileCost &q = kSmTiles[t];
        const long tiles = ((M + q.bm - 1) / q.bm) * ((N + q.bn - 1) / q.bn);
        if (!groups_fit(tiles, 256)) continue;
        for (int sp = 1; sp <= 32 && (sp == 1 || (sp * 2 <= most && tiles * sp <= 1024)); sp *= 2) {
            const long n = tiles * sp;
            const float step = n >= (t == SM_BIG ? 192 : 128) ? q.busy : q.step, one = q.start + (end == SM_DZ && sp == 1 ? q.dz : 0.f) + (float)(up(most, sp) * products) * step;
            const float out = end != SM_OUT && sp == 1 ? 0.f : (float)(q.bm * q.bn) * 4.f / 17.6e3f;      // written at a CU's share of the memory's rate
            const float work = one > out ? one : out;
            const float each = q.together > 1 && n > 256 ? (float)n / 256.f + 0.5f : (float)((n + 255) / 256);      // work-groups of a CU
            float us = 3.f + each * (q.together > 1 && n <= 256 ? q.start + (work - q.start) * 1.2f : work);
            if (sp > 1) us += 3.6f + (float)(sp + 1) * (float)M * (float)N * 4.f / 3e6f;        // the launch that adds up
            if (us < best.us) best = {t, sp, us};
        }
    }
    if (want_split > 0) best.splits = want_split < most ? want_split : most;
    return best;
}
static size_t partial_bytes(const SmPlan &pl, long M, long N) { return pl.splits > 1 ? (size_t)pl.splits * M * N * 4 : 0; }
static int strips_of(const SmPlan &z, int N) { return z.splits > 1 ? up(N, 32) : up(N, kSmTiles[z.tile].bm) * kSmTiles[z.tile].wm; }

// Both backward products in one launch, dx's sums perhaps split: worth its tile where neither fills the chip for long.  Returns the tile or SM_NOTHING, the plan of dx in x.
static int sm_pair(long N, long cols, long I, int products_x, int products_w, const SmPlan &dx, const SmPlan &dw, SmPlan &x)
{
    const int want = forced_tile() - kSmFirstTile;
    const int most = up((int)cols, 64), steps_w = up((int)N, 64) * products_w;
    if (forced_split() > 0) return SM_NOTHING;
    float least = want >= 0 && want < SM_TILES ? 1e30f : dx.us + dw.us;
    int best = SM_NOTHING;
    for (int t : {(int)SM_MID, (int)SM_SMALL}) {
        if (want >= 0 && want < SM_TILES && t != want) continue;
        const SmTileCost &q = kSmTiles[t];
        const long nx = ((N + q.bm - 1) / q.bm) * ((I + q.bn - 1) / q.bn), nw = ((cols + q.bm - 1) / q.bm) * ((I + q.bn - 1) / q.bn);
        if (!groups_fit(nx * 32 + nw + 16, 256)) continue;
        for (int sp = 1; sp <= 32 && (sp == 1 || (sp * 2 <= most && nx * sp <= 1024)); sp *= 2) {
            const float ux = q.start + (float)(up(most, sp) * products_x) * q.busy, uw = q.start + (float)steps_w * q.busy, longest = ux > uw ? ux : uw;
            const float sum = ((float)(nx * sp) * ux + (float)nw * uw) / 256.f + 0.3f * longest;
            float us = 3.f + (sum > longest ? sum : longest);
            if (sp > 1) us += 3.6f + (float)(sp + 1) * (float)N * (float)I * 4.f / 3e6f;
            if (us < least) {
                least = us;
                best = t;
                x = {t, sp, us};
            }
        }
    }
    return best;
}
static int low_groups(size_t rows) { return rows >= 4096 ? (int)((rows + 3) / 4) : (int)rows; }
// of `rows` rows or fewer: 4095, one by one, are more work-groups than 4096 by fours
static int most_low_groups(size_t rows) { return rows >= 4096 && low_groups(rows) < 4095 ? 4095 : low_groups(rows); }

// Few fp32 rows go by the weights as they lie (smfew.hpp): as planes these are read, written and read again.  us here and as planes, outputs and their statistics,
// then gradients: 1 x 2048 -> 65536 111 / 346 and 368 / 777, 48 x 1024 -> 65536 101 / 172 and 307 / 402, 12 x 2048 -> 1000 16 / 18 and 25 / 36, 64 x 1024 -> 65536 112 / 176
// and 345 / 405.  A work-group walks all of k, so that long rows of few classes leave most of the chip idle (48 x 8192 -> 2048: 71 / 53 and 123 / 105), and the
// gradients of more than 48 rows take the matrix unit's time where there are few classes, too (64 x 1024 -> 1000: 36 / 32).
constexpr int kSmFewRows = 64, kSmFew = SM_TILES;
static bool sm_few(bool half, bool forward, int N, int I, int ol)
{
    if (!half || N < 1 || N > kSmFewRows) return false;
    const int want = forced_tile() - kSmFirstTile;
    if (want >= 0 && want <= kSmFew) return want == kSmFew;
    return forced_split() <= 0 && (ol >= 4096 || (I <= 2048 && (forward || N <= 48)));
}

// dx takes dz in two bf16 values, 16 bits of it, in every bf16 layer.  A row's dz add up to zero, so that what all classes' weights have in common cancels in dx, and what one value
// loses, 2^-9 of each term, does not: where the weights differ by a 32nd of their size one value left dx off by 40 to 70 times what its sums and its own rounding explain.
// us with two (one): 16 x 2048 -> 65536 262 (247), 777 x 1537 -> 20011 363 (321), 4096 x 4096 -> 65536 8450 (7090).
// dw takes it in three, all its 24 bits, in bf16 layers of up to so many products, and a sixteenth as many weights, where launches are most of what it costs: dw of 15 x 192
// -> 512 is off by 5.4e-7 of its size then (2.2e-6 with two).  Rows of one step, up to 64, take three, too, as their sums are too short to lose as much themselves.  A quarter of the
// time of larger layers would be for what their outputs' own sums lose.
constexpr double kSmLittle = (double)((size_t)1 << 28);
constexpr int kSmFewOfAll = 64;

// Scratch of a pass, laid out in order.
struct SmLayout {
    bool few;                   // few fp32 rows
    int strip;                  // classes of a work-group of their backward pass
    bool half, laid;            // fp32; w is laid out
    int isteps, piece, pieces;  // steps of memory of a row of x or w; classes of a piece, pieces
    int products;               // of outputs, per step of memory
    int products_x, products_w; // of dx and of dw
    int planes;                 // of dz
    SmPlan z, dx, dw;           // of a whole piece
    int pair;                   // the tile of dx and dw in one launch, or nothing
    SmPlan together;            // dx's part of it
    size_t x, w, xexp, wexp, xlows, wlows, least, top, label_out, dz, dz_dx, dxs, strips, partial, total;
    SmLayout(const owt_fc_desc *d, int ol, bool forward)
    {
        const int N = d->N, I = d->I;
        half = d->dtype == OWT_F32;
        isteps = up(I, 64);
        laid = half || I % 64;
        products = half ? SM_THREE : SM_ONE;
        const bool little = !half && (double)N * I * ol <= kSmLittle && (double)I * ol <= kSmLittle / 16;
        products_x = half ? SM_THREE : SM_PAIR;
        products_w = half || little || N <= kSmFewOfAll ? SM_THREE : SM_PAIR;
        planes = !half && products_w == SM_THREE ? 3 : 2;
        few = sm_few(half, forward, N, I, ol);
        if (few) {
            size_t at = 0;
            auto take = [&](size_t bytes) { const size_t was = at; at += (bytes + 255) / 256 * 256; return was; };
            x = w = xexp = wexp = xlows = wlows = least = top = label_out = dz = dz_dx = dxs = strips = partial = 0;
            piece = ol;
            pieces = 1;
            z = dx = dw = {SM_BIG, 1, 0.f};
            pair = SM_NOTHING;
            // of 256 columns: as many strips of classes as fill the chip at its registers' two or four work-groups a CU, unless their parts of dx grow beyond w itself
            const int across = up(I, 256), most = up(ol, 16), rows = up(N, 16);
            auto strip_of = [&](int groups) { return up(most, most < up(groups, across) ? most : up(groups, across)); };
            strip = strip_of(rows > 2 ? 512 : 1024);
            if (strip < rows) strip = rows < strip_of(256) ? rows : strip_of(256);
            strip *= 16;
            if (forward) {
                top = take((size_t)up(ol, 16 * few_blocks(N, ol)) * few_blocks(N, ol) * N * sizeof(Top));
                label_out = take((size_t)N * 4);
            } else {
                dz = take((size_t)N * few_pitch(ol) * 4);
                partial = take((size_t)up(ol, strip) * N * I * 4);
            }
            total = at;
            return;
        }
        const size_t row = (size_t)isteps * (half ? 256 : 128);
        auto plans = [&](int cols) {
            piece = cols;
            pieces = up(ol, cols);
            z = sm_plan(N, cols, isteps * products, products, forward ? SM_TOP : SM_DZ);
            if (forward) return;
            dx = sm_plan(N, I, up(cols, 64) * products_x, products_x, SM_OUT);
            // 64 x 64 results of two products read w for each: a second work-group on the CU hides what the first waits for (us with one and two: 16 x 2048 -> 65536 84 and 71,
            // 1 x 2048 -> 65536 83 and 55, 64 x 4096 -> 32768 88 and 86, 40 x 1024 -> 10000 10.7 and 10.3).  Not where its sums get shorter than eight steps of memory, the first
            // join is for less than 32, or more than 32 parts are joined (us of the whole pass with one and two: 3 x 784 -> 8393 41.4 and 42.0, 200 x 4096 -> 1024 42.4 and 45.0,
            // 28 x 347 -> 32768 69.9 and 73.7; 96 x 2048 -> 4345 51.1 and 48.7, 250 x 4000 -> 2048 70.5 and 68.6, 1316 x 192 -> 12742 100.8 and 92.4)
            const long groups = dx.tile == SM_SMALL && !half && forced_split() <= 0 ? (long)up(N, 64) * up(I, 64) * dx.splits : 0;
            if (groups > 128 && groups <= 256 && dx.splits <= 16 && up(cols, 64) / dx.splits >= (dx.splits > 1 ? 16 : 32)) dx.splits *= 2;
            // (few rows of many weights: the third product is behind the results' writing, 16 x 2048 -> 65536 148 us, 161 where the tile is chosen for it)
            const int shown = planes == 3 && (double)I * ol > kSmLittle / 16 ? SM_PAIR : products_w;
            dw = sm_plan(cols, I, up(N > 0 ? N : 1, 64) * shown, shown, SM_OUT);
        };
        auto us = [&] { return (float)pieces * (z.us + dx.us + dw.us); };
        if (forward) plans(forward_piece(laid, row, ol));
        else {
            plans(backward_piece(laid, half, N, row, ol, 0));
            // Pieces whose tiles come in whole rounds of the chip: of 4096 rows, 4096 -> 65536, eight of 8192 classes take 7.16 ms, six of up to 12288 7.5, eleven 8.1.
            const int fewest = pieces;
            if (fewest > 1) {
                int best = piece;
                float least_us = us();
                for (int more = 1; more <= fewest && more <= 6; more++) {
                    plans(backward_piece(laid, half, N, row, ol, more));
                    if (us() < 0.98f * least_us) {
                        least_us = us();
                        best = piece;
                    }
                }
                plans(best);
            }
        }
        if (forward && pieces > 1) z.splits = 1;        // (a split row's outputs are joined in one go)
        size_t at = 0;
        auto take = [&](size_t bytes) { const size_t was = at; at += (bytes + 255) / 256 * 256; return was; };
        const size_t rows = forward ? N : (size_t)up(N, 64) * 64;
        x = take(!forward || laid ? rows * row : 0);
        w = take(laid ? (size_t)piece * row : 0);
        xexp = take(half ? (size_t)N * 4 : 0);
        wexp = take(half ? (size_t)piece * 4 : 0);
        xlows = take(half && !forward ? (size_t)low_groups(rows) * 4 : 0);
        wlows = take(half && !forward ? (size_t)most_low_groups(piece) * 4 : 0);      // (the last piece may be shorter)
        least = take(half && !forward ? 8 : 0);
        pair = SM_NOTHING;
        top = label_out = dz = dz_dx = dxs = strips = partial = total = 0;
        if (forward) dx = dw = z;
        if (z.tile < 0) return;
        size_t parts = partial_bytes(z, N, piece);
        if (forward) {
            top = take(z.splits > 1 ? 0 : (size_t)pieces * up(piece, kSmTiles[z.tile].bn) * kSmTiles[z.tile].wn * N * sizeof(Top));
            label_out = take((size_t)N * 4);
        } else {
            const int psteps = up(piece, 64);
            dz = take((size_t)N * psteps * 128 * planes);
            dz_dx = take(half ? (size_t)N * psteps * 256 : 0);
            dxs = take(!half && pieces > 1 ? (size_t)N * I * 4 : 0);
            strips = take((size_t)strips_of(z, N) * piece * 4);
            pair = sm_pair(N, piece, I, products_x, products_w, dx, dw, together);
            if (pair != SM_NOTHING) {
                dx = together;
                dw = {pair, 1, 0.f};
            }
            const size_t a = partial_bytes(dx, N, I), b = partial_bytes(dw, piece, I);
            parts = parts > a ? parts : a;
            parts = parts > b ? parts : b;
        }
        partial = take(parts);
        total = N ? at : 0;
    }
    // Blocks of 16 classes of a work-group of the outputs: more of them read x less often, fewer fill the chip (us with 1, 2, 4: 1 x 2048 -> 65536 99, 130, 112,
    // 32 x 2048 -> 8192 26, 24, 31, 48 x 2048 -> 16384 61, 48, 43).  dz's rows.
    static int few_blocks(int N, int ol) { return N <= 16 || ol < 8192 ? 1 : ol < 16384 ? 2 : 4; }
    static int few_pitch(int ol) { return up(ol, 64) * 64; }
    bool fits() const { return z.tile >= 0 && dx.tile >= 0 && dw.tile >= 0; }
    // Classes of a piece: as many as `fit`, but pieces alike
    static int alike(size_t fit, size_t least, int ol, int more = 0)
    {
        fit = fit < least ? least : fit;
        if (fit >= (size_t)ol) return ol;
        const int pieces = (int)((ol + fit - 1) / fit) + more;
        return up(up(ol, pieces), 256) * 256;
    }
    // Weights that are laid out go in pieces of at most 256 MB; outputs are not kept, so that the others are one piece.
    static int forward_piece(bool laid, size_t row, int ol) { return laid ? alike(((size_t)256 << 20) / row, 256, ol) : ol; }
    // dz, and weights that are laid out, stay in the 256 MB behind the L2 caches between the product that writes them and those that read them
    static int backward_piece(bool laid, bool half, int N, size_t row, int ol, int more)
    {
        const size_t each = (size_t)N * (half ? 8 : 4) + (laid ? row : 0);
        return alike(((size_t)128 << 20) / (each ? each : 1), 1024, ol, more);
    }
};

static owt_status check_fits(const SmLayout &l) { return l.fits() ? OWT_OK : fail(OWT_EUNSUPPORTED, "more work-groups than a launch holds"); }

static hipError_t launch(bool half, int product, int tile, const SmParams &p, hipStream_t s)
{
    const bool ends = product == SM_PRODUCT_TOP || product == SM_PRODUCT_DZ;
    if (half) return ends ? owt_launch_softmax_half_ends(product, tile, p, s) : owt_launch_softmax_half_out(product, tile, p, s);
    return ends ? owt_launch_softmax_bf16_ends(product, tile, p, s) : owt_launch_softmax_bf16_out(product, tile, p, s);
}
// Numbers the tiles of a product; a plan for a whole piece serves the last one, too.
static void lay_tiles(SmParams &p, const SmPlan &pl)
{
    const SmTileCost &q = kSmTiles[pl.tile];
    p.tiles_n = up(p.N, q.bn);
    p.tiles = p.tiles_n * up(p.M, q.bm);
    p.splits = pl.splits;
    p.steps_per_split = up(p.steps / p.products, pl.splits) * p.products;
}
static unsigned groups_of(size_t n, size_t most)
{
    const size_t g = (n + 255) / 256;
    return (unsigned)(g < most ? g : most);
}
static void join_parts(bool half, const SmParams &p, hipStream_t s)
{
    const dim3 grid(groups_of((size_t)p.M * ((p.N + 3) / 4), 8192));
    if (half) hipLaunchKernelGGL(sm_join_kernel<true>, grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL(sm_join_kernel<false>, grid, dim3(256), 0, s, p);
}
static hipError_t results(bool half, int product, SmParams p, const SmPlan &pl, hipStream_t s)
{
    lay_tiles(p, pl);
    const hipError_t e = launch(half, product, pl.tile, p, s);
    if (e == hipSuccess && pl.splits > 1) join_parts(half, p, s);
    return e;
}

static owt_status launched(hipError_t e = hipSuccess)
{
    if (e == hipSuccess) e = hipGetLastError();
    return e == hipSuccess ? OWT_OK : fail(OWT_ELAUNCH, "HIP launch failed: %s", hipGetErrorString(e));
}

// x, or a piece of w, as operands of the products
struct SmSource {
    const owt_fc_desc *d;
    const SmLayout &l;
    char *ws;
    hipStream_t s;

    SmOperand along(const void *at, int rows) const
    {
        const int planes = l.half ? 2 : 1;
        return {(const unsigned char *)at, (size_t)l.isteps * 128 * planes, (size_t)(128 * planes), rows, 0, planes};
    }
    static SmOperand across(const SmOperand &o, int rows, int steps)
    {
        return {o.at, o.ld, 64 * o.ld, rows, 8 * steps, o.planes};
    }
    // x for the products: backward, rows without a class and those up to a whole step are zeros
    SmPrep x_rows(const void *from, const int *labels, const float *weight, bool forward) const
    {
        SmPrep p;
        memset(&p, 0, sizeof(p));
        p.from = from;
        p.to = (unsigned char *)(ws + l.x);
        p.rows = d->N;
        p.out_rows = forward ? d->N : up(d->N, 64) * 64;
        p.cols = d->I;
        p.steps = l.isteps;
        p.labels = forward ? nullptr : labels;
        p.classes = d->O_total;
        p.weight = weight;
        p.exps = (int *)(ws + l.xexp);
        p.lows = forward ? nullptr : (int *)(ws + l.xlows);
        return p;
    }
    SmPrep w_rows(const void *from, int v0, int cols, bool forward) const
    {
        SmPrep p;
        memset(&p, 0, sizeof(p));
        p.from = (const char *)from + (size_t)v0 * d->I * (l.half ? 4 : 2);
        p.to = (unsigned char *)(ws + l.w);
        p.rows = p.out_rows = cols;
        p.cols = d->I;
        p.steps = l.isteps;
        p.exps = (int *)(ws + l.wexp);
        p.lows = forward ? nullptr : (int *)(ws + l.wlows);
        return p;
    }
    void lay(const SmPrep &a, const SmPrep &b) const
    {
        if (l.half) {
            // (x's and w's work-groups are of one kind where both are few or both are many; else each has a launch)
            const bool many_a = a.out_rows >= 4096, many_b = b.out_rows >= 4096;
            if (a.out_rows && b.out_rows && many_a != many_b) {
                SmPrep none;
                memset(&none, 0, sizeof(none));
                lay(a, none);
                lay(none, b);
                return;
            }
            const int ga = low_groups(a.out_rows), gb = low_groups(b.out_rows);
            if (many_a || many_b) hipLaunchKernelGGL(sm_halves_kernel<4>, dim3((unsigned)(ga + gb)), dim3(256), 0, s, a, b, ga);
            else hipLaunchKernelGGL(sm_halves_kernel<1>, dim3((unsigned)(ga + gb)), dim3(256), 0, s, a, b, ga);
        } else {
            auto groups = [&](const SmPrep &p) { const long n = (long)p.out_rows * up(p.steps * 8, 256); return (int)(n < 8192 ? n : 8192); };
            hipLaunchKernelGGL(sm_rows_kernel, dim3((unsigned)(groups(a) + groups(b))), dim3(256), 0, s, a, b, groups(a));
        }
    }
    // operands of a piece's outputs; x is laid out with the first
    void operands(const void *x, const void *w, int piece, int v0, int cols, const int *labels, const float *weight, bool forward, SmOperand &xo, SmOperand &wo) const
    {
        if (l.laid) {
            SmPrep a = x_rows(x, labels, weight, forward);
            if (piece) a.out_rows = 0;
            lay(a, w_rows(w, v0, cols, forward));
        }
        xo = along(l.laid ? ws + l.x : x, d->N);
        wo = along(l.laid ? ws + l.w : (const char *)w + (size_t)v0 * d->I * 2, cols);
    }
};

// outputs of a piece: what TOP, DZ and Z have in common
static SmParams outputs(const owt_fc_desc *d, const SmLayout &l, char *ws, const SmOperand &x, const SmOperand &w, int ol, int v0, int cols, const float *bias,
                        const int *labels)
{
    SmParams p;
    memset(&p, 0, sizeof(p));
    p.a = x;
    p.b = w;
    p.M = d->N;
    p.N = cols;
    p.products = l.products;
    p.steps = l.isteps * l.products;
    p.bias = bias ? bias + v0 : nullptr;
    p.row_exp = (const int *)(ws + l.xexp);
    p.col_exp = (const int *)(ws + l.wexp);
    p.labels = labels;
    p.classes = d->O_total;
    p.off = d->rank * ol + v0;
    p.alpha = 1.f;
    p.partial = (float *)(ws + l.partial);
    lay_tiles(p, l.z);
    return p;
}

// What the passes over few rows have in common, and their launches by blocks of 16 rows
static SmFewParams few_params(const owt_fc_desc *d, const SmLayout &l, int ol, const void *x, const void *w, const float *bias, const int *labels, char *ws)
{
    SmFewParams f;
    memset(&f, 0, sizeof(f));
    f.x = (const float *)x;
    f.w = (const float *)w;
    f.I = d->I;
    f.dz = (float *)(ws + l.dz);
    f.pitch = SmLayout::few_pitch(ol);
    f.p.M = d->N;
    f.p.N = ol;
    f.p.bias = bias;
    f.p.labels = labels;
    f.p.classes = d->O_total;
    f.p.off = d->rank * ol;
    f.strip = l.strip;
    f.strips = up(ol, l.strip);
    return f;
}
template <int NB, bool DZ> static void few_outputs(const SmFewParams &f, hipStream_t s)
{
    const int blocks = SmLayout::few_blocks(f.p.M, f.p.N);
    const dim3 grid((unsigned)up(f.p.N, 16 * blocks));
    if constexpr (NB > 1) {
        if (blocks == 4) { hipLaunchKernelGGL((sm_few_kernel<NB, 4, DZ>), grid, dim3(256), 0, s, f); return; }
        if (blocks == 2) { hipLaunchKernelGGL((sm_few_kernel<NB, 2, DZ>), grid, dim3(256), 0, s, f); return; }
    }
    hipLaunchKernelGGL((sm_few_kernel<NB, 1, DZ>), grid, dim3(256), 0, s, f);
}
template <bool DZ> static void few_outputs(const SmFewParams &f, hipStream_t s)
{
    switch (up(f.p.M, 16)) {
    case 1: return few_outputs<1, DZ>(f, s);
    case 2: return few_outputs<2, DZ>(f, s);
    case 3: return few_outputs<3, DZ>(f, s);
    default: return few_outputs<4, DZ>(f, s);
    }
}
static void few_gradients(const SmFewParams &f, hipStream_t s)
{
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)up(f.I, 256), (unsigned)f.strips), dim3(256), 0, s, f); };
    switch (up(f.p.M, 16)) {
    case 1: return go(sm_few_back_kernel<1>);
    case 2: return go(sm_few_back_kernel<2>);
    case 3: return go(sm_few_back_kernel<3>);
    default: return go(sm_few_back_kernel<4>);
    }
}

static owt_status forward(const owt_fc_desc *d, const SmLayout &l, int ol, const void *x, const void *w, const float *bias, const int *labels, float *lse, float *target,
                          float *loss, char *ws, hipStream_t s)
{
    const SmSource from{d, l, ws, s};
    SmRows r = {(const Top *)(ws + l.top), 0, d->N, (const float *)(ws + l.label_out), labels, d->O_total, d->rank * ol, ol, lse, target, loss};
    if (l.few) {
        SmFewParams f = few_params(d, l, ol, x, w, bias, labels, ws);
        f.p.top = (Top *)(ws + l.top);
        f.p.target = (float *)(ws + l.label_out);
        few_outputs<false>(f, s);
        const int blocks = SmLayout::few_blocks(d->N, ol);
        r.parts = up(ol, 16 * blocks) * blocks;
    }
    for (int k = 0; k < (l.few ? 0 : l.pieces); k++) {
        const int v0 = k * l.piece, cols = ol - v0 < l.piece ? ol - v0 : l.piece;
        SmOperand xo, wo;
        from.operands(x, w, k, v0, cols, nullptr, nullptr, true, xo, wo);
        SmParams p = outputs(d, l, ws, xo, wo, ol, v0, cols, bias, labels);
        p.target = (float *)(ws + l.label_out);
        p.top = (Top *)(ws + l.top) + (size_t)r.parts * d->N;
        if (p.splits > 1) {
            const hipError_t e = launch(l.half, SM_PRODUCT_Z, l.z.tile, p, s);
            if (e != hipSuccess) return launched(e);
            if (l.half) hipLaunchKernelGGL(sm_split_top_kernel<true>, dim3((unsigned)d->N), dim3(256), 0, s, p, r);
            else hipLaunchKernelGGL(sm_split_top_kernel<false>, dim3((unsigned)d->N), dim3(256), 0, s, p, r);
            return launched();
        }
        const hipError_t e = launch(l.half, SM_PRODUCT_TOP, l.z.tile, p, s);
        if (e != hipSuccess) return launched(e);
        r.parts += p.tiles_n * kSmTiles[l.z.tile].wn;
    }
    if (d->N > 1024) hipLaunchKernelGGL(sm_finish_kernel<8>, dim3((unsigned)up(d->N, 32)), dim3(256), 0, s, r);
    else hipLaunchKernelGGL(sm_finish_kernel<256>, dim3((unsigned)d->N), dim3(256), 0, s, r);
    return launched();
}

static owt_status backward(const owt_fc_desc *d, const SmLayout &l, int ol, const void *x, const void *w, const float *bias, const int *labels, const float *lse,
                           const float *weight, float alpha, float beta, void *dx, float *dw, float *db, char *ws, hipStream_t s)
{
    SmParams none;
    memset(&none, 0, sizeof(none));
    if (d->N == 0) {            // sums of nothing
        none.M = ol;
        none.N = d->I;
        none.alpha = alpha;
        none.beta = beta;
        none.out = dw;
        join_parts(false, none, s);
        if (db) {
            none.N = 1;
            none.out = db;
            join_parts(false, none, s);
        }
        return launched();
    }
    if (l.few) {
        SmFewParams f = few_params(d, l, ol, x, w, bias, labels, ws);
        f.p.lse = lse;
        f.p.weight = weight;
        few_outputs<true>(f, s);
        f.p.alpha = alpha;
        f.p.beta = beta;
        f.p.out = dw;
        f.p.db = db;
        f.p.big = (size_t)ol * d->I * 4 > (32u << 20) && d->I % 32 == 0;
        f.p.partial = dx ? (float *)(ws + l.partial) : nullptr;
        few_gradients(f, s);
        if (dx) {
            f.p.out = dx;
            hipLaunchKernelGGL(sm_few_join_kernel, dim3((unsigned)up((size_t)d->N * d->I, 256)), dim3(1024), 0, s, f);
        }
        return launched();
    }
    const SmSource from{d, l, ws, s};
    const int nsteps = up(d->N, 64), step = 128 * l.planes;
    int *least = (int *)(ws + l.least);
    for (int k = 0; k < l.pieces; k++) {
        const int v0 = k * l.piece, cols = ol - v0 < l.piece ? ol - v0 : l.piece, psteps = up(cols, 64);
        SmOperand xo, wo;
        from.operands(x, w, k, v0, cols, labels, weight, false, xo, wo);
        SmParams p = outputs(d, l, ws, xo, wo, ol, v0, cols, bias, labels);
        p.lse = lse;
        p.weight = weight;
        p.dz = (unsigned char *)(ws + l.dz);
        p.dz_dx = (unsigned char *)(ws + l.dz_dx);
        p.dz_ld = (size_t)psteps * step;
        p.dz_step = step;
        p.lows_x = (const int *)(ws + l.xlows);
        p.lows_w = (const int *)(ws + l.wlows);
        p.num_x = low_groups(up(d->N, 64) * 64);
        p.num_w = low_groups(cols);
        p.least = least;
        p.dbias = db ? (float *)(ws + l.strips) : nullptr;
        if (!l.laid && k == 0) p.copy = from.x_rows(x, labels, nullptr, false);
        hipError_t e = launch(l.half, p.splits > 1 ? SM_PRODUCT_Z : SM_PRODUCT_DZ, l.z.tile, p, s);
        if (e != hipSuccess) return launched(e);
        if (p.splits > 1) {
            const dim3 grid((unsigned)psteps, (unsigned)up(d->N, 32));
            if (l.half) hipLaunchKernelGGL(sm_split_dz_kernel<true>, grid, dim3(256), 0, s, p);
            else hipLaunchKernelGGL(sm_split_dz_kernel<false>, grid, dim3(256), 0, s, p);
        }

        SmParams qx = none;
        if (dx) {
            SmParams &q = qx;
            q.a = {l.half ? p.dz_dx : p.dz, p.dz_ld, (size_t)step, d->N, 0, l.planes};
            q.b = SmSource::across(wo, cols, l.isteps);
            q.M = d->N;
            q.N = d->I;
            q.products = l.products_x;
            q.steps = psteps * q.products;
            q.labels = labels;
            q.classes = d->O_total;
            q.weight = weight;
            q.alpha = 1.f;
            q.under = least + 1;
            q.partial = p.partial;
            float *sums = l.half ? (float *)dx : (float *)(ws + l.dxs);
            const bool last = k == l.pieces - 1;
            q.add = k ? sums : nullptr;
            q.out = last ? dx : sums;
            q.bf16 = last && !l.half;
            lay_tiles(q, l.dx);
        }
        SmParams q = none;
        q.a = {p.dz, p.dz_ld, 64 * p.dz_ld, d->N, 8 * psteps, l.planes};
        q.b = SmSource::across(from.along(ws + l.x, d->N), nsteps * 64, l.isteps);
        q.M = cols;
        q.N = d->I;
        q.products = l.products_w;
        q.steps = nsteps * l.products_w;
        q.alpha = alpha;
        q.beta = beta;
        q.under = least;
        q.partial = p.partial;
        q.out = dw + (size_t)v0 * d->I;
        q.big = (size_t)ol * d->I * 4 > (32u << 20) && d->I % 32 == 0;        // (rows of whole lines of 128 bytes: parts of lines join in the caches)
        q.dbias = p.dbias;
        q.strips = strips_of(l.z, d->N);
        q.db = db ? db + v0 : nullptr;
        lay_tiles(q, l.dw);
        if (dx && l.pair != SM_NOTHING) {
            e = l.half ? owt_launch_softmax_half_pair(l.pair, qx, q, qx.steps_per_split >= q.steps, s) : owt_launch_softmax_bf16_pair(l.pair, qx, q, qx.steps_per_split >= q.steps, s);
            if (e != hipSuccess) return launched(e);
            if (qx.splits > 1) join_parts(l.half, qx, s);
        } else {
            if (dx && (e = results(l.half, SM_PRODUCT_DX, qx, l.dx, s)) != hipSuccess) return launched(e);
            if ((e = results(l.half, SM_PRODUCT_DW, q, l.dw, s)) != hipSuccess) return launched(e);
        }
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
    const SmLayout l(d, ol, pass == OWT_PASS_FWD);
    if (check_fits(l) != OWT_OK) return (size_t)-1;
    return l.total;
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
    const SmLayout l(d, ol, true);
    OWT_TRY(check_fits(l));
    OWT_TRY(need_ws(ws, ws_bytes, l.total));
    const float *b = (d->flags & OWT_BIAS) ? bias : nullptr;
    hipStream_t s = (hipStream_t)hip_stream;
    return forward(d, l, ol, x, w, b, labels_or_null, lse, target_or_null, loss_or_null, (char *)ws, s);
}

owt_status owt_softmax_join(int workers, int N, int classes, const float *lses, const float *targets, const int *labels, float *lse,
                            float *target_or_null, float *loss_or_null, void *hip_stream)
{
    if (workers <= 0 || N < 0 || classes <= 0) return fail(OWT_EINVAL, "workers and classes must be positive, N not negative");
    if (N == 0) return OWT_OK;
    OWT_TRY(need_ptr(lses, "lses")); OWT_TRY(need_ptr(targets, "targets")); OWT_TRY(need_ptr(labels, "labels")); OWT_TRY(need_ptr(lse, "lse"));
    OWT_TRY(may_ptr(target_or_null, "target")); OWT_TRY(may_ptr(loss_or_null, "loss"));
    hipLaunchKernelGGL(softmax_join_kernel, dim3(((unsigned)N + 255) / 256), dim3(256), 0, (hipStream_t)hip_stream, workers, N, classes, lses, targets, labels, lse,
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
    const SmLayout l(d, ol, false);
    OWT_TRY(check_fits(l));
    OWT_TRY(need_ws(ws, ws_bytes, l.total));
    const float *b = (d->flags & OWT_BIAS) ? bias : nullptr;
    hipStream_t s = (hipStream_t)hip_stream;
    return backward(d, l, ol, x, w, b, labels, lse, weight_or_null, alpha, beta, dx_partial_or_null, dw, dbias_or_null, (char *)ws, s);
}

}  // extern "C"

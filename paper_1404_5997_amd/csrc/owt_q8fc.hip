// The fully-connected column shard in 8 bits: entry points of q8gemm.hpp, q8prep.hpp, q8few.hpp and q8fewbwd.hpp.
#include <cmath>
#include <initializer_list>

#include "owt_host.hpp"
#include "q8.hpp"
#include "q8few.hpp"
#include "q8fewbwd.hpp"
#include "q8gemm.hpp"
#include "q8prep.hpp"

namespace owt {

// Tiles of the products, 256 x 256, 128 x 128 and 64 x 64 (owt_test_force_variant: 110.. name these), the forward product's kernel for few
// results (113) and the backward pass in one launch (114).
constexpr int kNumQ8Tiles = 3, kQ8FirstTile = 110, kQ8Few = 3, kQ8FewBwd = 4;
// What a work-group takes: `start` for its beginning and end, `step` for a step on a quiet chip, `busy` where 128 or more run (256 x 256:
// all 256; the chip is then bound by its power).  us, fitted to 20 products of 1 x 1024 -> 1024 to 8192 x 4096 -> 8192 with every tile and split.
struct Q8Tile { int bm, bn; float start, step, busy; };
static const Q8Tile kQ8Tiles[kNumQ8Tiles] = {{256, 256, 11.f, 1.05f, 1.5f}, {128, 128, 3.f, 0.4f, 0.55f}, {64, 64, 1.2f, 0.21f, 0.21f}};

template <class Op> static hipError_t launch_tile(int t, const Q8GemmParams &p, hipStream_t s)
{
    const dim3 grid((unsigned)owt_split_major_grid(p.tiles, p.splits));
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, p); };
    if (t == 0) {
        // two planes: step by step where a sum is of four pairs or fewer (us, by steps and by pairs: dx of 8192 x 9216 from 64 outputs 69 and 72,
        // from 256 107 and 109, from 512 166 and 164; dw of 8192 x 4096 -> 4096 466 and 432)
        bool paired = false;
        if constexpr (std::is_same<Op, Q8Half>::value) {
            paired = p.ksteps_per_split > 8;
            if (paired) go(q8gemm_kernel<Op, 2, 2, 4, 4, 5, true, 1>);
        }
        if (!paired) go(q8gemm_kernel<Op, 2, 2, 4, 4, 2, false, 1>);
    } else if (t == 1) go(q8gemm_kernel<Op, 2, 2, 2, 2, 3, false, 1>);
    else go(q8gemm_kernel<Op, 2, 2, 1, 1, 4, false, 2>);
    return hipGetLastError();
}

struct Q8Plan { int tile, splits; float us; };
static Q8Plan q8_plan(long M, long N, int ksteps, bool forward)
{
    Q8Plan best{0, 1, 0.f};
    float &least = best.us;
    least = 1e30f;
    const int want = forced_tile() - kQ8FirstTile, want_split = forced_split();
    if (forward && want == kQ8Few) return {kQ8Few, 1, 0.f};
    for (int t = 0; t < kNumQ8Tiles; t++) {
        if (want >= 0 && want < kNumQ8Tiles && t != want) continue;
        const Q8Tile &q = kQ8Tiles[t];
        const long tiles = ((M + q.bm - 1) / q.bm) * ((N + q.bn - 1) / q.bn);
        for (int sp = 1; sp <= 32 && (sp == 1 || (sp * 2 <= ksteps && tiles * sp <= 1024)); sp *= 2) {
            const long each = (tiles * sp + 255) / 256;         // work-groups of a CU
            const float step = tiles * sp >= (t == 0 ? 256 : 128) ? q.busy : q.step;
            float us = 3.f + (float)each * (q.start + (float)((ksteps + sp - 1) / sp) * step);
            if (sp > 1) us += 3.6f + (float)(sp + 1) * (float)M * (float)N * 4.f / 3e6f;        // the launch that adds up
            if (us < least) best = {t, sp, us};
        }
    }
    if (want_split > 0) best.splits = want_split < ksteps ? want_split : ksteps;
    else if (forward && want < 0) {     // 16 x 16 results a work-group (us, this and the best of the tiles: 16 rows of 4096 -> 4096 5.2 and 9, 64 rows 11 and 10)
        const long tiles = ((M + 15) / 16) * ((N + 15) / 16);
        if (3.f + (float)((tiles + 255) / 256) * (1.1f + 0.035f * (float)ksteps) < least) best = {kQ8Few, 1, 0.f};
    }
    return best;
}

// Both backward products in one launch of the same tile: the two tiles that have one.  0: apart they take less (`least` on entry; it
// leaves as what the choice takes).
static int q8_pair_tile(long N, long I, long O, int dx_steps, int dw_steps, float &least)
{
    const int want = forced_tile() - kQ8FirstTile;
    if (forced_split() > 0) return 0;
    int best = 0;
    for (int t = 1; t < kNumQ8Tiles; t++) {
        if (want >= 0 && want < kNumQ8Tiles && t != want) continue;
        const Q8Tile &q = kQ8Tiles[t];
        const float tx = (float)(((N + q.bm - 1) / q.bm) * ((I + q.bn - 1) / q.bn)), tw = (float)(((O + q.bm - 1) / q.bm) * ((I + q.bn - 1) / q.bn));
        const float ux = q.start + (float)dx_steps * q.busy, uw = q.start + (float)dw_steps * q.busy;
        const float longest = ux > uw ? ux : uw, sum = (tx * ux + tw * uw) / 256.f + 0.2f * longest;
        const float us = 3.f + (sum > longest ? sum : longest);
        if (us < least) { least = us; best = t; }
    }
    return best;
}

// The whole backward pass in one launch (q8fewbwd.hpp), where that takes less than the preparation and the products.  us, fitted to both sides of
// 65 shapes from 1 x 512 -> 512 to 64 x 9216 -> 9216 in both types, with dx and without; the choice then takes 0.5 % (bf16 0.8 %) longer than the
// faster side on average.  (This and the rest, fp32: 128 rows of 512 -> 128 7.0 and 14.9, of 9216 -> 512 19.0 and 26.9, 256 rows of 4096 -> 4096 88 and 78,
// 8192 of 512 -> 125 90 and 45.)
static bool q8_few_bwd_is(float products, bool with_dx, long N, long I, long O, bool bf16)
{
    const int want = forced_tile() - kQ8FirstTile;
    if (want >= 0 || forced_split() > 0) return want == kQ8FewBwd;
    const float dz = (float)(bf16 ? 16 : 20) * (float)N * (float)O, x = 3.f * (float)N * (float)I, w = 3.f * (float)O * (float)I;    // bytes of the preparation
    const float rest = products + (with_dx ? 11.f + (dz + x + w) / 7e6f : 6.f + (dz + x) / 5e6f);
    const float its = (float)((I + 127) / 128), tx = with_dx ? its * (float)((N + 31) / 32) : 0.f, tw = its * (float)((O + 31) / 32);   // work-groups
    const float part = bf16 ? 0.65f : 1.f, sx = part * (float)((O + 15) / 16), sw = (float)((N + 15) / 16);                         // steps
    const float longest = 2.5f + 0.65f * fmaxf(with_dx ? sx / 4.f : 0.f, ceilf(sw / 4.f));
    const float all = (tx + tw) * 2.5f / 768.f + (tx * sx + tw * sw) * 0.45f / 1024.f;
    return 3.f + fmaxf(longest, all + 0.4f * longest) < rest;
}

static size_t partial_bytes(const Q8Plan &pl, long M, long N) { return pl.splits > 1 ? (size_t)pl.splits * M * N * 4 : 0; }

// Whether a launch holds the tiles of a product.
static bool product_fits(const Q8Plan &pl, long M, long N)
{
    const Q8Tile &q = kQ8Tiles[pl.tile];
    return groups_fit(((M + q.bm - 1) / q.bm) * ((N + q.bn - 1) / q.bn) * pl.splits, 256);
}
static owt_status too_many_groups() { return fail(OWT_EUNSUPPORTED, "more work-groups than a launch holds"); }

// Numbers the tiles of a product.
static void lay_tiles(Q8GemmParams &p, const Q8Plan &pl)
{
    const Q8Tile &q = kQ8Tiles[pl.tile];
    p.tiles_n = (p.N + q.bn - 1) / q.bn;
    p.tiles = p.tiles_n * ((p.M + q.bm - 1) / q.bm);
    p.splits = pl.splits;
    p.big = (size_t)p.M * p.N * (p.bf16 ? 2 : 4) > (32u << 20);
    p.ksteps_per_split = ((p.ksteps / p.planes + pl.splits - 1) / pl.splits) * p.planes;
}

template <class Op> static owt_status run_product(Q8GemmParams p, const Q8Plan &pl, void *partial, hipStream_t s)
{
    lay_tiles(p, pl);
    p.partial = partial;
    hipError_t e = launch_tile<Op>(pl.tile, p, s);
    if (e == hipSuccess && pl.splits > 1) {
        const size_t n = (size_t)p.M * ((p.N + 3) / 4), want = (n + 255) / 256;
        hipLaunchKernelGGL(q8_join_kernel<Op>, dim3((unsigned)(want < 8192 ? want : 8192)), dim3(256), 0, s, p);
        e = hipGetLastError();
    }
    return e == hipSuccess ? OWT_OK : fail(OWT_ELAUNCH, "HIP launch failed: %s", hipGetErrorString(e));
}

constexpr int kQ8MaxI = 131071;         // 128 * 128 * 131071 < 2^31: no sum of products leaves 32 bits
constexpr int kQ8MaxRows = 1 << 22;     // of x and of w
// an operand's row, two f16 planes of kQ8MaxRows values or kQ8MaxI bytes: the last of a tile's 256 is addressed from the first with 32 bits
static_assert(255ull * (kQ8MaxRows / 64 * 256ull) + 128 <= 0xffffffffull && kQ8MaxI < kQ8MaxRows, "offsets within a tile fit 32 bits");

static owt_status check_q8_fc(const owt_fc_desc *d, int &o_local)
{
    if (!d) return fail(OWT_EINVAL, "descriptor is NULL");
    if (d->N < 0 || d->I <= 0 || d->O_total <= 0 || d->workers <= 0)
        return fail(OWT_EINVAL, "N must not be negative; I, O_total and workers must be positive");
    if (d->rank < 0 || d->rank >= d->workers) return fail(OWT_EINVAL, "need 0 <= rank < workers");
    if (d->O_total % d->workers) return fail(OWT_EINVAL, "O_total must be divisible by workers");
    if (d->dtype != OWT_F32 && d->dtype != OWT_BF16) return fail(OWT_EINVAL, "unknown dtype %d", (int)d->dtype);
    if (d->flags & ~(unsigned)(OWT_BIAS | OWT_RELU)) return fail(OWT_EINVAL, "unknown flag bits 0x%x", d->flags);
    o_local = d->O_total / d->workers;
    if (d->I > kQ8MaxI) return fail(OWT_EUNSUPPORTED, "more than %d inputs", kQ8MaxI);
    if (d->N > kQ8MaxRows || o_local > kQ8MaxRows) return fail(OWT_EUNSUPPORTED, "more than 2^22 rows or columns");
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

// The backward pass's scratch, laid out in order; `take` returns the offset of each part.
struct Q8BwdLayout {
    int nk, ok, strips, strip_rows, pair;
    float both_us;                      // both products
    Q8Plan dw, dx;
    size_t colsum, colmax, rowmax, cexp, rexp, aw, ax, bw, bx, partial, total;
    Q8BwdLayout(int N, int I, int O)
    {
        nk = N > 0 ? (N + 63) / 64 : 1;
        ok = (O + 63) / 64;
        // strips: enough parts of 64 columns for the chip, no more than 64 to add up, and 64 rows or more each
        long want = (2048 + ok - 1) / ok;
        want = want > 64 ? 64 : want;
        long rows = (N + want - 1) / want;
        rows = (rows + 63) / 64 * 64;
        rows = rows < 64 ? 64 : rows;
        strip_rows = (int)rows;
        strips = (int)((N + rows - 1) / rows);
        dw = q8_plan(O, I, 2 * nk, false);
        dx = q8_plan(N, I, 2 * ok, false);
        both_us = dx.us + dw.us;
        pair = q8_pair_tile(N, I, O, 2 * ok, 2 * nk, both_us);
        size_t at = 0;
        auto take = [&](size_t bytes) { const size_t was = at; at += (bytes + 255) / 256 * 256; return was; };
        colsum = take((size_t)strips * O * 4);
        colmax = take((size_t)strips * O * 4);
        rowmax = take((size_t)ok * N * 4);
        cexp = take((size_t)O * 4);
        rexp = take((size_t)N * 4);
        aw = take((size_t)O * nk * 256);
        ax = take((size_t)N * ok * 256);
        bw = take((size_t)I * nk * 128);
        bx = take((size_t)I * ok * 128);
        const size_t a = partial_bytes(dw, O, I), b = partial_bytes(dx, N, I);
        partial = take(a > b ? a : b);
        total = at;
    }
};

}  // namespace owt

using namespace owt;
#define OWT_TRY(e) do { const owt_status st_ = (e); if (st_ != OWT_OK) return st_; } while (0)

extern "C" {

size_t owt_fc_shard_q8_workspace_bytes(const owt_fc_desc *d, int pass)
{
    int ol;
    if (pass < 0 || pass > 2) { fail(OWT_EINVAL, "pass must be 0, 1 or 2"); return (size_t)-1; }
    if (check_q8_fc(d, ol) != OWT_OK) return (size_t)-1;
    if (pass == OWT_PASS_FWD) {
        if (d->N == 0) return 0;
        const int ks = (int)(q8_pitch(d->I) / 128);
        return partial_bytes(q8_plan(d->N, ol, ks, true), d->N, ol);
    }
    return Q8BwdLayout(d->N, d->I, ol).total;
}

owt_status owt_fc_shard_q8_fwd(const owt_fc_desc *d, const signed char *xq, const float *xscale, const signed char *wq, const float *wscale,
                               const float *bias, void *y, void *ws, size_t ws_bytes, void *hip_stream)
{
    int ol;
    OWT_TRY(check_q8_fc(d, ol));
    if (d->N == 0) return OWT_OK;
    OWT_TRY(need_ptr(xq, "xq")); OWT_TRY(need_ptr(xscale, "xscale")); OWT_TRY(need_ptr(wq, "wq")); OWT_TRY(need_ptr(wscale, "wscale"));
    OWT_TRY(need_ptr(y, "y"));
    if (d->flags & OWT_BIAS) OWT_TRY(need_ptr(bias, "bias"));
    const size_t pitch = q8_pitch(d->I);
    const Q8Plan pl = q8_plan(d->N, ol, (int)(pitch / 128), true);
    OWT_TRY(need_ws(ws, ws_bytes, partial_bytes(pl, d->N, ol)));
    Q8GemmParams p;
    memset(&p, 0, sizeof(p));
    p.a = (const unsigned char *)xq; p.b = (const unsigned char *)wq;
    p.lda = p.ldb = pitch;
    p.M = d->N; p.N = ol; p.ksteps = (int)(pitch / 128); p.planes = 1;
    p.out = y; p.bf16 = d->dtype == OWT_BF16;
    p.f = {xscale, wscale, (d->flags & OWT_BIAS) ? bias : nullptr, (d->flags & OWT_RELU) ? 0.f : -INFINITY};
    if (pl.tile == kQ8Few) {
        const long tiles = (long)((p.M + 15) / 16) * ((p.N + 15) / 16);
        if (!groups_fit(tiles, 1024)) return too_many_groups();
        p.tiles = (int)tiles;
        hipLaunchKernelGGL(q8_few_kernel, dim3((unsigned)owt_split_major_grid(p.tiles, 1)), dim3(1024), 0, (hipStream_t)hip_stream, p);
        const hipError_t e = hipGetLastError();
        return e == hipSuccess ? OWT_OK : fail(OWT_ELAUNCH, "HIP launch failed: %s", hipGetErrorString(e));
    }
    if (!product_fits(pl, d->N, ol)) return too_many_groups();
    return run_product<Q8Int>(p, pl, ws, (hipStream_t)hip_stream);
}

owt_status owt_fc_shard_q8_bwd(const owt_fc_desc *d, const signed char *xq, const float *xscale, const signed char *wq, const float *wscale,
                               const void *y_or_null, const void *dy, float alpha, float beta, void *dx_partial_or_null, float *dw,
                               float *dbias_or_null, void *ws, size_t ws_bytes, void *hip_stream)
{
    int ol;
    OWT_TRY(check_q8_fc(d, ol));
    if (!std::isfinite(alpha) || !std::isfinite(beta)) return fail(OWT_EINVAL, "alpha and beta must be finite");
    OWT_TRY(need_ptr(dw, "dw"));
    OWT_TRY(need_ptr(wq, "wq")); OWT_TRY(need_ptr(wscale, "wscale"));
    OWT_TRY(may_ptr(dx_partial_or_null, "dx_partial")); OWT_TRY(may_ptr(dbias_or_null, "dbias"));
    if (d->N > 0) {
        OWT_TRY(need_ptr(xq, "xq")); OWT_TRY(need_ptr(xscale, "xscale")); OWT_TRY(need_ptr(dy, "dy"));
        if (d->flags & OWT_RELU) OWT_TRY(need_ptr(y_or_null, "y (needed for the ReLU mask)"));
    }
    const bool bf16 = d->dtype == OWT_BF16, want_dx = dx_partial_or_null && d->N > 0;
    const Q8BwdLayout l(d->N, d->I, ol);
    OWT_TRY(need_ws(ws, ws_bytes, l.total));
    hipStream_t s = (hipStream_t)hip_stream;
    char *at = (char *)ws;
    if (q8_few_bwd_is(want_dx ? l.both_us : l.dw.us, want_dx, d->N, d->I, ol, bf16)) {
        Q8FewBwdParams f = {dy, (d->flags & OWT_RELU) ? y_or_null : nullptr, xscale, wscale, xq, wq, d->N, d->I, ol, q8_pitch(d->I), alpha, beta,
                            dx_partial_or_null, dw, dbias_or_null, 0, 0};
        const long its = (d->I + 127) / 128;
        const long tw = (ol + 31) / 32 * its, tx = want_dx ? (d->N + 31) / 32 * its : 0;
        if (!groups_fit(tw + tx + 8, 256)) return too_many_groups();
        f.tiles_w = (int)tw; f.tiles_x = (int)tx;
        const dim3 grid((unsigned)((tx ? owt_split_major_grid(f.tiles_x, 1) : 0) + owt_split_major_grid(f.tiles_w, 1)));
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, f); };
        if (bf16) { if (f.y) go(q8_few_bwd_kernel<bf16_t, true>); else go(q8_few_bwd_kernel<bf16_t, false>); }
        else if (f.y) go(q8_few_bwd_kernel<float, true>); else go(q8_few_bwd_kernel<float, false>);
        const hipError_t e = hipGetLastError();
        return e == hipSuccess ? OWT_OK : fail(OWT_ELAUNCH, "HIP launch failed: %s", hipGetErrorString(e));
    }

    Q8PrepParams q;
    memset(&q, 0, sizeof(q));
    q.dy = dy; q.y = (d->flags & OWT_RELU) ? y_or_null : nullptr;
    q.xs = xscale; q.ws = wscale; q.xq = xq; q.wq = wq;
    q.N = d->N; q.I = d->I; q.O = ol; q.xpitch = q8_pitch(d->I);
    q.want_dx = want_dx;
    q.alpha = alpha; q.beta = beta; q.db = dbias_or_null;
    q.strips = l.strips; q.strip_rows = l.strip_rows;
    q.colsum = (float *)(at + l.colsum); q.colmax = (float *)(at + l.colmax); q.rowmax = (float *)(at + l.rowmax);
    q.col_exp = (int *)(at + l.cexp); q.row_exp = (int *)(at + l.rexp);
    q.aw = (_Float16 *)(at + l.aw); q.ax = (_Float16 *)(at + l.ax); q.bw = (_Float16 *)(at + l.bw); q.bx = (_Float16 *)(at + l.bx);
    q.nk = l.nk; q.ok = l.ok;
    const long its = (d->I + 127) / 128, tz = (long)l.nk * l.ok, ts = (long)l.ok * l.strips, tx = its * l.nk, tw = want_dx ? its * l.ok : 0;
    const bool together = want_dx && l.pair;
    const Q8Plan pair{l.pair, 1, 0.f}, &plan_w = together ? pair : l.dw, &plan_x = together ? pair : l.dx;
    if (!groups_fit(ts + tx + tw, 256) || !groups_fit(tz, 256) || !product_fits(plan_w, ol, d->I) || (want_dx && !product_fits(plan_x, d->N, d->I)))
        return too_many_groups();
    q.tiles_s = (int)ts; q.tiles_x = (int)tx;
    auto prepare = [&](auto stat, auto halves) {
        hipLaunchKernelGGL(stat, dim3((unsigned)(ts + tx + tw)), dim3(256), 0, s, q);
        hipLaunchKernelGGL(halves, dim3((unsigned)tz), dim3(256), 0, s, q);
    };
    if (bf16) { if (want_dx) prepare(q8_stat_kernel<bf16_t>, q8_prep_kernel<bf16_t, true>); else prepare(q8_stat_kernel<bf16_t>, q8_prep_kernel<bf16_t, false>); }
    else { if (want_dx) prepare(q8_stat_kernel<float>, q8_prep_kernel<float, true>); else prepare(q8_stat_kernel<float>, q8_prep_kernel<float, false>); }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(OWT_ELAUNCH, "HIP launch failed: %s", hipGetErrorString(e));

    Q8GemmParams w, x;          // dw, dx
    memset(&w, 0, sizeof(w));
    w.a = (const unsigned char *)q.aw; w.b = (const unsigned char *)q.bw;
    w.lda = (size_t)l.nk * 256; w.ldb = (size_t)l.nk * 128;
    w.M = ol; w.N = d->I; w.ksteps = 2 * l.nk; w.planes = 2;
    w.out = dw; w.bf16 = 0;
    w.d = {q.col_exp, alpha, beta};
    x = w;
    x.a = (const unsigned char *)q.ax; x.b = (const unsigned char *)q.bx;
    x.lda = (size_t)l.ok * 256; x.ldb = (size_t)l.ok * 128;
    x.M = d->N; x.ksteps = 2 * l.ok;
    x.out = dx_partial_or_null; x.bf16 = bf16;
    x.d = {q.row_exp, 1.f, 0.f};
    if (together) {
        lay_tiles(w, pair);
        lay_tiles(x, pair);
        const dim3 grid((unsigned)(owt_split_major_grid(x.tiles, 1) + owt_split_major_grid(w.tiles, 1)));
        const bool dx_first = x.ksteps >= w.ksteps;
        const Q8GemmParams &p0 = dx_first ? x : w, &p1 = dx_first ? w : x;
        if (l.pair == 1) hipLaunchKernelGGL((q8gemm_pair_kernel<2, 2, 2, 2, 3, 1>), grid, dim3(256), 0, s, p0, p1);
        else hipLaunchKernelGGL((q8gemm_pair_kernel<2, 2, 1, 1, 4, 2>), grid, dim3(256), 0, s, p0, p1);
        e = hipGetLastError();
        return e == hipSuccess ? OWT_OK : fail(OWT_ELAUNCH, "HIP launch failed: %s", hipGetErrorString(e));
    }
    OWT_TRY(run_product<Q8Half>(w, l.dw, at + l.partial, s));
    return want_dx ? run_product<Q8Half>(x, l.dx, at + l.partial, s) : OWT_OK;
}

}  // extern "C"

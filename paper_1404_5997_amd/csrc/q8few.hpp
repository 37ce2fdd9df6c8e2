// Forward product of the dense shard in 8 bits where there are few results: tokens of a served model, shards of a small batch.
//
// The kernel of q8gemm.hpp has too few tiles for the chip there, or splits their sums over work-groups and adds them up in a second launch,
// which costs such a product as much as the product.  Here a work-group has 16 x 16 results (v_mfma_i32_16x16x64_i8) and its sixteen wavefronts take every sixteenth step of 128 bytes of the whole sum, straight from memory into
// registers; they add up through LDS.  Sums are of whole numbers, so their order does not matter.  Which operand values a lane holds is free as
// long as both operands agree: a lane takes 32 neighbouring bytes of a row, so that a row's four read a line of it.
// What bounds it: for a token the weights' bytes, each read once; for more rows what the tiles read again from the L2 caches.  (32 x 32
// results a work-group: half the reads, a quarter of the work-groups, 14.9 us for 64 rows of 4096 -> 4096 where this takes 19.2 and the
// tiles of q8gemm.hpp 11.4.)
#pragma once
#include "q8gemm.hpp"

namespace owt {

__global__ void __launch_bounds__(1024) q8_few_kernel(const Q8GemmParams p)
{
    constexpr int WAVES = 16, AHEAD = 6;            // steps of a wavefront on their way at a time: all of 12288 values
    __shared__ __attribute__((aligned(16))) int lds[WAVES * 256];
    int tile, split;
    if (!owt_split_major_wg(p.tiles, 1, tile, split)) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // tiles of the same columns of C, which read the same weights, follow each other
    const int tiles_m = (p.M + 15) / 16, tn = tile / tiles_m, m0 = (tile - tn * tiles_m) * 16, n0 = tn * 16;
    const unsigned char *a = p.a + (size_t)min(m0 + lane % 16, p.M - 1) * p.lda + lane / 16 * 32;
    const unsigned char *b = p.b + (size_t)min(n0 + lane % 16, p.N - 1) * p.ldb + lane / 16 * 32;
    // Four registers of a lane are columns 4 (lane / 16) + r of C, row lane % 16: the first wavefront adds up and writes.  What its results
    // need besides the sums is on its way from the start.
    const int m = m0 + lane % 16, c = n0 + 4 * (lane / 16);
    Q8Cols k = {};
    int row = 0;
    if (wave == 0) {
        k = q8_cols(p, c, q8_i32x16());
        row = q8_row(p, m, q8_i32x16());
    }
    q8_i32x4 acc = {0, 0, 0, 0};
    for (int s = wave; s < p.ksteps; s += WAVES * AHEAD) {
        q8_i32x4 fa[AHEAD][2], fb[AHEAD][2];
#pragma unroll
        for (int u = 0; u < AHEAD; u++) {
            if (s + u * WAVES >= p.ksteps) break;
            const size_t at = (size_t)(s + u * WAVES) * 128;
#pragma unroll
            for (int f = 0; f < 2; f++) {
                fa[u][f] = *(const q8_i32x4 *)(a + at + 16 * f);
                fb[u][f] = *(const q8_i32x4 *)(b + at + 16 * f);
            }
        }
#pragma unroll
        for (int u = 0; u < AHEAD; u++) {
            if (s + u * WAVES >= p.ksteps) break;
#pragma unroll
            for (int f = 0; f < 2; f++) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[u][f], fa[u][f], acc, 0, 0, 0);
        }
    }
    *(q8_i32x4 *)(lds + tid * 4) = acc;
    __syncthreads();
    if (wave != 0) return;
    q8_i32x4 sum = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < WAVES; w++) sum += *(const q8_i32x4 *)(lds + (w * 64 + lane) * 4);
    if (m >= p.M) return;
    int s[4];
#pragma unroll
    for (int t = 0; t < 4; t++) s[t] = sum[t];
    float v[4];
    q8_values(p, k, row, s, v);
    q8_how(p, false, [&](auto how, auto vec) __attribute__((always_inline)) {
        q8_put<decltype(how)::value, decltype(vec)::value>(p, (char *)p.out + (size_t)m * p.N * (p.bf16 ? 2 : 4), c, v);
    });
}

}  // namespace owt

// Forward product of the dense shard in 8 bits where there are few results: tokens of a served model, shards of a small batch.
//
// The kernel of q8gemm.hpp has too few tiles for the chip there, or splits their sums over work-groups and adds them up in a second launch,
// which costs such a product as much as the product.  Here a work-group has 16 x 16 results (v_mfma_i32_16x16x64_i8) and its sixteen wavefronts
// take every sixteenth step of 128 bytes of the whole sum and add up through LDS; sums are of whole numbers, so their order does not matter.
// A wavefront's rows go from memory straight into LDS of its own, 8 rows of a line an instruction, two steps ahead, and it waits for
// nobody.  (Straight into registers a lane takes the pieces of the row that the instruction wants it to have, so that four neighbouring
// lanes ask for four lines: 10.2 us for 128 rows of 9216 -> 512, this way 5.8.)
// What bounds it: for a token the weights' bytes, each read once; for more rows what the tiles read again from the L2 caches.  (32 x 32
// results a work-group: half the reads, a quarter of the work-groups, slower from one row to 64.)
#pragma once
#include "q8gemm.hpp"

namespace owt {

__global__ void __launch_bounds__(1024) q8_few_kernel(const Q8GemmParams p)
{
    constexpr int WAVES = 16, STAGE = 32 * 128;     // 16 rows of either operand
    __shared__ __attribute__((aligned(16))) unsigned char lds[WAVES * 2 * STAGE];
    int tile, split;
    if (!owt_split_major_wg(p.tiles, 1, tile, split)) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // tiles of the same columns of C, which read the same weights, follow each other
    const int tiles_m = (p.M + 15) / 16, tn = tile / tiles_m, m0 = (tile - tn * tiles_m) * 16, n0 = tn * 16;
    // Four registers of a lane are columns 4 (lane / 16) + r of C, row lane % 16: the first wavefront adds up and writes.  What its results
    // need besides the sums is on its way from the start.
    const int m = m0 + lane % 16, c = n0 + 4 * (lane / 16);
    Q8Cols k = {};
    int row = 0;
    if (wave == 0) {
        k = q8_cols(p, c, q8_i32x16());
        row = q8_row(p, m, q8_i32x16());
    }
    // 16-byte piece q of row r lies in slot q ^ ((r >> 1) & 7), as in q8gemm.hpp
    unsigned asrc[2], bsrc[2];
#pragma unroll
    for (int i = 0; i < 2; i++) {
        const int r = 8 * i + (lane >> 3), piece = (lane & 7) ^ ((r >> 1) & 7);
        asrc[i] = (unsigned)min(r, p.M - 1 - m0) * (unsigned)p.lda + 16 * piece;
        bsrc[i] = (unsigned)min(r, p.N - 1 - n0) * (unsigned)p.ldb + 16 * piece;
    }
    const unsigned char *ag = q8_uniform(p.a + (size_t)m0 * p.lda), *bg = q8_uniform(p.b + (size_t)n0 * p.ldb);
    unsigned char *mine = lds + wave * (2 * STAGE);
    const unsigned to = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char *)mine;
    auto load = [&](int i) __attribute__((always_inline)) {
        const size_t at = (size_t)(wave + WAVES * i) * 128;
        const unsigned char *ap = q8_uniform(ag + at), *bp = q8_uniform(bg + at);
        const unsigned dst = __builtin_amdgcn_readfirstlane(to + (i & 1) * STAGE);
        q8_load_lds(asrc[0], ap, dst);
        q8_load_lds(asrc[1], ap, dst + 1 * 1024);
        q8_load_lds(bsrc[0], bp, dst + 2 * 1024);
        q8_load_lds(bsrc[1], bp, dst + 3 * 1024);
    };
    const int steps = (p.ksteps - wave + WAVES - 1) / WAVES;            // of this wavefront
    const int fr = lane % 16 * 128, sw = (lane % 16 >> 1) & 7, part = lane / 16;
    q8_i32x4 acc = {0, 0, 0, 0};
    if (steps > 0) load(0);
    if (steps > 1) load(1);
    for (int i = 0; i < steps; i++) {
        if (i + 1 < steps) __builtin_amdgcn_s_waitcnt(0x0F74);          // vmcnt(4): this step has landed, the next one may be on its way
        else __builtin_amdgcn_s_waitcnt(0x0F70);
        asm volatile("" ::: "memory");
        const unsigned char *at = mine + (i & 1) * STAGE + fr;
        q8_i32x4 fa[2], fb[2];
#pragma unroll
        for (int f = 0; f < 2; f++) {
            fa[f] = *(const q8_i32x4 *)(at + 16 * ((4 * f + part) ^ sw));
            fb[f] = *(const q8_i32x4 *)(at + 2048 + 16 * ((4 * f + part) ^ sw));
        }
        __builtin_amdgcn_s_waitcnt(0xC07F);                             // lgkmcnt(0): the fragments are in registers, their place is free
        asm volatile("" ::: "memory");
        if (i + 2 < steps) load(i + 2);
#pragma unroll
        for (int f = 0; f < 2; f++) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[f], fa[f], acc, 0, 0, 0);
    }
    __syncthreads();                                // (the sums come where the operands were)
    *(q8_i32x4 *)(lds + tid * 16) = acc;
    __syncthreads();
    if (wave != 0) return;
    q8_i32x4 sum = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < WAVES; w++) sum += *(const q8_i32x4 *)(lds + (w * 64 + lane) * 16);
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

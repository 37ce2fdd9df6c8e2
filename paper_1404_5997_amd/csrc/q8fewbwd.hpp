// Backward pass of the dense shard in 8 bits where there is little of it: one launch from dy and the 8-bit rows to dx, dw and the bias gradient.
//
// The products of q8gemm.hpp want operands with consecutive k and a power of two for each row of a result, which take two launches.
// Here both operands are read as they lie and put in order in registers.  dz times its scale is split in bf16 parts by truncation: three of
// 8 bits are all 24 of an fp32 value, and bf16 has fp32's exponents, so that nothing needs to be known of the other values.  Whole numbers of 8 bits
// are exact in bf16.  A wavefront has 32 rows x 128 columns of a result (v_mfma_f32_32x32x16_bf16): of each of a step's sixteen rows of whole numbers a lane reads the four of columns 4 (lane % 32) .., one
// column of each of its four tiles, so that a lane's results of a row are four neighbours.  The four wavefronts of a work-group take every
// fourth step and add up in LDS, in a fixed order.
//
// What bounds it: the splitting and widening, about 150 vector instructions beside a step's 12 matrix instructions, and a work-group's beginning
// and end, where dw's sums are of few steps.  128 rows of 4096 -> 512 in fp32 12 us (22 with the preparation), 9216 -> 512 19 (27).
// Three work-groups a CU: two with steps read two ahead 22, and 20.6 one ahead; wavefronts with tiles and whole sums of their own 23.3.
#pragma once
#include "q8gemm.hpp"

namespace owt {

struct Q8FewBwdParams {
    const void *dy, *y;                 // y: ReLU mask
    const float *xs, *ws;
    const signed char *xq, *wq;
    int N, I, O;
    size_t pitch;                       // of xq and wq
    float alpha, beta;
    void *dx;
    float *dw, *db;                     // db may be null
    int tiles_x, tiles_w;               // 32 x 128 results each
};

typedef __bf16 q8_bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t q8_u32x4 __attribute__((ext_vector_type(4)));
constexpr int kQ8FewBwdLds = 2 * 16 * 64 * 16 + 4 * 32 * 4;

// Rows mt * 32 .. and columns it * 128 .. of dx (DX) or dw.
template <class T, bool DX, bool MASK>
__device__ __forceinline__ void q8_few_bwd(const Q8FewBwdParams &p, int mt, int it, unsigned char *lds)
{
    constexpr int PARTS = 3, WAVES = 4;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, l = lane & 31;
    const int M = DX ? p.N : p.O, K = DX ? p.O : p.N;
    const signed char *q = (DX ? p.wq : p.xq) + it * 128;
    const float *scale = DX ? p.ws : p.xs;
    const unsigned m = (unsigned)min(mt * 32 + l, M - 1);
    // A step's values of both operands and its scales through descriptors that end behind them: what lies past K reads as zero, and a lane's
    // offsets of eight loads are the same for all steps.
    constexpr unsigned E = sizeof(T) == 2 ? 2 : 4;
    unsigned aoff[8], boff[8];
#pragma unroll
    for (int j = 0; j < 8; j++) {
        aoff[j] = E * (DX ? (m - (unsigned)mt * 32) * (unsigned)p.O + 8 * half + j : (unsigned)(8 * half + j) * (unsigned)p.O + m);
        boff[j] = (unsigned)(8 * half + j) * (unsigned)p.pitch + 4 * l;
    }
    struct Raw { float a[8], y[8], s[8]; unsigned b[8]; };
    auto load = [&](auto near, Raw &r, int step) __attribute__((always_inline)) {
        const int k0 = step * 16;
        const unsigned rows = min(16, K - k0);
        const size_t at = DX ? (size_t)mt * 32 * p.O + k0 : (size_t)k0 * p.O;
        const unsigned bytes = E * (DX ? (unsigned)min(32, M - mt * 32) * (unsigned)p.O - k0 : rows * (unsigned)p.O);
        const __amdgpu_buffer_rsrc_t dy = owt_make_rsrc((const char *)p.dy + at * E, bytes), y = owt_make_rsrc((const char *)p.y + at * E, bytes);
        const __amdgpu_buffer_rsrc_t b = owt_make_rsrc(q + (size_t)k0 * p.pitch, rows * (unsigned)p.pitch - it * 128), sc = owt_make_rsrc(scale + k0, rows * 4);
        auto value = [&](__amdgpu_buffer_rsrc_t of, unsigned o) {
            if (E == 4) return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(of, (int)o, 0, 0));
            return __uint_as_float((uint32_t)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(of, (int)o, 0, 0) << 16);
        };
#pragma unroll
        for (int j = 0; j < 8; j++) r.b[j] = __builtin_amdgcn_raw_buffer_load_b32(b, (int)boff[j], 0, 0);
        if (decltype(near)::value) {                // dx, but for its last step: eight neighbours of a row, which begin anywhere
            constexpr int V = Piece<T>::V;
#pragma unroll
            for (int i = 0; i < 8; i += V) {
                float v[V], w[V];
                Piece<T>::load((const T *)p.dy + at + aoff[0] / E + i, v);
                if (MASK) Piece<T>::load((const T *)p.y + at + aoff[0] / E + i, w);
#pragma unroll
                for (int t = 0; t < V; t++) {
                    r.a[i + t] = v[t];
                    if (MASK) r.y[i + t] = w[t];
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; j++) {
                r.a[j] = value(dy, aoff[j]);
                if (MASK) r.y[j] = value(y, aoff[j]);
            }
        }
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
            const float4 v = buffer_load4(sc, 4 * (unsigned)(8 * half + i));
            r.s[i] = v.x; r.s[i + 1] = v.y; r.s[i + 2] = v.z; r.s[i + 3] = v.w;
        }
    };
    q8_f32x16 acc[4] = {};
    float bias = 0.f;
    auto multiply = [&](const Raw &r, int step) __attribute__((always_inline)) {
        uint32_t part[PARTS][8];
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; j++) {
            const float dz = !MASK || r.y[j] > 0.f ? r.a[j] : 0.f;
            v[j] = dz * r.s[j];
            if (!DX) bias += dz;
        }
        if (DX && step * 16 + 16 > K)                                           // (behind a row's end is the next row)
#pragma unroll
            for (int j = 0; j < 8; j++) v[j] = step * 16 + 8 * half + j < K ? v[j] : 0.f;
#pragma unroll
        for (int j = 0; j < 8; j++) {
#pragma unroll
            for (int i = 0; i < PARTS; i++) {
                part[i][j] = __float_as_uint(v[j]);
                const float rest = v[j] - __uint_as_float(part[i][j] & 0xffff0000u);
                v[j] = i || fabsf(v[j]) < __uint_as_float(0x7f800000u) ? rest : 0.f;    // what is not finite is its first part
            }
        }
        q8_bf16x8 a[PARTS];
#pragma unroll
        for (int i = 0; i < PARTS; i++) {
            q8_u32x4 w;
#pragma unroll
            for (int j = 0; j < 4; j++) w[j] = __builtin_amdgcn_perm(part[i][2 * j + 1], part[i][2 * j], 0x07060302u);
            a[i] = __builtin_bit_cast(q8_bf16x8, w);
        }
#pragma unroll
        for (int t = 0; t < 4; t++) {
            q8_u32x4 w;
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const float b0 = (float)(int)(signed char)(r.b[2 * j] >> (8 * t)), b1 = (float)(int)(signed char)(r.b[2 * j + 1] >> (8 * t));
                w[j] = __builtin_amdgcn_perm(__float_as_uint(b1), __float_as_uint(b0), 0x07060302u);
            }
            const q8_bf16x8 b = __builtin_bit_cast(q8_bf16x8, w);
#pragma unroll
            for (int i = PARTS - 1; i >= 0; i--) acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i], b, acc[t], 0, 0, 0);
        }
    };
    const std::integral_constant<bool, DX> near;
    const int steps = (DX ? K : K + 15) / 16, last = steps - 1;         // dx's last step by itself, if it is short
    if (wave < steps) {
        Raw r0, r1;
        load(near, r0, wave);
        for (int s = wave; s < steps; s += 2 * WAVES) {
            load(near, r1, min(s + WAVES, last));
            multiply(r0, s);
            load(near, r0, min(s + 2 * WAVES, last));
            if (s + WAVES < steps) multiply(r1, s + WAVES);
        }
    }
    if (DX && K % 16 && wave == steps % WAVES) {
        Raw r;
        load(std::integral_constant<bool, false>{}, r, steps);
        multiply(r, steps);
    }
    // Register r of a lane is row 8 (r / 4) + 4 half + r % 4 of its column.
    const int c = it * 128 + 4 * l;
    auto write = [&](auto vec, int row, float (&v)[4]) __attribute__((always_inline)) {
        constexpr bool VEC = decltype(vec)::value;
        if (row >= M) return;
        if (DX) q8_store4<VEC>((T *)p.dx + (size_t)row * p.I, c, p.I, v);
        else {
            float old[4] = {}, *to = p.dw + (size_t)row * p.I;
            if (p.beta != 0.f) q8_load4<VEC>(to, c, p.I, old);
#pragma unroll
            for (int t = 0; t < 4; t++) v[t] = p.alpha * v[t] + (p.beta != 0.f ? p.beta * old[t] : 0.f);
            q8_store4<VEC>(to, c, p.I, v);
        }
    };
    auto write_bias = [&](float sum) __attribute__((always_inline)) {
        if (lane >= 32 || mt * 32 + l >= M) return;
        float *to = p.db + mt * 32 + l;
        *to = p.alpha * sum + (p.beta != 0.f ? p.beta * *to : 0.f);
    };
    const bool with_bias = !DX && it == 0 && p.db;
    if (with_bias) bias += __shfl_xor(bias, 32, 64);
    // Wavefronts 2 and 3 hand theirs to 0 and 1, these both sums to all, which write a quarter of the rows each.
    float4 *sums = (float4 *)lds;
    float *biases = (float *)(lds + 2 * 16 * 64 * 16);
    if (with_bias && lane < 32) biases[wave * 32 + lane] = bias;
    if (wave >= 2) {
#pragma unroll
        for (int r = 0; r < 16; r++) sums[((wave - 2) * 16 + r) * 64 + lane] = make_float4(acc[0][r], acc[1][r], acc[2][r], acc[3][r]);
    }
    __syncthreads();
    if (wave < 2) {
#pragma unroll
        for (int r = 0; r < 16; r++) {
            float4 *at = sums + (wave * 16 + r) * 64 + lane;
            const float4 o = *at;
            *at = make_float4(acc[0][r] + o.x, acc[1][r] + o.y, acc[2][r] + o.z, acc[3][r] + o.w);
        }
    }
    __syncthreads();
    if (with_bias && wave == 0) write_bias((biases[l] + biases[32 + l]) + (biases[64 + l] + biases[96 + l]));
    auto finish = [&](auto vec) __attribute__((always_inline)) {
#pragma unroll
        for (int r = 0; r < 4; r++) {
            const float4 s = sums[(wave * 4 + r) * 64 + lane], u = sums[(16 + wave * 4 + r) * 64 + lane];
            float v[4] = {s.x + u.x, s.y + u.y, s.z + u.z, s.w + u.w};
            write(vec, mt * 32 + 8 * wave + 4 * half + r, v);
        }
    };
    if ((p.I & 3) == 0) finish(std::integral_constant<bool, true>{});
    else finish(std::integral_constant<bool, false>{});
}

template <class T, bool MASK> __global__ void __launch_bounds__(256, 3) q8_few_bwd_kernel(const Q8FewBwdParams p)
{
    __shared__ __attribute__((aligned(16))) unsigned char lds[kQ8FewBwdLds];
    // (the numbering of owt_split_major_wg, within a product's work-groups: their number is a multiple of 8; tiles of the same columns
    // follow each other)
    const int first = p.tiles_x ? owt_split_major_grid(p.tiles_x, 1) : 0;
    auto run = [&](auto dx, int l, int tiles, int rows) __attribute__((always_inline)) {
        constexpr bool DX = decltype(dx)::value;
        const int xcd = l & 7, jx = l >> 3, each = tiles >> 3, more = tiles & 7;
        if (jx >= each + (xcd < more ? 1 : 0)) return;
        const int tile = xcd * each + min(xcd, more) + jx, tiles_m = (rows + 31) / 32, it = tile / tiles_m;
        q8_few_bwd<T, DX, MASK>(p, tile - it * tiles_m, it, lds);
    };
    if ((int)blockIdx.x < first) run(std::integral_constant<bool, true>{}, (int)blockIdx.x, p.tiles_x, p.N);
    else run(std::integral_constant<bool, false>{}, (int)blockIdx.x - first, p.tiles_w, p.O);
}

}  // namespace owt

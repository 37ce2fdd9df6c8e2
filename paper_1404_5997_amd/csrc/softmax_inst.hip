// Instantiations of smgemm.hpp: -DOWT_INST_HALF=0 (bf16) or 1 (f16), -DOWT_INST_OUT=0 (outputs as statistics or dz), 1 (stored sums) or
// 2 (bf16 dx of long sums in 256 x 256 tiles).
#include "softmax.hpp"

namespace owt {

#if OWT_INST_HALF
typedef SmHalf Op;
#else
typedef SmBf16 Op;
#endif

template <bool TA, bool TB, class S, int END> static hipError_t go(const SmParams &p, hipStream_t s)
{
    hipLaunchKernelGGL((sm_kernel<Op, TA, TB, S, END>), dim3((unsigned)(owt_split_major_grid(p.tiles, p.splits) + (p.copy.out_rows ? kSmCopyGroups : 0))), dim3(64 * S::NW), 0,
                       s, p);
    return hipGetLastError();
}
#if OWT_INST_OUT == 2
hipError_t owt_launch_softmax_bf16_dx(const SmParams &p, hipStream_t s) { return go<false, true, SmBigPair, SM_OUT>(p, s); }
#else

template <bool TA, bool TB, int END> static hipError_t tiled(int tile, const SmParams &p, hipStream_t s)
{
    if (tile == SM_BIG) {
        const bool ring = p.steps_per_split > kSmRing * p.products;
#if OWT_INST_HALF
        if (ring) return go<TA, TB, SmBigThree, END>(p, s);
#else
        if constexpr (TB)
            if (ring && p.products == SM_PAIR) {
                if constexpr (TA) return go<TA, TB, SmBigPair, END>(p, s);
                else return owt_launch_softmax_bf16_dx(p, s);
            }
#endif
        return go<TA, TB, SmBig, END>(p, s);
    }
    if (tile == SM_MID) return go<TA, TB, SmMid, END>(p, s);
    if (tile == SM_TWO) return go<TA, TB, SmPair, END>(p, s);
    if (tile == SM_SMALL) return go<TA, TB, SmSmall, END>(p, s);
    return hipErrorInvalidValue;
}

#if OWT_INST_HALF && OWT_INST_OUT
#define OWT_INST_NAME owt_launch_softmax_half_out
#elif OWT_INST_HALF
#define OWT_INST_NAME owt_launch_softmax_half_ends
#elif OWT_INST_OUT
#define OWT_INST_NAME owt_launch_softmax_bf16_out
#else
#define OWT_INST_NAME owt_launch_softmax_bf16_ends
#endif

hipError_t OWT_INST_NAME(int product, int tile, const SmParams &p, hipStream_t s)
{
#if OWT_INST_OUT
    if (product == SM_PRODUCT_Z) return tiled<false, false, SM_OUT>(tile, p, s);
    if (product == SM_PRODUCT_DX) return tiled<false, true, SM_OUT>(tile, p, s);
    if (product == SM_PRODUCT_DW) return tiled<true, true, SM_OUT>(tile, p, s);
#else
    if (product == SM_PRODUCT_TOP) return tiled<false, false, SM_TOP>(tile, p, s);
    if (product == SM_PRODUCT_DZ) return tiled<false, false, SM_DZ>(tile, p, s);
#endif
    return hipErrorInvalidValue;
}

#if OWT_INST_OUT
#if OWT_INST_HALF
hipError_t owt_launch_softmax_half_pair(int tile, const SmParams &x, const SmParams &w, bool x_first, hipStream_t s)
#else
hipError_t owt_launch_softmax_bf16_pair(int tile, const SmParams &x, const SmParams &w, bool x_first, hipStream_t s)
#endif
{
    const dim3 grid((unsigned)(owt_split_major_grid(x.tiles, x.splits) + owt_split_major_grid(w.tiles, 1)));
    if (tile == SM_MID) hipLaunchKernelGGL((sm_pair_kernel<Op, SmMid>), grid, dim3(256), 0, s, x, w, x_first);
    else if (tile == SM_SMALL) hipLaunchKernelGGL((sm_pair_kernel<Op, SmSmall>), grid, dim3(256), 0, s, x, w, x_first);
    else return hipErrorInvalidValue;
    return hipGetLastError();
}
#endif
#endif

}  // namespace owt

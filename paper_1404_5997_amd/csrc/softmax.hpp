// Host side of softmax cross-entropy: the tiles of its products and where they are launched (softmax_inst.hip).
#pragma once
#include "owt_host.hpp"
#include "smgemm.hpp"

namespace owt {

// 256 x 256; 128 x 128 with three stages, one work-group a CU, and with two stages, two a CU; 64 x 64.  owt_test_force_variant: 120.. name these.
// The pair of 128 x 128 covers one another's beginnings and ends where there are enough of them, the single one has more on its way where there are few (us, one and the
// other: outputs of 777 rows 1536 -> 20000, 1104 tiles, 86 and 69, their dx, 88 tiles, 161 and 210).  256 x 128 and 32 x 256 were never the fastest.
typedef SmShape<2, 2, 4, 4, 2, 1> SmBig;
typedef SmShape<2, 2, 4, 4, 5, 1, SM_PAIR> SmBigPair;        // (256 x 256, too: where more than kSmRing steps of memory have several products)
typedef SmShape<2, 2, 4, 4, 5, 1, SM_THREE> SmBigThree;
constexpr int kSmRing = 4;
typedef SmShape<2, 2, 2, 2, 3, 1> SmMid;
typedef SmShape<2, 2, 2, 2, 2, 2> SmPair;
typedef SmShape<2, 2, 1, 1, 4, 2> SmSmall;
enum { SM_BIG, SM_MID, SM_TWO, SM_SMALL, SM_TILES };
constexpr int kSmFirstTile = 120;

enum { SM_PRODUCT_TOP, SM_PRODUCT_DZ, SM_PRODUCT_Z, SM_PRODUCT_DX, SM_PRODUCT_DW };
// half: fp32 values as two f16 ones; else bf16
hipError_t owt_launch_softmax_bf16_ends(int product, int tile, const SmParams &, hipStream_t);      // TOP, DZ
hipError_t owt_launch_softmax_bf16_out(int product, int tile, const SmParams &, hipStream_t);       // Z, DX, DW
hipError_t owt_launch_softmax_bf16_dx(const SmParams &, hipStream_t);       // DX, long sums of two products in 256 x 256 tiles
hipError_t owt_launch_softmax_half_ends(int product, int tile, const SmParams &, hipStream_t);
hipError_t owt_launch_softmax_half_out(int product, int tile, const SmParams &, hipStream_t);
// dx and dw together: 128 x 128 or 64 x 64
hipError_t owt_launch_softmax_bf16_pair(int tile, const SmParams &x, const SmParams &w, bool x_first, hipStream_t);
hipError_t owt_launch_softmax_half_pair(int tile, const SmParams &x, const SmParams &w, bool x_first, hipStream_t);

}  // namespace owt

// Host side of softmax cross-entropy: the tiles of its products and where they are launched (softmax_inst.hip).
#pragma once
#include "owt_host.hpp"
#include "smgemm.hpp"

namespace owt {

// 256 x 256, 128 x 128, 64 x 64, and 32 x 256 for few rows (not of dw, whose rows are classes).  owt_test_force_variant: 120.. name these.
typedef SmShape<2, 2, 4, 4, 2, 1> SmBig;
typedef SmShape<2, 2, 2, 2, 3, 1> SmMid;
typedef SmShape<2, 2, 1, 1, 4, 2> SmSmall;
typedef SmShape<1, 4, 1, 2, 4, 1> SmFew;
enum { SM_BIG, SM_MID, SM_SMALL, SM_FEW, SM_TILES };
constexpr int kSmFirstTile = 120;

enum { SM_PRODUCT_TOP, SM_PRODUCT_DZ, SM_PRODUCT_Z, SM_PRODUCT_DX, SM_PRODUCT_DW };
// half: fp32 values as two f16 ones; else bf16
hipError_t owt_launch_softmax_bf16_ends(int product, int tile, const SmParams &, hipStream_t);      // TOP, DZ
hipError_t owt_launch_softmax_bf16_out(int product, int tile, const SmParams &, hipStream_t);       // Z, DX, DW
hipError_t owt_launch_softmax_half_ends(int product, int tile, const SmParams &, hipStream_t);
hipError_t owt_launch_softmax_half_out(int product, int tile, const SmParams &, hipStream_t);

}  // namespace owt

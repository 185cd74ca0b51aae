// The product in 8-bit integers, tile by tile: the kernels of each shape of tiles.
#include "i8_tiles.hpp"

namespace spqt {
namespace i8 {

void launch_tiles_of(const Plan &plan, const Product &p, bool gated, void *workspace, hipStream_t stream) {
    switch (plan.shape) {
        case 0: launch_tiles<256, 256, 2, 4, 2, 3>(p, gated, plan.parts, workspace, stream); break;
        case 1: launch_tiles<128, 256, 2, 4, 4, 3>(p, gated, plan.parts, workspace, stream); break;
        case 2: launch_tiles<128, 128, 2, 2, 4, 5>(p, gated, plan.parts, workspace, stream); break;
        default: launch_tiles<64, 128, 2, 2, 6, 7>(p, gated, plan.parts, workspace, stream); break;
    }
}

}  // namespace i8
}  // namespace spqt

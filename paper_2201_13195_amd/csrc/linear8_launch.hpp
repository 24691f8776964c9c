// All kernels of one format, kind of scales and type of Y.
#pragma once
#include "linear8_few.hpp"
#include "linear8_plan.hpp"
#include "linear8_tile.hpp"

namespace rmm {

template <int F8, int SCALE, typename T>
void launch_linear8_by(int kernel, const Linear8Args &g, hipStream_t stream) {
    switch (kernel) {
        case LINEAR8_FEW_16x16: return launch_few<T, F8, SCALE, 1, 1, 8>(g, stream);
        case LINEAR8_FEW_16x32: return launch_few<T, F8, SCALE, 1, 2, 8>(g, stream);
        case LINEAR8_FEW_32x32: return launch_few<T, F8, SCALE, 2, 2, 8>(g, stream);
        case LINEAR8_FEW_64x32: return launch_few<T, F8, SCALE, 4, 2, 8>(g, stream);
        case LINEAR8_MANY_16x64: return launch_few<T, F8, SCALE, 1, 4, 4>(g, stream);
        case LINEAR8_MANY_32x32: return launch_few<T, F8, SCALE, 2, 2, 4>(g, stream);
        case LINEAR8_MANY_64x32: return launch_few<T, F8, SCALE, 4, 2, 4>(g, stream);
        case LINEAR8_TILE_64x128: return launch_tile<Half8, F8, SCALE, T>(g, stream);
        case LINEAR8_TILE_128_SPLIT: return launch_tile<Split8, F8, SCALE, T>(g, stream);
        case LINEAR8_TILE_256:
            if constexpr (sizeof(T) == 2) return launch_tile<Large8, F8, SCALE, T>(g, stream);
            [[fallthrough]];
        default: return launch_tile<Mid8, F8, SCALE, T>(g, stream);
    }
}

}  // namespace rmm

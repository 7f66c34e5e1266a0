// 128 x 256 tiles of the scaled product, B stored [N x K].
#include "scaled_tile.hpp"
namespace coda {
template <>
hipError_t launch_scaled_128<true>(int mode, bool q8, const GemmParams &g, const Q8Params &q, const ScaledParams &p, hipStream_t s)
{
    return launch_program<ScaledCfg<128, 256, 2, 4, 3>, true>(mode, q8, g, q, p, s);
}
}  // namespace coda

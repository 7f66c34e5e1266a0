// 256 x 256 tiles of the scaled product, B stored [K x N].
#include "scaled_tile.hpp"
namespace coda {
template <>
hipError_t launch_scaled_256<false>(int mode, bool q8, const GemmParams &g, const Q8Params &q, const ScaledParams &p, hipStream_t s)
{
    return launch_large_program<false>(mode, q8, g, q, p, s);
}
}  // namespace coda

// linear8_tiles.h's kernels for tiles of 64 channels
#include "linear8_tiles.h"

namespace gpusq {
void launch_linear8_tiles2(const Linear8Args& a, const Tokens8Plan& plan, hipStream_t s) { launch_linear8_tiles_of<2>(a, plan, s); }
}  // namespace gpusq

// linear8_tiles.h's kernels for tiles of 128 channels
#include "linear8_tiles.h"

namespace gpusq {
void launch_linear8_tiles4(const Linear8Args& a, const Tokens8Plan& plan, hipStream_t s) { launch_linear8_tiles_of<4>(a, plan, s); }
}  // namespace gpusq

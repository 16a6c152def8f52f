// linear8_tiles.h's kernels for tiles of 256 channels
#include "linear8_tiles.h"

namespace gpusq {
void launch_linear8_tiles8(const Linear8Args& a, const Tokens8Plan& plan, hipStream_t s) { launch_linear8_tiles_of<8>(a, plan, s); }
}  // namespace gpusq

// What launches decide on the host by plain arithmetic, apart from CUDA so that it
// can be checked without a GPU.
#pragma once
#include <cstdint>

namespace ra {

// Are the (segment, sample) pairs of a row call few, and more than one? Then its
// CTAs' shares may end with them (residual_norm.cu, piece_share: a ballot of the
// samples of a segment, so no more than 32).
constexpr int FEW_PIECES = 12;
constexpr bool few_pieces(int64_t samples, int segs) {
  return samples * segs > 1 && samples * segs <= FEW_PIECES;
}

}  // namespace ra

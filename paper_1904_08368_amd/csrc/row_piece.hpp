// Where the lanes of a row's loads read: chunks of 128 elements of 16 bits, 16 lanes to a row, eight elements (16 bytes) to a lane.
#pragma once
#include "fastdiv.hpp"

namespace relay {

// The first element of lane `col`'s piece of a chunk; behind the end of a row of k elements (a multiple of 8) its last piece, which is there whatever k is.
RELAY_HD inline int row_piece(int chunk, int col, int k) {
  const int at = chunk * 128 + col * 8;
  return at < k ? at : k - 8;
}

}  // namespace relay

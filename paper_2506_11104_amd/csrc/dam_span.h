// Which rows of a cache a call takes from a sequence, and which blocks of rows they fall into. Plain C++, constexpr: callable on
// the device and on the host. Row numbers go up to a cache's capacity; a block behind the last one of a call may start beyond
// 2^31, so that blocks are told apart before they are multiplied out.
#pragma once
#include <stdint.h>

namespace dam {

struct Span {
  int start, count;
};

// (start and count are device data that the host cannot check: a start outside the cache has no rows, and none are taken beyond
// the cache's end or the caller's n_rows.)
constexpr Span span_of(int start, int count, int n_rows, int capacity) {
  if (start < 0 || start >= capacity) return {0, 0};
  const int given = count < 0 ? 0 : count < n_rows ? count : n_rows, room = capacity - start;
  return {start, given < room ? given : room};
}

// The nth of the blocks of `block` rows that hold a row of the span, or -1 where it has fewer.
constexpr int nth_block(const Span &span, int block, int nth) {
  if (span.count < 1 || nth > (span.start % block + (span.count - 1)) / block) return -1;
  return span.start / block + nth;
}

// Blocks that n_rows >= 1 rows can fall into, wherever they start.
constexpr int64_t most_blocks(int n_rows, int capacity, int block) {
  const int64_t from_a_last_row = ((int64_t)n_rows + block - 2) / block + 1, all = ((int64_t)capacity + block - 1) / block;
  return from_a_last_row < all ? from_a_last_row : all;
}

}  // namespace dam

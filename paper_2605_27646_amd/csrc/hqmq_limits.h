// Arithmetic on callers' limits, in plain C++: constant expressions, which a compiler refuses where they overflow.
#pragma once

namespace hqmq {

// How many tokens a query head sees whose limit is `visible`, any 32-bit number: negative ones mean none.  What is computed from it
// (the end of the rows to read, rows left of a tile) is then a difference of numbers that are not negative.
constexpr int seen_tokens(int visible) { return visible > 0 ? visible : 0; }

// Rows of a tile of `most` that starts at `first`, of those before `end`; none, where that is not positive.
constexpr int tile_rows(int end, int first, int most) { return end - first < most ? end - first : most; }

}  // namespace hqmq

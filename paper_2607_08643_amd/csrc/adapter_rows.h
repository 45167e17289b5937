// Which row of an adapter's A is read for a rank: plain C++, the same on the
// host, where every rank can be tried, and in the kernels.
#pragma once
#include <cstdint>

namespace bsq {

// Rank blocks of 16 of a projection: one, two, four or eight.
constexpr int rank_blocks(int rank) { return rank <= 16 ? 1 : (rank <= 32 ? 2 : (rank <= 64 ? 4 : 8)); }

// The row of A [n][rank][d_in] that stands for rank r (0 .. 16 rank_blocks - 1)
// of adapter `ad`: its own, or, past the adapter's own rank `own` (0 .. rank), the
// adapter's first, which the callers mask or drop. Rows are loaded without a
// condition and the blocks reach past the rank, so every r has to give a row of
// this very adapter.
constexpr int64_t adapter_row(int64_t ad, int rank, int r, int own) { return ad * rank + (r < own ? r : 0); }

}  // namespace bsq

// Into which pieces the pages of trees' attention are cut (plain C++: the host sizes a launch, and the kernels cut, by the same numbers).
//
// What has to be done is units: a sequence's pages (those that its nodes see), a tile of its rows, a key head.  `work` is the pages of all units.  Units of more than `per` pages are cut into pieces of about
// as many.  The card has `places` workgroups at once.  If they are to be done in k turns, pieces have at least work / (k places - units) pages (cutting makes at most work / per pieces more than there are
// units), and cost k (per + kPieceCost) pages' time, kPieceCost for what a workgroup does beside its pages; the best k up to 4 is taken.  Calls with one turn alone | two alone | the rule, four sequences of up to 60 nodes
// and 50 000 to 65 011 tokens 240 | 250 | 241 us, 48 sequences of up to 26 nodes and 4000 tokens, two layers, 111.3 | 110.7 | 111.4.
//
// But no piece is longer than twice the average of a place.  Where units nearly fill the turns, what is left of them would have long units stay whole (with one place left all the work goes to one piece), and where units
// are more than that nothing else cuts them.  One sequence of 60 000 tokens, the others of 500, 8 nodes, 8 heads of 128 channels, 250 | 255 | 257 sequences: 134 | 133 | 142 us; by the turns alone 272 | 479 | 140.
#pragma once
#include <cstdint>

namespace spg {

constexpr int kMostEven = 512;     // sequences that a workgroup looks through
constexpr int kLeastPages = 4, kPieceCost = 8, kMostTurns = 4;

// rcp: 1 / x in 32 bits.
template <typename F>
constexpr int pages_of_piece(float work, float units, int places, F rcp) {
  float best = __builtin_inff(), per = __builtin_inff();
#pragma unroll
  for (int k = 1; k <= kMostTurns; ++k) {
    const float room = (float)(k * places) - units;
    // (in 24 digits the sums and the quotient are off by less than 2^-12 of them: what is added keeps the number of pieces within k places)
    const float pages = __builtin_ceilf(work * (1.0f + 0x1p-11f) * rcp(room)), cost = (float)k * (__builtin_fmaxf(pages, (float)kLeastPages) + kPieceCost);
    if (room > 0.0f && cost < best) { best = cost; per = pages; }
  }
  return (int)__builtin_fminf(__builtin_fmaxf(__builtin_fminf(per, __builtin_ceilf(2.0f * work * rcp((float)places))), (float)kLeastPages), 1e9f);
}

// Bounds that the host has, which knows how much work and how many units there are at most.  Pieces: with the k turns at most k places; with pieces of twice the average half a place more than the units for each; and never
// more than the units and one for every kLeastPages pages.
constexpr int64_t most_pieces(int64_t work, int64_t units, int places) {
  const int64_t turns = (int64_t)kMostTurns * places, some = units + places, most = turns > some ? turns : some, each = units + work / kLeastPages;
  return most < each ? most : each;
}
// Cells are for pieces of cut units alone: the k turns, or (a unit that is cut has at most two pieces for every `per` pages) a place each; and at most two for every kLeastPages pages.
constexpr int64_t most_cells(int64_t work, int places) {
  const int64_t turns = (int64_t)kMostTurns * places, each = 2 * (work / kLeastPages);
  return turns < each ? turns : each;
}

constexpr int kLongest = 1 << 25;   // pages of a sequence: lengths are below 2^31

// More sequences than a workgroup looks through: pieces are chunks of so many pages of a sequence, found by the table's row pointers (page `at` of the table is the sequence's first).  Half the average of a place by the
// whole table and the bound of the trees, for lengths and trees the host does not know: 1024 sequences of 100 to 1000 tokens, 8 of them of 20 000, up to 26 nodes under a bound of 64, 32 heads on 8 of 128 channels 1070 us, of which 300 would be memory.
constexpr int chunk_pages(int64_t work, int places) {
  const int64_t chunk = (work + 2 * (int64_t)places - 1) / (2 * (int64_t)places);
  return (int)(chunk < 8 ? 8 : chunk < kLongest ? (chunk + 3) / 4 * 4 : kLongest);
}
// Cells again for what is cut alone: p pages make ceil(p / chunk) pieces, which is at most floor(2 p / chunk) where it is more than one; so sequences have places of their own by their begins, and all together at
// most four for each place of the card, however many they are.
constexpr int64_t chunk_cell(int64_t at, int chunk) { return 2 * at / chunk; }

}  // namespace spg

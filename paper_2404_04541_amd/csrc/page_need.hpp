// How many pages a row of a page table takes (plain C++: the host and the kernels count alike).
#pragma once
#include <cstdint>

namespace spg {

constexpr int kPage = 64;                              // tokens of a page
constexpr int64_t kMaxPages = int64_t(1) << 24;        // a cache has fewer
static_assert(64 * kMaxPages <= 0x7fffffff, "a wave's rows are added up in 32 bits");

// Pages of len tokens, or -1 where that is more than all the pages of the cache: lengths come from the caller's memory, and only what a cache can hold
// may reach the sums.
constexpr int page_need(int64_t len, int64_t pages) {
  const int64_t need = len / kPage + (len % kPage != 0);
  return need <= pages ? (int)need : -1;
}

}  // namespace spg

// C entries to the paged cache's index arithmetic, for the tests without a GPU.
#include "ckv_paged.hpp"

namespace {

// Whether any of the step's pages is there (`there`: of each table entry).
bool has_pages(const uint8_t* there, int shift, int p, int n) {
  return there[ckv::half_first(p, 0, n) >> shift] || there[ckv::half_first(p, 1, n) >> shift];
}

}  // namespace

extern "C" {
// A wave's steps through positions [step, step + take) * kPagedStep of a context
// of n, in the attention's order: the first positions of all halves whose rows it
// loads, steps without pages passed over.  Returns their number.
int t_attn_halves(int n, int shift, const uint8_t* there, int step, int take, int wave,
                  int32_t* first, int room) {
  const int end = std::min((step + take) * ckv::kPagedStep, n);
  int p = step * ckv::kPagedStep + wave * ckv::kPagedTile, count = 0;
  auto skip = [&](int next) {
    while (next < end && !has_pages(there, shift, next, n)) next += ckv::kPagedStep;
    return next;
  };
  auto load = [&](int at) {
    for (int i = 0; i < 2 && count < room; ++i) first[count++] = ckv::half_first(at, i, n);
  };
  if (p >= end || (p = skip(p)) >= end) return 0;
  load(p);
  for (int next = p + ckv::kPagedStep; next < end;) {
    next = skip(next);
    load(ckv::lookup_at(next, end));
    next += ckv::kPagedStep;
  }
  return count;
}
int t_half_last(int first, int n) { return ckv::half_last(first, n); }
}

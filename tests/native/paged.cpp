// C entries to the paged cache's index arithmetic, for the tests without a GPU.
#include "ckv_paged.hpp"

#include <sys/mman.h>

#include <atomic>
#include <condition_variable>
#include <cstring>
#include <mutex>
#include <thread>
#include <vector>

namespace {

// Whether any of the step's pages is there (`there`: of each table entry).
bool has_pages(const uint8_t* there, int shift, int p, int n) {
  return there[ckv::half_first(p, 0, n) >> shift] || there[ckv::half_first(p, 1, n) >> shift];
}

// A flag whose two users take turns as `turns` says, an access at a time (bit i:
// the joining one has the i-th; who is alone goes on).
struct Turns {
  uint64_t word;
  uint32_t turns;
  int at = 0;
  bool ended[2] = {false, false}, given = false;
  std::mutex mu = {};
  std::condition_variable cv = {};
};

struct TurnFlag {
  Turns* t;
  int me;
  template <class Access>
  uint64_t access(Access a) const {
    std::unique_lock<std::mutex> lk(t->mu);
    t->cv.wait(lk, [&] { return t->ended[1 - me] || (int)(t->turns >> t->at & 1u) == me; });
    const uint64_t was = a();
    t->at = std::min(t->at + 1, 31);
    t->cv.notify_all();
    return was;
  }
  uint64_t load() const {
    return access([&] { return t->word; });
  }
  void store(uint64_t x) const {
    access([&] { return t->word = x; });
  }
  uint64_t exchange(uint64_t x) const {
    return access([&] {
      const uint64_t was = t->word;
      t->word = x;
      if (me == 0) t->given = true;
      return was;
    });
  }
  void pause() const {}
  void end() const {
    std::lock_guard<std::mutex> lk(t->mu);
    t->ended[me] = true;
    t->cv.notify_all();
  }
};

}  // namespace

extern "C" {
// One hand-over through *word in that order of accesses.  Bit 0: it was taken;
// bit 1: it had been given by then.
int t_hand_over(uint64_t* word, uint64_t tag, uint32_t limit, uint32_t turns) {
  Turns t{*word, turns};
  int result = 0;
  std::thread give([&] {
    const TurnFlag f{&t, 0};
    ckv::hand_over(f, tag);
    f.end();
  });
  std::thread take([&] {
    const TurnFlag f{&t, 1};
    result = ckv::take_over(f, tag, limit);
    std::lock_guard<std::mutex> lk(t.mu);
    if (t.given) result |= 2;
    t.ended[1] = true;
    t.cv.notify_all();
  });
  give.join();
  take.join();
  *word = t.word;
  return result;
}
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
// Debug mode's check of a reading call whose table is the columns from `col` on
// of [B][stride] entries that end where readable memory ends: the smallest
// finding (kind << 56 | item, all ones: none).
uint64_t t_check_table(int B, int max_ctx, int shift, int num_pages, const int32_t* lens,
                       const int32_t* wide, int stride, int col, int* slots) {
  const size_t bytes = (size_t)B * stride * 4, guard = 1 << 16;
  const size_t room = (bytes + guard - 1) / guard * guard;
  char* m = static_cast<char*>(mmap(nullptr, room + guard, PROT_READ | PROT_WRITE,
                                    MAP_PRIVATE | MAP_ANONYMOUS, -1, 0));
  if (m == MAP_FAILED || mprotect(m + room, guard, PROT_NONE)) return 0;
  int32_t* t = reinterpret_cast<int32_t*>(m + room - bytes);
  std::memcpy(t, wide, bytes);
  ckv::PagedCheckArgs a = {};
  a.pg.table = t + col;
  a.pg.shift = shift;
  a.pg.num_pages = num_pages;
  a.pg.table_stride = stride;
  a.ctx_lens = lens;
  a.B = B;
  a.max_ctx = max_ctx;
  a.slots = *slots = (max_ctx + (1 << shift) - 1) >> shift;
  uint64_t got = ~0ull;
  for (int64_t i = 0; i < ckv::paged_check_items(a); ++i)
    if (const uint64_t kind = ckv::paged_check_item(a, i)) got = std::min(got, kind << 56 | i);
  munmap(m, room + guard);
  return got;
}
// Threads that take and give debug mode's flags: times that one was found in use,
// and (flags) how many there were.
int t_flag_pool(int threads, int rounds, int* flags) {
  ckv::FlagPool pool;
  std::atomic<unsigned long long> words[256] = {};
  std::atomic<int> made{0}, met{0};
  std::vector<std::thread> all;
  for (int t = 0; t < threads; ++t)
    all.emplace_back([&] {
      for (int i = 0; i < rounds; ++i) {
        ckv::FlagPool::Flag* f = pool.take([&](unsigned long long** word) {
          const int n = made.fetch_add(1);
          *word = reinterpret_cast<unsigned long long*>(&words[n < 256 ? n : 255]);
          return n < 256;
        });
        if (!f) continue;
        auto* w = reinterpret_cast<std::atomic<unsigned long long>*>(f->word);
        if (w->exchange(1)) met.fetch_add(1);
        std::this_thread::yield();
        w->store(0);
        pool.give(f);
      }
    });
  for (std::thread& t : all) t.join();
  *flags = made.load();
  return met.load();
}
int t_half_last(int first, int n) { return ckv::half_last(first, n); }
}

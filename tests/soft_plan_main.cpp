// The workspace plans of ps_soft under the host's compiler: over seeded tables, options and sizes up to the limits, what
// ps_soft_reserve grows to holds every smaller call, every piece of an axis has work, and no size overflows.
// Compiled by test_soft_plan.py with the undefined-behaviour sanitizer; ends with a count of failures.
#include <cmath>
#include <cstdint>
#include <cstdio>

#include "../paper_1410_8043_amd/csrc/soft_plan.h"

using namespace pssoft;

namespace {

uint64_t state = 0x14108043u;
uint64_t draw() {
  state += 0x9e3779b97f4a7c15ull;
  uint64_t z = state;
  z = (z ^ (z >> 30)) * 0xbf58476d1ce4e5b9ull;
  z = (z ^ (z >> 27)) * 0x94d049bb133111ebull;
  return z ^ (z >> 31);
}
double unit() { return (draw() >> 11) * 0x1p-53; }
// between lo and hi, even over the logarithm
int64_t between(int64_t lo, int64_t hi) {
  const double v = std::exp(std::log(lo + 1.0) + unit() * (std::log(hi + 1.0) - std::log(lo + 1.0))) - 1.0;
  return std::min(hi, std::max(lo, static_cast<int64_t>(std::llround(v))));
}

int failures = 0;
void fail(const char *what, const Shape &h, int64_t n, int64_t entries, int32_t k, int64_t need, int64_t have) {
  if (++failures <= 20)
    std::printf("%s: items %lld K %d type %d splits %d search %d: n %lld entries %lld k %d: needs %lld, reserved %lld\n", what,
                static_cast<long long>(h.items), h.K, h.type, h.splits, h.search, static_cast<long long>(n),
                static_cast<long long>(entries), k, static_cast<long long>(need), static_cast<long long>(have));
}

void check_loss(const Shape &h, int64_t n, int64_t entries, bool dx, bool dw, int64_t room) {
  const Plan p = plan(&h, n, entries, dx, dw);
  if (p.bytes > room) fail("loss", h, n, entries, 0, p.bytes, room);
  const bool pieces_work = p.rsplits >= 1 && (p.few ? (p.rsplits - 1) * p.few_items < h.items && p.rsplits * p.few_items >= h.items
                                                    : (p.rsplits - 1) * p.rper < p.wt && p.rsplits * p.rper >= p.wt);
  if (!pieces_work || (dw && !((p.csplits - 1) * p.cper < p.xt && p.csplits * p.cper >= p.xt)) || p.bytes <= 0) fail("pieces", h, n, entries, 0, p.bytes, room);
}

void check_top(const Shape &h, int64_t n, int32_t k, bool exclude, int64_t room) {
  const TopPlan p = top_plan(&h, n, k, exclude, h.search);
  if (p.bytes > room) fail(exclude ? "top with exclusions" : "top", h, n, 0, k, p.bytes, room);
  if (p.rows < 1 || p.bytes <= 0) fail("rows", h, n, 0, k, p.bytes, room);
  if (p.filter && !((p.splits - 1) * p.per_split < p.steps && p.splits * p.per_split >= p.steps && p.per_split % 2 == 0))
    fail("steps", h, n, 0, k, p.bytes, room);
  // a launch of one form's rows stays near a gigabyte, whatever the table's size
  const int64_t row = p.filter ? 0 : static_cast<int64_t>(p.groups) * (kTopGroup + 1) * 8;
  if (!p.filter && p.rows > 1 && p.rows * row > (1LL << 30)) fail("a launch's rows", h, n, 0, k, p.rows * row, 1LL << 30);
}

void reserve_and_call(const Shape &h, int64_t n, int64_t entries, int32_t top) {
  const int64_t room = reserved_bytes(&h, n, entries, top);
  for (int call = 0; call < 60; ++call) {
    const int64_t m = call == 0 ? n : call == 1 ? 0 : call < 20 ? std::max<int64_t>(0, n - between(0, 600)) : between(0, n);
    const int64_t e = call % 3 == 0 ? entries : between(0, entries);
    check_loss(h, m, e, draw() & 1, draw() & 1, room);
    check_loss(h, m, e, false, false, room);
    if (top > 0) {
      const int32_t k = call % 4 == 0 ? top : static_cast<int32_t>(between(1, top));
      check_top(h, m, k, draw() & 1, room);
      check_top(h, m, call % 5 == 0 ? 1 : k, false, room);
    }
  }
}

}  // namespace

int main() {
  // tables whose rows of a launch differ with and without exclusions
  for (const Shape &h : {Shape{95'190, 34, 2, 0, -1}, Shape{100'000, 128, 0, 0, -1}, Shape{100'000, 16, 0, 0, 1}, Shape{20'000, 64, 1, 0, -1}})
    for (int64_t n : {40'000, 62'884, 120'000}) reserve_and_call(h, n, 4 * n, 64), reserve_and_call(h, n, n, 1);
  // the limits
  for (int32_t K : {1, 512})
    for (int32_t search : {-1, 0, 1})
      for (int64_t items : {int64_t{1}, kMaxItems, kMaxItems - 1, int64_t{1} << 30, (int64_t{1} << 30) - 1, int64_t{1} << 25})
        for (int64_t n : {int64_t{0}, int64_t{1}, kMaxRows}) reserve_and_call(Shape{items, K, PS_SOFT_F32, 0, search}, n, kMaxEntries, kMaxTop);
  for (int k = 0; k < 20'000; ++k) {
    Shape h;
    h.items = between(1, k % 10 == 0 ? kMaxItems : 3'000'000);
    h.K = static_cast<int32_t>(between(1, kMaxK));
    h.type = static_cast<int32_t>(draw() % 3);
    h.splits = draw() % 4 == 0 ? static_cast<int32_t>(between(1, 1024)) : 0;
    h.search = draw() % 3 == 0 ? static_cast<int32_t>(draw() % 2) : -1;
    reserve_and_call(h, between(0, k % 10 == 1 ? kMaxRows : 300'000), between(0, k % 7 == 0 ? kMaxEntries : 5'000'000),
                     draw() % 8 == 0 ? 0 : static_cast<int32_t>(between(1, kMaxTop)));
  }
  std::printf("%d failures\n", failures);
  return failures != 0;
}

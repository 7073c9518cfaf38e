// Holds the paged attention's host-side plan (csrc/plan.cpp) against the device; built with
// g++ under AddressSanitizer and UndefinedBehaviorSanitizer by
// tests/test_paged_plan_host.py. The device chooses from the lengths how many
// blocks a range has; for drawn shapes, lengths and chunks it repeats the
// device's counts and checks, for every choice the device may make, that
//  * a sequence's rows belong to one class, in tiles that the kernels have;
//  * the items fit the grid and the split items' partials their slots;
//  * the regions of the workspace are aligned, ordered and inside its total,
//    and sps_paged_workspace_bytes covers every smaller call.
#include <algorithm>
#include <cmath>
#include <cstdio>
#include <random>
#include <utility>
#include <vector>

#include "../../paper_2302_01318_amd/csrc/plan.h"

using namespace sps;

static int failures = 0;
#define CHECK(cond, ...)                                              \
  do {                                                                \
    if (!(cond)) {                                                    \
      if (failures++ < 20) {                                          \
        std::fprintf(stderr, "FAIL %s:%d: ", __FILE__, __LINE__);     \
        std::fprintf(stderr, __VA_ARGS__);                            \
        std::fprintf(stderr, "\n");                                   \
      }                                                               \
    }                                                                 \
  } while (0)

struct Seq {
  long tiles, blocks;
};

// Items and slots per KV head with the first `whole` tiles unsplit and `per`
// blocks to a range of the others.
static void count(const std::vector<Seq>& s, long whole, long per, long* items, long* slots) {
  *items = *slots = 0;
  for (const Seq& q : s) {
    const long ranges = std::max(1L, (q.blocks + per - 1) / per), kept = std::min(whole, q.tiles);
    whole -= kept;
    *items += kept + (q.tiles - kept) * ranges;
    if (ranges > 1) *slots += (q.tiles - kept) * ranges;
  }
}

static void check_class(const sps_paged_config& c, const PagedClass& k, const std::vector<Seq>& s, const char* name) {
  long tiles = 0, most = 0, work = 0;
  for (const Seq& q : s)
    if (q.tiles) {
      tiles += q.tiles;
      most = std::max(most, q.blocks);
      work += q.tiles * q.blocks;
    }
  if (!tiles) return;
  CHECK(k.items > 0, "%s: rows but no grid", name);
  std::vector<std::pair<long, long>> choices;                           // (whole, per)
  if (c.B > kMaxFew) {
    choices.push_back({0, std::max<long>(kPagedMinBlocks, static_cast<long>(std::ceil(static_cast<double>(work) *
                                                                                      c.n_kv_heads / k.target)))});
  } else {
    const long rounds = tiles * c.n_kv_heads / k.target;
    for (long whole : {0L, rounds * k.target / c.n_kv_heads})
      for (long n = 1; n <= 64; ++n) {
        const long per = std::max<long>(kPagedMinBlocks, (most + n - 1) / n);
        long items, slots;
        count(s, whole, per, &items, &slots);
        if ((n == 1 && !whole) || (items - whole) * c.n_kv_heads <= static_cast<long>(whole ? 1 : kPagedMostItems) * k.target)
          choices.push_back({whole, per});
      }
  }
  for (const auto& [whole, per] : choices) {
    long items, slots;
    count(s, whole, per, &items, &slots);
    CHECK(items * c.n_kv_heads <= k.items, "%s: %ld items x %d, grid %ld (B %d, per %ld)", name, items, c.n_kv_heads,
          k.items, c.B, per);
    CHECK(slots * c.n_kv_heads <= k.slots, "%s: %ld slots x %d, have %ld (B %d, per %ld)", name, slots, c.n_kv_heads,
          k.slots, c.B, per);
  }
}

int main() {
  std::mt19937_64 g(20260101);
  auto draw = [&](long lo, long hi) { return lo + static_cast<long>(g() % static_cast<uint64_t>(hi - lo + 1)); };
  auto log_draw = [&](double lo, double hi) {
    return static_cast<long>(lo * std::exp(std::uniform_real_distribution<double>(0, std::log(hi / lo + 1e-9))(g)) + 0.5);
  };
  for (int round = 0; round < 20000; ++round) {
    sps_paged_config c{};
    c.n_kv_heads = static_cast<int>(log_draw(1, 40));
    c.n_heads = c.n_kv_heads * static_cast<int>(log_draw(1, round % 5 ? 8 : 25));
    c.head_dim = draw(0, 1) ? 128 : 64;
    c.dtype = draw(0, 2) ? SPS_DTYPE_BF16 : SPS_DTYPE_F32;
    c.n_layers = 1;
    c.n_pages = 64;
    c.page_size = 32 << draw(0, 5);
    c.B = static_cast<int>(log_draw(1, round % 3 ? 64 : 1024));
    c.max_pages = static_cast<int>(log_draw(1, (1 << 22) / c.page_size));
    if (!valid_paged(&c)) {
      CHECK(false, "a drawn shape is refused");
      continue;
    }
    const int G = c.n_heads / c.n_kv_heads;
    const long cap = static_cast<long>(c.max_pages) * c.page_size;
    const bool ragged = draw(0, 3) != 0;
    const long longest = log_draw(1, draw(0, 1) ? 8 : 2000);
    std::vector<long> n(c.B);
    long rows = 0, max_tokens = 0;
    for (long& x : n) {
      x = !ragged ? longest : draw(0, 2) ? log_draw(1, static_cast<double>(longest)) : draw(0, 1) ? 0 : longest;
      if (rows + x > kMaxPagedRows) x = 0;
      rows += x;
      max_tokens = std::max(max_tokens, x);
    }
    if (!ragged && rows != longest * c.B) continue;
    if (!rows) continue;
    if (ragged && draw(0, 1)) max_tokens += draw(0, 100);               // a bound that no sequence reaches
    const long more = ragged && draw(0, 3) == 0 ? draw(0, 50) : 0;      // rows of no sequence
    const PagedPlan p = paged_plan(c, ragged, static_cast<int>(rows + more), static_cast<int>(max_tokens));
    const long window = draw(0, 2) ? 0 : log_draw(1, 100000);
    const double far = draw(0, 1) ? static_cast<double>(cap) : static_cast<double>(std::min(cap, 200L));
    std::vector<Seq> few, many;
    for (int b = 0; b < c.B; ++b) {
      const long p0 = draw(0, 9) ? log_draw(1, far) - 1 : cap - 1;
      const long end = std::min(std::max(p0 + n[b], 0L), cap), lo = window ? std::min(std::max(p0 - window + 1, 0L), end) : 0;
      const long q = n[b] * G, blocks = (end + 31) / 32 - lo / 32;
      if (q > 0 && q <= p.limit) {
        few.push_back({1, blocks});
        CHECK(q <= p.few.tile && q <= 16L * paged_few_tiles(c.dtype), "%ld rows in a tile of %d", q, p.few.tile);
      } else if (q > 0) {
        many.push_back({(q + kManyTile - 1) / kManyTile, blocks});
      }
    }
    check_class(c, p.few, few, "few");
    check_class(c, p.many, many, "many");
    // The workspace.
    size_t at = 0;
    for (const PagedClass* k : {&p.few, &p.many}) {
      if (!k->items) continue;
      CHECK(k->o_off >= at && k->o_off % 256 == 0 && k->ml_off % 256 == 0 && k->join_off % 256 == 0 && k->count_off % 256 == 0,
            "regions");
      CHECK(k->ml_off - k->o_off >= static_cast<size_t>(k->slots) * k->tile * c.head_dim * 4 &&
                k->join_off - k->ml_off >= static_cast<size_t>(k->slots) * k->tile * 8 &&
                k->count_off - k->join_off >= static_cast<size_t>(k->slots) * kPagedJoinBytes,
            "region sizes");
      at = k->count_off + 4;
    }
    CHECK(at <= p.total, "the workspace's end");
    const long r2 = rows + more + draw(0, 300), m2 = max_tokens + draw(0, 300);
    if (r2 <= kMaxPagedRows && m2 <= kMaxPagedRows)
      CHECK(paged_workspace_bytes(&c, static_cast<int>(r2), static_cast<int>(m2)) >= p.total, "workspace of a larger call");
  }
  if (failures) {
    std::fprintf(stderr, "%d failures\n", failures);
    return 1;
  }
  std::puts("paged plan check ok");
  return 0;
}

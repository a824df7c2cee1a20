// The shares that an attention over a paged cache is cut into, walked through on the host as the kernels do: every column of
// every sequence once, partial results within the memory that the call asks for, none written twice, none where nobody merges
// them.  Built with -fsanitize=address,undefined.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <random>
#include <vector>

#include "treekv_shares.h"

using namespace tkv;
typedef long long ll;

#define CHECK(cond) do { if (!(cond)) { fprintf(stderr, "%s:%d: %s: CHECK failed: %s\n", __FILE__, __LINE__, name, #cond); exit(1); } } while (0)

struct Case {
  int dtype, kv_heads, G, d, page_size, longest;
  std::vector<int> lens, news;
};

// The sequences of one launch with least to most rows; `part`: bytes of partial results, of tiles of `rows` rows.
static void walk(const char* name, const Case& x, const treekv_paged_cache& c, int shares, int tiles, int rows, bool tiled, bool keep,
                 int least, int most, size_t part) {
  const int B = c.batch;
  const bool wide = past_32_bits(c);
  std::vector<int> length(B);
  ll total = 0;
  for (int b = 0; b < B; ++b) {
    const ll r = (ll)x.news[b] * x.G;
    length[b] = r >= least && r <= most ? (x.lens[b] + 31) & ~31 : 0;
    total += length[b];
  }
  const Cut cut = cut_columns(total, shares, B, tiled, wide, [&](int size) {
    int n = 0;
    for (int b = 0; b < B && b < 64; ++b) n += shares_in(length[b], size);
    return n;
  });
  CHECK(cut.size >= MIN_SHARE && cut.size % 32 == 0);
  const ll slots = (ll)(part / ((size_t)c.kv_heads * tiles * rows * (c.head_dim + 4) * 4));
  const bool sparse = is_sparse(shares, B, keep);
  std::vector<ll> start(B);
  std::vector<Runs> run(B);
  std::vector<ll> next(B, 0);              // columns seen
  std::vector<int> pieces(B, 0), part0(B);
  ll at = 0, column = 0;
  for (int b = 0; b < B; ++b) {
    start[b] = at;
    run[b] = runs_of(cut, wide, at, length[b]);
    part0[b] = part_of_first(cut, wide, sparse, run[b], column, b);
    column += length[b];
    at += cut.own ? shares_in(length[b], cut.size) : length[b];
  }
  std::map<ll, int> taken;
  for (ll w = 0; w < shares + B - 1; ++w) {
    const ll share_end = cut.own ? w + 1 : (w + 1) * cut.size;
    for (ll from = cut.own ? w : w * cut.size; from < share_end;) {
      int b = 0;                           // the sequence that holds `from`
      ll mine = 0;
      for (; b < B; ++b) {
        mine = cut.own ? shares_in(length[b], cut.size) : length[b];
        if (mine > 0 && start[b] + mine > from) break;
      }
      if (b == B) break;
      const ll lo = cut.own ? (w - run[b].first) * cut.size : from - start[b];
      const ll hi = std::min((ll)length[b], cut.own ? lo + cut.size : share_end - start[b]);
      CHECK(lo == next[b] && hi > lo && lo <= INT_MAX && hi <= INT_MAX);
      next[b] = hi;
      CHECK(w - run[b].first == pieces[b]);
      if (run[b].count > 1 || keep) {
        const ll slot = part0[b] + part_at(sparse, pieces[b]);
        CHECK(slot >= 0 && slot < slots && taken.emplace(slot, b).second);
      }
      if (run[b].count > 1) CHECK(shares > 1);           // (or nothing merges them)
      ++pieces[b];
      from = cut.own ? share_end : start[b] + length[b];
    }
  }
  for (int b = 0; b < B; ++b) CHECK(next[b] == length[b] && pieces[b] == run[b].count);
}

static void check(const char* name, const Case& x) {
  treekv_paged_cache c;
  memset(&c, 0, sizeof(c));
  int cap = 1, tokens = 0, longest = x.longest;
  for (int n : x.lens) cap = std::max(cap, n);
  for (int n : x.news) { tokens += n; longest = std::max(longest, n); }
  c.page_size = x.page_size;
  c.table_width = (int)(((ll)cap + x.page_size - 1) / x.page_size);
  c.pages = 8; c.batch = (int)x.lens.size(); c.kv_heads = x.kv_heads; c.q_heads = x.kv_heads * x.G; c.head_dim = x.d; c.dtype = x.dtype;
  for (int weigh = 0; weigh < 2; ++weigh) {
    if (weigh && (ll)c.batch * c.kv_heads * cap > 1 << 30) continue;
    const AttendShape s = attend_shape(c, std::max(tokens, longest), longest, weigh);
    CHECK(s.shares >= 1 && s.tiles >= 1);
    if (s.short_shares) walk(name, x, c, s.short_shares, 1, 16, false, s.short_keep, 1, 16, s.short_part);
    walk(name, x, c, s.shares, s.tiles, s.rows, s.tiled, s.keep, s.short_shares ? 17 : 1, INT_MAX, s.part);
  }
}

int main() {
  const int M = 1 << 20;
  // more than 2^30 columns: shares of a sequence each where there is one share, two or many; up to the longest sequences
  check("two of 256 heads", {TREEKV_BF16, 256, 1, 64, 256, 1, {(1 << 30) - 1000, 5000}, {1, 1}});
  check("1024 beams", {TREEKV_F32, 1, 32, 64, 256, 256, std::vector<int>(1024, M + 40), std::vector<int>(1024, 1)});
  check("two shares", {TREEKV_BF16, 128, 1, 128, 256, 1, {1 << 30, 1 << 30, 1 << 30, 77}, {1, 1, 1, 1}});
  check("one head", {TREEKV_BF16, 1, 4, 64, 128, 1, {1 << 30, 3, 1 << 29, 1 << 30, 1 << 30}, {1, 1, 1, 1, 1}});
  check("row tiles", {TREEKV_BF16, 8, 8, 64, 256, 8192, {1 << 30, 1 << 30, 4096}, {8192, 1, 4096}});
  check("row tiles of one", {TREEKV_BF16, 8, 64, 64, 256, 4096, {1 << 30}, {4096}});
  // scratch goes by what a call has to merge, not by as many sequences as there are of the longest chunk
  {
    const char* name = "scratch";
    treekv_paged_cache c;
    memset(&c, 0, sizeof(c));
    c.page_size = 32; c.table_width = 512; c.pages = 8; c.batch = 256; c.kv_heads = 8; c.q_heads = 32; c.head_dim = 128; c.dtype = TREEKV_BF16;
    const AttendShape s = attend_shape(c, 1024 + 255, 1024, 0);
    CHECK(s.part + s.short_part + s.logits + s.stat + s.gains < (size_t)200 << 20);            // (out: 10 MB)
    c.dtype = TREEKV_F32;
    CHECK(attend_shape(c, 256 * 200, 200, 0).part < (size_t)300 << 20);                        // (out: 838 MB)
  }
  // a merge's launch: as many workgroups as there may be, each row of a sequence has one
  for (int batch : {1, 20, 4096, 16384, 1 << 20})
    for (int kv_heads : {1, 8, 32, 256})
      for (int G : {1, 7, 32})
        for (int longest : {1, 64, 255, 512, 1 << 20})
          for (int at_once : {1, 2, 8, 16})
            for (int full : {1, 2, 4, 1000}) {       // tokens: a part of what the longest chunk of all would be
              const char* name = "merge";
              if ((ll)batch * kv_heads > 1 << 20 || (ll)longest * G * kv_heads * batch > 1 << 28) continue;
              const int tokens = (int)std::min(std::max((ll)batch * longest / full, (ll)longest), 1ll << 27), rows = longest * G;
              const MergeGrid m = merge_grid(batch, kv_heads, G, tokens, rows, at_once);
              const ll groups = (ll)m.groups * kv_heads * (m.packed ? 1 : batch);
              CHECK(m.groups >= 1 && groups <= MAX_GROUPS);
              if (m.packed) CHECK(m.groups >= ((ll)tokens * G + at_once - 1) / at_once);      // one or more a sequence, no row without
            }
  std::mt19937 g(5);
  auto any = [&](std::initializer_list<int> of) { return of.begin()[g() % of.size()]; };
  for (int i = 0; i < 6000; ++i) {
    Case x;
    x.dtype = any({TREEKV_BF16, TREEKV_BF16, TREEKV_F32});
    x.kv_heads = any({1, 1, 2, 3, 8, 32, 100, 256});
    x.G = any({1, 1, 2, 4, 7, 16, 40});
    x.d = any({64, 128});
    x.page_size = any({16, 64, 256});
    const int B = any({1, 2, 3, 5, 16, 63, 64, 65, 130}), top = any({40, 500, 3000, 40000, M}), most = any({1, 1, 5, 40, 300});
    x.longest = any({1, 1, most, 2 * most});
    for (int b = 0; b < B; ++b) {
      const int n = g() % 7 == 0 ? 0 : 1 + (int)(g() % (g() % 3 ? 1 : most));
      x.news.push_back(n);
      x.lens.push_back(n + (int)(g() % top));
    }
    char name[64];
    snprintf(name, sizeof(name), "random %d", i);
    check(name, x);
  }
  puts("shares cover every column");
  return 0;
}

// Index arithmetic of the paged cache's kernels, run on the host: random batches, sound and
// unsound ones.  Every row and position that a call should touch is dealt to exactly one tile,
// and nothing outside the rows or the table is, whatever the lengths say.
#include <stdio.h>
#include <stdlib.h>

#include <algorithm>
#include <map>
#include <random>
#include <tuple>
#include <vector>

#include "../../paper_2403_01164_amd/csrc/paged.h"

using namespace hg;

#define CHECK(c)                                                  \
  do {                                                            \
    if (!(c)) {                                                   \
      printf("line %d: %s (case %d)\n", __LINE__, #c, g_case);    \
      exit(1);                                                    \
    }                                                             \
  } while (0)
static int g_case = 0;

// The device's search: the last sequence whose tiles begin at or before `tile`, counted as the
// wavefronts count (64 at a time, ending at the first group that is not wholly before).
static int find(const PagedSeqs& b, int tile, int unit, int shift, int extra, int* local) {
  int count = 0;
  for (int i0 = 0; i0 < b.n_seq; i0 += 64) {
    int c = 0;
    for (int i = i0; i < std::min(b.n_seq, i0 + 64); ++i)
      c += paged_tile_base(b.start[i], i, b.n_tokens, unit, shift, extra) <= tile;
    count += c;
    if (c < 64) break;
  }
  const int s = count - 1;
  *local = s < 0 ? 0 : tile - paged_tile_base(b.start[s], s, b.n_tokens, unit, shift, extra);
  return *local < 0 ? -1 : s;
}

int main() {
  std::mt19937 rng(7);
  auto pick = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); };
  for (g_case = 0; g_case < 3000; ++g_case) {
    const bool sound = g_case % 4 != 0;
    const int shift = 5 + pick(0, 3), page = 1 << shift;
    PagedSeqs b{};
    b.n_seq = pick(1, g_case % 10 == 0 ? 200 : 9);
    b.max_pages = pick(1, 40);
    std::vector<int32_t> start(b.n_seq + 1), len(b.n_seq);
    int t = pick(0, 3) ? 0 : pick(0, 5);
    for (int s = 0; s < b.n_seq; ++s) {
      start[s] = t;
      const int n = pick(0, 3) == 0 ? 0 : pick(0, 3) ? pick(1, 4) : pick(1, 300);
      t += n;
      len[s] = pick(0, 9) == 0 ? pick(0, n) : n + pick(0, 1200);
    }
    start[b.n_seq] = t;
    b.n_tokens = t + (pick(0, 3) ? 0 : pick(0, 70));
    b.max_new = pick(0, 3) ? std::max(1, b.n_tokens) : pick(1, 50);
    if (!sound) {  // anything at all
      for (auto& v : start) if (pick(0, 2) == 0) v = pick(0, 1) ? pick(-400, 2000) : (int32_t)rng();
      for (auto& v : len) if (pick(0, 2) == 0) v = pick(0, 1) ? pick(-400, 2000) : (int32_t)rng();
    }
    b.start = start.data();
    b.len = len.data();

    // rows of (token, head of the group), in tiles of 16 and of 128
    for (int tile_shift : {4, 7}) {
      const int group = pick(1, 9), M = 1 << tile_shift;
      std::vector<int> hits((size_t)b.n_tokens * group);
      for (long long tile = 0; tile < paged_tiles(b, group, tile_shift, 1); ++tile) {
        int local;
        const int s = find(b, (int)tile, group, tile_shift, 1, &local);
        if (s < 0) continue;
        CHECK(s < b.n_seq && local >= 0);
        const PagedSeq q = paged_seq(b.start[s], b.start[s + 1], b.len[s], b, shift);
        CHECK(q.row >= 0 && q.n >= 0 && q.row + q.n <= b.n_tokens && q.done <= q.n && q.done <= b.max_new);
        CHECK(q.held >= 0 && q.held <= b.max_pages * page);
        const long long row0 = (long long)local << tile_shift;
        for (long long r = row0; r < std::min<long long>(row0 + M, (long long)q.done * group); ++r) {
          const long long at = ((long long)q.row * group) + r;
          CHECK(at < (long long)hits.size());
          ++hits[at];
        }
      }
      if (sound)
        for (int s = 0; s < b.n_seq; ++s)
          for (int i = 0; i < start[s + 1] - start[s]; ++i)
            for (int g = 0; g < group; ++g)
              CHECK(hits[(size_t)(start[s] + i) * group + g] == (i < b.max_new ? 1 : 0));
    }

    // positions, in tiles of 32
    std::vector<int> hits(b.n_tokens);
    for (long long tile = 0; tile < paged_tiles(b, 1, 5, 2); ++tile) {
      int local;
      const int s = find(b, (int)tile, 1, 5, 2, &local);
      if (s < 0) continue;
      const PagedSeq q = paged_seq(b.start[s], b.start[s + 1], b.len[s], b, shift);
      const PagedTile p = paged_tile(q, local);
      if (p.hi <= p.lo) continue;
      CHECK(p.j0 % 32 == 0 && p.lo >= 0 && p.hi <= 32);
      for (int i = p.lo; i < p.hi; ++i) {
        const long long row = (long long)p.row + i;
        CHECK(row >= 0 && row < b.n_tokens);
        if (sound) CHECK((long long)q.first + (row - q.row) == (long long)p.j0 + i);
        ++hits[row];
      }
      if (p.j0 < q.held) CHECK((p.j0 >> shift) < b.max_pages);
    }
    if (sound)
      for (int s = 0; s < b.n_seq; ++s)
        for (int i = 0; i < start[s + 1] - start[s]; ++i) {
          const int n = start[s + 1] - start[s];
          CHECK(hits[start[s] + i] == (i < b.max_new && len[s] - n + i >= 0 ? 1 : 0));
        }

    // pieces of a sequence: no more than its cap allows, whole steps, nothing left over or empty
    const int cap = pick(0, 1) ? pick(1, 100) * 32 : pick(1, 1 << 25) * 32;
    const int most = pick(1, kPagedMaxSplits), heads = pick(1, 100), want = pick(1, 2000);
    const int held = std::min(cap, pick(0, 1) ? pick(0, 3000) : pick(0, 1 << 30));
    const long long others = pick(0, 1) ? 0 : pick(0, 1 << 24);
    const PagedPieces s = paged_pieces(held, paged_unit(((held + 127) >> 7) + others, heads, want), most);
    CHECK(s.size >= 128 && s.size % 128 == 0 && s.count >= 1);
    CHECK((long long)s.count * s.size >= held);
    CHECK(s.count <= paged_most_pieces(cap, heads, want, most) && paged_most_pieces(cap, heads, want, most) <= most);

    // items (tile, piece) of a batch without gaps: no more than the launch has workgroups for
    if (b.n_seq > kPagedDense || b.n_tokens == 0) continue;
    const int group = pick(1, 4), R = pick(0, 1) ? 16 : 32, cap_b = b.max_pages * page;
    const bool limited = pick(0, 1);  // the kernel for many rows takes the others
    const int max_rows = limited ? 64 : 0x7FFFFFFF;
    const long long longest = (long long)std::min(b.max_new, b.n_tokens) * group;
    const int each = (int)((std::min<long long>(longest, limited ? 64 : longest) + R - 1) / R);
    long long total = 0, items = 0;
    for (int pass = 0; pass < 2; ++pass) {
      const int unit = paged_unit(total, heads, want);
      for (int i = 0; i < b.n_seq; ++i) {
        const PagedSeq q = paged_seq(b.start[i], b.start[i + 1], b.len[i], b, shift);
        const int tiles = paged_few_tiles(q, group, 0, max_rows, R);
        CHECK(tiles <= each);
        if (pass == 0) total += (long long)tiles * ((q.held + 127) >> 7);
        else items += (long long)tiles * paged_pieces(q.held, unit, most).count;
        if (pass == 1 && tiles)
          CHECK(paged_pieces(q.held, unit, most).count <= paged_most_pieces(cap_b, heads, want, most));
      }
    }
    CHECK(items <= paged_most_items(cap_b, b.n_seq, each, heads, want, most));

    // the kernel's numbering: every (sequence, tile, piece) is one item, and items past the last none
    const int unit = paged_unit(total, heads, want);
    std::vector<int> tiles(b.n_seq), count(b.n_seq);
    std::map<std::tuple<int, int, int>, int> seen;
    for (int i = 0; i < b.n_seq; ++i) {
      const PagedSeq q = paged_seq(b.start[i], b.start[i + 1], b.len[i], b, shift);
      tiles[i] = paged_few_tiles(q, group, 0, max_rows, R);
      count[i] = paged_pieces(q.held, unit, most).count;
    }
    if (items > 20000) continue;
    for (int w = 0; w < items + 70; ++w) {
      int c = 0, before = 0;
      auto upto_piece = [&](int n) {
        long long sum = 0;
        for (int i = 0; i < b.n_seq; ++i) sum += (long long)tiles[i] * std::min(count[i], n);
        return sum;
      };
      if (b.n_seq > 1) {
        for (int bit = kPagedMaxSplits / 2; bit > 0; bit >>= 1)
          if (upto_piece(c + bit) <= w) {
            c += bit;
            before = (int)upto_piece(c);
          }
      } else {
        c = tiles[0] > 0 ? w / tiles[0] : 0;
        before = c * tiles[0];
      }
      int upto = 0, found = -1, local = 0;
      for (int i = 0; i < b.n_seq && found < 0; ++i) {
        const int n = count[i] > c ? tiles[i] : 0;
        if (upto + n > w - before) {
          found = i;
          local = w - before - upto;
        }
        upto += n;
      }
      CHECK((found >= 0) == (w < items));
      if (found < 0) continue;
      CHECK(local >= 0 && local < tiles[found] && c < count[found]);
      CHECK(++seen[std::make_tuple(found, local, c)] == 1);
    }
  }
  printf("index check ok\n");
  return 0;
}

// Internal launch interface of the paged KV cache's kernels (not part of the C ABI).
//
// Layout.  The cache is n_pages pages; a page holds page_size positions of every key/value
// head, one record per head: record (page, head) at (page * heads + head) * record bytes.  A
// record is the keys, then the values, then (8-bit formats) page_size binary32 scales of the
// keys and page_size of the values.  Keys and values stand in the order in which the matrix
// cores take them, so that every load of a wavefront is 1 KiB of consecutive memory:
//   keys    tiles of 16 positions; the 16 bytes of lane l (position l % 16 of the tile, dimension
//           group g = l / 16) of load i hold the tile's dimensions 32 i + 8 g + [0, 8), or, in 8
//           bits, 64 i + 8 g + [0, 8) and 64 i + 32 + 8 g + [0, 8);
//   values  tiles of 32 positions; the 16 bytes of lane l (dimension l % 16 of a group of 16,
//           g = l / 16) of load i hold 8 positions of dimension 16 i + l % 16, or, in 8 bits, 8 of
//           32 i + l % 16 and 8 of 32 i + 16 + l % 16; element e is position
//           16 (e / 4) + 4 g + e % 4, where the product of keys and queries leaves the weights.
#pragma once
#include <hip/hip_runtime_api.h>
#include <stddef.h>
#include <stdint.h>

namespace hg {

enum KvFormat : int { KV_SAME = 0, KV_I8 = 1, KV_E4M3 = 2 };

struct PagedCache {
  void* pages;
  long long record;  // bytes of one head of one page
  int heads, head_dim, page_size, page_shift, n_pages;
  int dtype, format;
};

// Rows [start[s], start[s + 1]) of the batch are sequence s's newest positions, which end at
// len[s].  Device arrays; whatever they hold, no kernel reads or writes outside the batch's rows,
// the table and the pages.
struct PagedSeqs {
  const int32_t* start;  // [n_seq + 1]
  const int32_t* len;    // [n_seq]
  const int32_t* table;  // [n_seq, max_pages]
  int n_tokens, n_seq, max_new, max_pages;
};

inline size_t paged_record_bytes(int head_dim, int page_size, int format) {
  const size_t data = (size_t)2 * page_size * head_dim * (format == KV_SAME ? 2 : 1);
  return data + (format == KV_SAME ? 0 : (size_t)2 * page_size * 4);
}

// ---- index arithmetic shared by kernels and host ----

// A sequence's rows and positions: rows [row, row + n) of the batch are positions first + [0, n);
// only the first `done` of them are worked on; the cache holds positions [0, held).
struct PagedSeq {
  int row, n, done, first, held;
};

__host__ __device__ inline int paged_clamp(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }

__host__ __device__ inline PagedSeq paged_seq(int start, int end, int len, const PagedSeqs& b, int page_shift) {
  PagedSeq s;
  s.row = paged_clamp(start, 0, b.n_tokens);
  s.n = paged_clamp(end, s.row, b.n_tokens) - s.row;
  s.done = s.n < b.max_new ? s.n : b.max_new;
  len = len < 0 ? 0 : len;
  s.first = len - s.n;
  const int cap = b.max_pages << page_shift;
  s.held = len < cap ? len : cap;
  return s;
}

// Work is dealt in tiles of 2^shift units (rows of a head group, or positions) of one sequence.
// The tiles of sequence s begin at tile paged_tile_base: sequence s has at most
// base(s + 1) - base(s) of them, because ceil(n / M) <= floor(end / M) - floor(start / M) + 1
// (extra = 1), and n positions touch at most floor(n / M) + 2 aligned tiles (extra = 2).  So
// a workgroup finds its sequence without a prefix sum over the others' lengths.
__host__ __device__ inline int paged_tile_base(int start, int s, int n_tokens, int unit, int shift, int extra) {
  return ((paged_clamp(start, 0, n_tokens) * unit) >> shift) + s * extra;
}
inline long long paged_tiles(const PagedSeqs& b, int unit, int shift, int extra) {
  return (((long long)b.n_tokens * unit) >> shift) + (long long)b.n_seq * extra;
}

// Positions [j0, j0 + 32) of a sequence, its local-th aligned tile from its first new position
// on: those of j0 + [lo, hi) are new, position j0 + i in row `row` + i of the batch.
struct PagedTile {
  int j0, row, lo, hi;  // hi <= lo: nothing to do
};
__host__ __device__ inline PagedTile paged_tile(const PagedSeq& q, int local) {
  PagedTile t = {0, 0, 0, 0};
  const int from = q.first > 0 ? q.first : 0;
  const long long to = (long long)q.first + q.done;
  const long long j0 = ((long long)(from >> 5) + local) << 5;
  if (j0 >= to) return t;
  t.j0 = (int)j0;
  t.row = q.row + (t.j0 - q.first);
  t.lo = from > t.j0 ? from - t.j0 : 0;
  t.hi = to - j0 < 32 ? (int)(to - j0) : 32;
  return t;
}

// The kernel for few rows shares a sequence's positions among workgroups, in units of 128: pieces
// of at most `unit` units, all of them alike, as long as there are no more than `most`.
constexpr int kPagedMaxSplits = 64;
constexpr int kPagedMaxUnit = 16;
struct PagedPieces {
  int count, size;  // pieces (at least 1), positions in each but the last
};
__host__ __device__ inline PagedPieces paged_pieces(int held, int unit, int most) {
  const int units = (held + 127) >> 7;
  int n = (units + unit - 1) / unit;
  n = n < 1 ? 1 : n < most ? n : most;
  const int each = units <= n ? 1 : (units + n - 1) / n;
  return PagedPieces{n, each << 7};
}
// The unit for `total` units in all of a batch's tiles, `heads` key/value heads: as many pieces as
// `want` workgroups, or as a few times that, so that the last of them end together.
__host__ __device__ inline int paged_unit(long long total, int heads, int want) {
  const long long work = total * heads;
  const long long rounds = (work + (long long)want * kPagedMaxUnit - 1) / ((long long)want * kPagedMaxUnit);
  const long long u = (work + want * rounds - 1) / (want * (rounds < 1 ? 1 : rounds));
  return u < 1 ? 1 : (int)u;
}
// The most pieces of a sequence of up to `cap` positions, whatever the others' lengths: in one
// round the unit is at least its own units * heads / want, in several at least half of
// kPagedMaxUnit.
inline int paged_most_pieces(long long cap, int heads, int want, int most) {
  const long long units = (cap + 127) >> 7;
  long long n = units / (kPagedMaxUnit / 2) + 1;
  if (n < want / heads + 1) n = want / heads + 1;
  if (n > units) n = units;
  return (int)(n < 1 ? 1 : n < most ? n : most);
}
// Tiles of a sequence with min_rows < rows <= max_rows, of `tile` rows.
__host__ __device__ inline int paged_few_tiles(const PagedSeq& q, int group, int min_rows, int max_rows, int tile) {
  const long long rows = (long long)q.n * group;
  return rows <= min_rows || rows > max_rows ? 0 : (q.done * group + tile - 1) / tile;
}
// Items (tile, piece) of a batch of up to kPagedDense sequences are numbered without gaps, so that
// workgroups without work do not come between the others (the device deals neighbouring workgroups
// to its engines in turn); this many at most, tiles <= tiles_each for each sequence.
constexpr int kPagedDense = 64;
inline long long paged_most_items(long long cap, int n_seq, int tiles_each, int heads, int want, int most) {
  const long long units = (cap + 127) >> 7;
  const long long n = units * n_seq * tiles_each / kPagedMaxUnit + want / heads + 1 + (long long)n_seq * tiles_each;
  const long long top = (long long)n_seq * tiles_each * paged_most_pieces(cap, heads, want, most);
  return n < top ? n : top;
}

// ---- launches ----

// Rows [n_tokens, heads * head_dim] of keys and values (row stride ld elements) in the cache's
// 16-bit type, into the cache or out of it.
struct PagedCopyParams {
  PagedCache kv;
  PagedSeqs seqs;
  void* k;
  void* v;
  long long ld;
};
hipError_t launch_paged_write(const PagedCopyParams& p, hipStream_t stream);
hipError_t launch_paged_read(const PagedCopyParams& p, hipStream_t stream);

struct PagedAttnParams {
  PagedCache kv;
  PagedSeqs seqs;
  const void* q;  // [n_tokens, heads * head_dim], row stride ldq
  long long ldq;
  void* out;      // likewise
  long long ldo;
  int heads;      // query heads, a multiple of kv.heads
  int group;      // set by the launcher: heads / kv.heads
  float scale;    // set by the launcher: the caller's scale times log2 e
  uint32_t* cnt;  // kPagedCounters arrival counters, zero between launches
  float* part;    // partial results of split sequences
  int splits;     // set by the launcher: the most workgroups that share a sequence's positions
  int want, most; // set by the launcher: workgroups that fill the device, and splits there is room for
  int tiles_each; // set by the launcher: the most tiles of a sequence
  int min_rows;   // set by the launcher: sequences with more than min_rows rows per key/value head
  int max_rows;   // and at most max_rows are worked on
};

constexpr int kPagedCounters = 65536;
// Bytes of workspace (counters, then partials) that any launch of these sizes needs; does not
// shrink as n_tokens, n_seq, max_new or max_pages grow.
size_t paged_ws_bytes(const PagedCache& kv, const PagedSeqs& b, int heads);
hipError_t launch_paged_attention(PagedAttnParams p, double scale, void* ws, hipStream_t stream);

}  // namespace hg

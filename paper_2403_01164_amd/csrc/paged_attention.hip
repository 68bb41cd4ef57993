// Attention of new tokens over a paged KV cache, on gfx950.
//
//   s_j = scale * q . K_j  for the positions j <= p that the cache holds,
//   out = sum_j softmax(s)_j V_j      (no such position: 0)
//
// for every new token (position p) and query head; `group` query heads share a key/value head,
// and the rows of a tile are (token, head of the group) pairs, so that all of them share its keys
// and values.
//
// Both kernels work on the matrix cores without moving the weights between lanes: keys are the
// 16-row operand of a 16x16x32 product whose 16 columns are queries, so lane l ends up with four
// keys' scores of query l % 16; those, rounded to 16 bits, are the 16-column operand of the product
// with the values (whose rows are dimensions), because the order in which that product sums over
// keys is free and the pages store the values in the order in which the scores come out.  A
// query's running maximum and sum are the lane's own numbers.  Softmax statistics and sums are
// binary32; scores carry log2 e.
//
// 8-bit caches: codes become fp16 exactly and are multiplied as fp16 (queries, too: a power of
// two per row, taken back in the score's factor, keeps bf16 queries in range, exactly unless a value
// is 2^29 times smaller than its row's largest).  A key's scale multiplies its score; a value's
// scale multiplies its weight, relative to a power of two per wavefront that follows the largest
// scale seen, so that the product is no larger than the weight.
#include "paged_device.h"

#include <math.h>

#include <algorithm>
#include <type_traits>

namespace hg {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kTiny = 1.4e-45f;  // the least factor of a score: with 0, a masked one would be -inf * 0

template <class A, int FMT>
struct Compute {
  typedef F16 type;
};
template <class A>
struct Compute<A, KV_SAME> {
  typedef A type;
};

// 8 codes -> 8 fp16 values, exactly.
template <int FMT>
__device__ __forceinline__ u32x4 codes_f16(uint32_t lo, uint32_t hi) {
  u32x4 r;
  const uint32_t w[2] = {lo, hi};
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (FMT == KV_I8) {
      // 0x6400 | u is 1024 + u; u = code + 128
      const uint32_t u = w[h] ^ 0x80808080u;
      const f16x2 bias = {(_Float16)1152.f, (_Float16)1152.f};
      const f16x2 a = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) - bias;
      const f16x2 b = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) - bias;
      r[2 * h] = __builtin_bit_cast(uint32_t, a);
      r[2 * h + 1] = __builtin_bit_cast(uint32_t, b);
    } else {
      r[2 * h] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w[h], 1.0f, false));
      r[2 * h + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w[h], 1.0f, true));
    }
  }
  return r;
}

// A query row's fragments for the key products, 8 dimensions of each 32 a lane, and *mult, what
// turns a sum of products into a score (positive: a negative scale changes the query's sign).  ok: the row exists (0 otherwise).
template <class A, int FMT, int D>
__device__ __forceinline__ void load_query(const uint16_t* q, bool ok, float scale, u32x4* f, float* mult) {
#pragma unroll
  for (int k = 0; k < D / 32; ++k) {
    f[k] = ok ? load16(q + 32 * k) : u32x4{0u, 0u, 0u, 0u};
    f[k] ^= scale < 0.f ? 0x80008000u : 0u;
  }
  scale = fabsf(scale);
  *mult = fmaxf(scale, kTiny);
  if (FMT == KV_SAME && __is_same(A, F16)) return;
  // power of two that takes the row's largest value to [2^14, 2^15) (fp16 products), or to
  // [2^-8, 2^-7) (bf16: then no sum of products overflows whose score does not)
  uint32_t m = 0;
#pragma unroll
  for (int k = 0; k < D / 32; ++k)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t w = f[k][j] & 0x7FFF7FFFu;
      m = max(m, max(w & 0xFFFFu, w >> 16));
    }
  const float top = A::to_f32(groups_umax(m));
  int e = 0;
  if (top > 0.f && top < INFINITY) e = (FMT == KV_SAME ? -7 : 15) - __builtin_amdgcn_frexp_expf(top);
#pragma unroll
  for (int k = 0; k < D / 32; ++k) {
    float v[8];
    unpack8<A>(f[k], v);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      f[k][j] = Compute<A, FMT>::type::pack(__builtin_amdgcn_ldexpf(v[2 * j], e), __builtin_amdgcn_ldexpf(v[2 * j + 1], e));
  }
  *mult = fmaxf(__builtin_amdgcn_ldexpf(scale, -e), kTiny);
}

// Scales (none is negative) compare as their bits do, infinity above every number and NaN above it.
constexpr uint32_t kInfBits = 0x7F800000u;
__device__ __forceinline__ uint32_t bits_of(float v) { return __builtin_bit_cast(uint32_t, v); }
__device__ __forceinline__ float as_float(uint32_t v) { return __builtin_bit_cast(float, v); }
__device__ __forceinline__ uint32_t finite_bits(float v) { return bits_of(v) < kInfBits ? bits_of(v) : 0u; }

// The larger of two numbers in one instruction: fmaxf would first make each one canonical, which
// the products' sums are not known to be.
__device__ __forceinline__ float max_of(float a, float b) { return __builtin_amdgcn_fmed3f(a, b, INFINITY); }

__device__ __forceinline__ float exp2_hw(float v) { return __builtin_amdgcn_exp2f(v); }

// Infinities and NaNs in values.  A product gives 0 * infinity = NaN to queries that do not see a
// key (weight 0), and to those whose weight of it rounded to 0.  The kernels look for that in
// their sums only, at the end, and when one is not finite they walk the positions again with
// this: it takes the infinities and NaNs out of 32 keys' values and adds them to the sums of
// the queries that see their keys.  vis: bit e set where this lane's query sees element e of
// this lane's group.
template <class T>
__device__ __forceinline__ u32x4 seen_keys(uint32_t vis) {
  u32x4 r;
#pragma unroll
  for (int w = 0; w < 4; ++w) r[w] = ((vis >> (2 * w) & 1u) | (vis >> (2 * w + 1) & 1u) << 16) * (uint32_t)T::from_f32(1.f);
  return r;
}
// v: 16 dimensions of 32 keys; sees[u] = seen_keys of the u-th 16 queries, *O[u] their sums.
template <class T, int U>
__device__ __forceinline__ void take_nonfinite(u32x4& v, const u32x4* sees, f32x4* const* O) {
  constexpr uint32_t kOnes = 0x00010001u;  // 1 in both halves of a word
  constexpr uint32_t kMantissa = T::kExpLow - kOnes;
  constexpr int kBits = __builtin_ctz(T::kExpLow);
  const uint32_t one = T::from_f32(1.f);
  u32x4 up, down, nan;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    // an exponent of all ones carries into the sign's place
    const uint32_t odd = ((v[w] & T::kExp) + T::kExpLow) >> 15 & kOnes;
    const uint32_t is_nan = odd & ((v[w] & kMantissa) + kMantissa) >> kBits;
    const uint32_t is_down = odd & v[w] >> 15 & ~is_nan;
    nan[w] = is_nan * one;
    down[w] = is_down * one;
    up[w] = (odd & ~is_nan & ~is_down) * one;
    v[w] &= ~(odd * 0xFFFFu);
  }
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const f32x4 a = T::mfma(up, sees[u], zero), b = T::mfma(down, sees[u], zero), c = T::mfma(nan, sees[u], zero);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      (*O[u])[i] += (a[i] > 0.f ? INFINITY : 0.f) + (b[i] > 0.f ? -INFINITY : 0.f) + (c[i] > 0.f ? NAN : 0.f);
  }
  __builtin_amdgcn_sched_barrier(0);  // one fragment at a time: this path is rare, registers are not
}

// Partials cross workgroups on different XCDs (separate L2s): buffer accesses that go to memory (sc0
// sc1), so that no cache has to be written back or emptied.  Word 3 is the gfx9 raw-buffer format.
constexpr int kThrough = 1 | 16;
__device__ __forceinline__ __amdgpu_buffer_rsrc_t partials(float* p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(p, (short)0, (int)bytes, 0x00020000);
}

// v of the lane that the DPP control names, and op over the N (8 or 16) lanes that share a row.
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, false));
}
template <int N, class F>
__device__ __forceinline__ float over_lanes(float v, F op) {
  v = op(v, dpp<0xB1>(v));
  v = op(v, dpp<0x4E>(v));
  v = op(v, dpp<0x141>(v));
  return N == 16 ? op(v, dpp<0x140>(v)) : v;
}

// ---- few rows: one token of a sequence, or some ----
//
// Workgroup (tile of 16 U rows, key/value head, chunk of positions) of four wavefronts, each with
// 32 positions at a time; keys and values go from memory straight into the products' operands,
// 1 KiB a load, and feed U products.  The wavefronts' sums meet in LDS; a sequence of several
// chunks leaves partials [m, l, o] in the workspace and the last workgroup of (tile, head) to arrive
// joins them in chunk order (an arrival counter, no waiting), so results do not depend on timing.
// Memory bounds it, and a fixed part of each launch: 8 sequences over 16000 positions, 40 heads of
// 128, int8, 215 us (6.1 TB/s), over 4000 64 us (4.8); one sequence of 513, 32 heads, fp16, 8.6 us.
constexpr int kFewWaves = 4;
template <int U>
constexpr int kFewShift = U == 2 ? 5 : 4;  // rows per tile: 16 U

// A workgroup's work: rows [row0, row0 + 16 U) of sequence s and its chunk-th piece of positions.
struct FewItem {
  PagedSeq q;
  int s, tile, chunk, size;  // size: positions of a piece
  uint32_t counter;
};

// Item number w, the same in every lane of the wavefront; false: there is none.
template <int U>
__device__ __forceinline__ bool few_item(const PagedAttnParams& p, int w, FewItem* it) {
  const PagedSeqs& b = p.seqs;
  constexpr int R = 16 * U;
  if (b.n_seq > kPagedDense) {  // work enough in large pieces; gaps and all, a piece of every tile at a time
    const int tiles = (int)(((long long)b.n_tokens * p.group >> kFewShift<U>) + b.n_seq);
    const int tile = w % tiles;
    it->s = paged_find(b, p.kv.page_shift, tile, p.group, kFewShift<U>, 1, &it->tile, &it->q);
    if (it->s < 0 || it->tile >= paged_few_tiles(it->q, p.group, p.min_rows, p.max_rows, R)) return false;
    const PagedPieces piece = paged_pieces(it->q.held, kPagedMaxUnit, p.most);
    it->chunk = w / tiles;
    it->size = piece.size;
    it->counter = (uint32_t)tile;
    return it->chunk < piece.count;
  }
  const int lane = threadIdx.x & 63, i = min(lane, b.n_seq - 1);
  const int st = load_i32(b.start + i);
  const PagedSeq q = paged_seq(st, load_i32(b.start + i + 1), load_i32(b.len + i), b, p.kv.page_shift);
  const int tiles = lane < b.n_seq ? paged_few_tiles(q, p.group, p.min_rows, p.max_rows, R) : 0;
  // (at most 4 tiles of 2^23 units for each of 64 sequences)
  const int unit = paged_unit(wave_sum((uint32_t)tiles * ((q.held + 127) >> 7)), p.kv.heads, p.want);
  const PagedPieces piece = paged_pieces(q.held, unit, p.most);
  // the first pieces of all tiles come first, then the second ones: c is the piece with no more
  // than w items in all pieces before it
  int c = 0, before = 0;
  if (b.n_seq > 1) {
#pragma unroll
    for (int bit = kPagedMaxSplits / 2; bit > 0; bit >>= 1) {
      const int n = (int)wave_sum((uint32_t)(tiles * min(piece.count, c + bit)));
      if (n <= w) {
        c += bit;
        before = n;
      }
    }
  } else {
    const int t = __builtin_amdgcn_readfirstlane(tiles);
    c = t > 0 ? w / t : 0;
    before = c * t;
  }
  const int items = piece.count > c ? tiles : 0;
  const int upto = wave_scan(items);  // of this sequence and those before it
  const uint64_t behind = __ballot(upto > w - before);
  if (!behind) return false;
  const int s = __builtin_ctzll(behind);
  it->s = s;
  it->q = PagedSeq{__builtin_amdgcn_readlane(q.row, s), __builtin_amdgcn_readlane(q.n, s),
                   __builtin_amdgcn_readlane(q.done, s), __builtin_amdgcn_readlane(q.first, s),
                   __builtin_amdgcn_readlane(q.held, s)};
  it->tile = w - before - __builtin_amdgcn_readlane(upto - items, s);
  it->chunk = c;
  it->size = __builtin_amdgcn_readlane(piece.size, s);
  it->counter = (uint32_t)(s * p.tiles_each + it->tile);
  return true;
}

template <class A, int FMT, int D, int U>
__global__ __launch_bounds__(64 * kFewWaves, U == 2 ? 2 : D == 128 ? 3 : 4) void paged_few_kernel(PagedAttnParams p) {
  typedef typename Compute<A, FMT>::type T;
  constexpr int ES = FMT == KV_SAME ? 2 : 1;
  constexpr int KK = D / 32, DT = D / 16, R = 16 * U;
  constexpr int NL = 32 * D * ES / 1024;   // loads of 32 positions' keys (or values)
  constexpr int OS = D + 4;
  __shared__ __align__(16) float sacc[kFewWaves][R][OS];
  __shared__ float sm[kFewWaves][R], sl[kFewWaves][R];  // sm: then the wavefronts' weights
  __shared__ float s_m[R], s_l[R];
  __shared__ int s_last;

  const int head = blockIdx.x % p.kv.heads;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, g = lane >> 4;
  FewItem it;
  // a lone sequence's first 64 pages need not wait for its length
  const bool lone = p.seqs.n_seq == 1;
  const int first_pages = lone && lane < p.seqs.max_pages ? load_i32(p.seqs.table + lane) : -1;
  if (!few_item<U>(p, blockIdx.x / p.kv.heads, &it)) return;
  const PagedSeq& q = it.q;
  const int s = it.s, c = it.chunk;
  const int row0 = it.tile << kFewShift<U>;
  const int rows = min(q.done * p.group - row0, R);  // of this tile
  // a token at position t sees positions [0, t]; the tile's last one sees the most
  const int last = q.first + (row0 + rows - 1) / p.group;
  const int kend = max(min(q.held, last + 1), 0);
  const int nchunk = max((kend + it.size - 1) / it.size, 1);
  if (c >= nchunk) return;
  const int j0 = c * it.size, j1 = min(j0 + it.size, kend);
  const int nsteps = (max(j1 - j0, 0) + 31) >> 5;

  const int minpos = q.first + row0 / p.group;  // the least a row of the tile sees to
  int mypos[U];
  u32x4 qf[U][KK];
  float mult[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int row = row0 + 16 * u + col;
    const bool ok = 16 * u + col < rows;
    mypos[u] = ok ? q.first + row / p.group : -1;
    load_query<A, FMT, D>((const uint16_t*)p.q + (long long)(q.row + row / p.group) * p.ldq +
                              (head * p.group + row % p.group) * D + 8 * g,
                          ok, p.scale, qf[u], &mult[u]);
  }

  const long long P = p.kv.page_size;
  const int pmask = p.kv.page_size - 1;
  const char* base = (const char*)p.kv.pages + (long long)head * p.kv.record;
  const long long page_bytes = p.kv.record * p.kv.heads;

  u32x4 kr[NL], vr[NL];
  f32x4 ksc[2], vsc[2];
  float m[U], l[U];
  uint32_t seen[U];
  int ve;  // values' scales are taken relative to 2^ve
  f32x4 O[U][DT];

  // lane i holds the page of this wavefront's step number n0 + i
  int pages = -1;
  auto look_up = [&](int n0) {
    const int j = j0 + 32 * (wave + kFewWaves * (n0 + lane));
    if (lone && (j1 - 1) >> p.kv.page_shift < 64) {
      const int entry = paged_entry(p.kv, __shfl(first_pages, (j >> p.kv.page_shift) & 63));
      pages = j < j1 ? entry : -1;
    } else {
      pages = j < j1 ? paged_page(p.seqs, p.kv, s, j) : -1;
    }
  };
  auto load_keys = [&](int page, int j) {
    const char* rec = base + max(page, 0) * page_bytes;
    const char* src = rec + (long long)(j & pmask) * D * ES + lane * 16;
#pragma unroll
    for (int i = 0; i < NL; ++i) kr[i] = load16_nt(src + i * 1024);
    if (FMT != KV_SAME) {
      const char* sc = rec + 2 * P * D + ((j & pmask) + 4 * g) * 4;
#pragma unroll
      for (int t = 0; t < 2; ++t) ksc[t] = __builtin_bit_cast(f32x4, load16(sc + 64 * t));
    }
  };
  auto load_values = [&](int page, int j) {
    const char* rec = base + max(page, 0) * page_bytes;
    const char* src = rec + (P + (j & pmask)) * D * ES + lane * 16;
#pragma unroll
    for (int i = 0; i < NL; ++i) vr[i] = load16_nt(src + i * 1024);
    if (FMT != KV_SAME) {
      const char* sc = rec + 2 * P * D + P * 4 + ((j & pmask) + 4 * g) * 4;
#pragma unroll
      for (int t = 0; t < 2; ++t) vsc[t] = __builtin_bit_cast(f32x4, load16(sc + 64 * t));
    }
  };

  auto walk = [&](auto again) {
    constexpr bool careful = decltype(again)::value;
    ve = -126;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      m[u] = -INFINITY;
      l[u] = 0.f;
      seen[u] = 0;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) O[u][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    int page = -1, n = 0;
    if (wave < nsteps) {
      look_up(0);
      page = __builtin_amdgcn_readlane(pages, 0);
      if (!careful) {
        load_keys(page, j0 + 32 * wave);
        load_values(page, j0 + 32 * wave);
      }
    }
    for (int st = wave; st < nsteps; st += kFewWaves) {
      const int jb = j0 + 32 * st;
      const bool more = st + kFewWaves < nsteps;
      int next = -1;
      if (more) {
        if ((++n & 63) == 0) look_up(n);
        next = __builtin_amdgcn_readlane(pages, n & 63);
      }
      if (careful) load_keys(page, jb);  // nothing ahead of its use: fewer registers
      // scores
      f32x4 sc[U][2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int u = 0; u < U; ++u) sc[u][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < KK; ++k) {
          u32x4 kf;
          if (FMT == KV_SAME) {
            kf = kr[t * KK + k];
          } else {
            const u32x4& w = kr[t * (KK / 2) + (k >> 1)];
            kf = codes_f16<FMT>(w[2 * (k & 1)], w[2 * (k & 1) + 1]);
          }
#pragma unroll
          for (int u = 0; u < U; ++u) sc[u][t] = T::mfma(kf, qf[u][k], sc[u][t]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (FMT == KV_SAME) sc[u][t] *= mult[u];
          else sc[u][t] *= mult[u] * ksc[t];
        }
      }
      if (more && !careful) load_keys(next, jb + 32 * kFewWaves);
      if (careful) load_values(page, jb);
      // the last positions, and positions of a page that is not there, are masked
      const bool whole = page >= 0 && jb + 32 <= q.held;
      const bool full = whole && jb + 31 <= minpos;
      const int top = (page >= 0 ? q.held - 1 : -1) - (jb + 4 * g);  // element e is held if up to here
      uint32_t vis[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        vis[u] = 0xFFu;
        if (!full) {
          const int to = min(mypos[u] - (jb + 4 * g), top);
          vis[u] = 0u;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const bool see = 16 * (e >> 2) + (e & 3) <= to;
            vis[u] |= (see ? 1u : 0u) << e;
            sc[u][e >> 2][e & 3] = see ? sc[u][e >> 2][e & 3] : -INFINITY;
          }
        }
        seen[u] |= vis[u];
      }
      f32x4 vs[2];
      int e2 = ve;
      if (FMT != KV_SAME) {
        uint32_t most = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) most = max(most, bits_of(vsc[e >> 2][e & 3]));
        if (!whole || __ballot(most >= kInfBits)) {  // scales that no position has, or that are no numbers
          most = 0;
#pragma unroll
          for (int e = 0; e < 8; ++e)
            most = max(most, 16 * (e >> 2) + (e & 3) <= top ? finite_bits(vsc[e >> 2][e & 3]) : 0u);
        }
        e2 = max(ve, (int)(groups_umax(most) >> 23) - 126);
        const float to = __builtin_amdgcn_ldexpf(1.f, -e2);
#pragma unroll
        for (int t = 0; t < 2; ++t) vs[t] = vsc[t] * to;
      }
      if (!whole) {
        // what lies behind a sequence's end was never written: it may be anything
        u32x4 keep;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (FMT == KV_SAME) {  // elements 2 i and 2 i + 1 of a dimension
            const int to = top - (16 * (i >> 1) + 2 * (i & 1));
            keep[i] = (to >= 0 ? 0xFFFFu : 0u) | (to >= 1 ? 0xFFFF0000u : 0u);
          } else {  // elements 4 (i % 2) + [0, 4) of one of two dimensions
            const int to = top - 16 * (i & 1);
            keep[i] = to >= 3 ? ~0u : to < 0 ? 0u : ~0u >> (24 - 8 * to);
          }
        }
#pragma unroll
        for (int i = 0; i < NL; ++i) vr[i] &= keep;
      }
      auto fragment = [&](int dt) {
        if (FMT == KV_SAME) return vr[dt];
        return codes_f16<FMT>(vr[dt >> 1][2 * (dt & 1)], vr[dt >> 1][2 * (dt & 1) + 1]);
      };
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float mx = fmaxf(fmaxf(fmaxf(sc[u][0][0], sc[u][0][1]), fmaxf(sc[u][0][2], sc[u][0][3])),
                         fmaxf(fmaxf(sc[u][1][0], sc[u][1][1]), fmaxf(sc[u][1][2], sc[u][1][3])));
        mx = fmaxf(m[u], groups_max(mx));
        const float ms = mx == -INFINITY ? 0.f : mx;
        float al = exp2_hw(m[u] - ms), w[8], sum = 0.f;
        m[u] = mx;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          w[e] = exp2_hw(sc[u][e >> 2][e & 3] - ms);
          sum += w[e];
        }
        l[u] = fmaf(l[u], al, sum);
        if (FMT != KV_SAME) {
          al = __builtin_amdgcn_ldexpf(al, ve - e2);
#pragma unroll
          for (int e = 0; e < 8; ++e) w[e] *= vs[e >> 2][e & 3];
          if (!full) {
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = vis[u] >> e & 1u ? w[e] : 0.f;
          }
        }
        if (__ballot(al != 1.f)) {
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) O[u][dt] *= al;
        }
        // weights to 16 bits twice: a second product takes what the first rounding left (memory is
        // what bounds this kernel), so that weights count as in binary32 but for fp16's smallest step
        u32x4 pf, pl;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          pf[i] = T::pack(w[2 * i], w[2 * i + 1]);
          pl[i] = T::pack(w[2 * i] - T::to_f32(pf[i] & 0xFFFFu), w[2 * i + 1] - T::to_f32(pf[i] >> 16));
        }
        const u32x4 sees = seen_keys<T>(vis[u]);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          u32x4 vf = fragment(dt);
          if (careful) {
            f32x4* const o[1] = {&O[u][dt]};
            take_nonfinite<T, 1>(vf, &sees, o);
          }
          O[u][dt] = T::mfma(vf, pl, T::mfma(vf, pf, O[u][dt]));
        }
      }
      ve = e2;
      if (more && !careful) load_values(next, jb + 32 * kFewWaves);
      page = next;
    }
  };
  walk(std::false_type{});
  if (FMT == KV_SAME) {
    bool odd = false;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) odd |= !(fabsf(O[u][dt][i]) < INFINITY);
    if (__ballot(odd)) walk(std::true_type{});
  }

#pragma unroll
  for (int u = 0; u < U; ++u) {
    // a row that saw positions, all of score -infinity, has no softmax: NaN, as the formula has it
    l[u] = groups_sum(l[u]);
    if (m[u] == -INFINITY && groups_umax(seen[u]) != 0) l[u] = NAN;
    const int r = 16 * u + col;
    if (r >= rows) continue;
    if (g == 0) {
      sm[wave][r] = m[u];
      sl[wave][r] = l[u];
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      f32x4 o = O[u][dt];
      if (FMT != KV_SAME) {
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = __builtin_amdgcn_ldexpf(o[i], ve);
      }
      *(f32x4*)&sacc[wave][r][16 * dt + 4 * g] = o;
    }
  }
  __syncthreads();

  // the wavefronts' sums, in order; one without a visible position has m = -inf and weight 0
  const int t = threadIdx.x;
  if (t < rows) {
    float M = -INFINITY, L = 0.f;
#pragma unroll
    for (int i = 0; i < kFewWaves; ++i) M = fmaxf(M, sm[i][t]);
#pragma unroll
    for (int i = 0; i < kFewWaves; ++i) {
      const bool none = sm[i][t] == -INFINITY;
      const float f = none ? 0.f : exp2_hw(sm[i][t] - M);
      // (without any, what counts is whether one of them saw a position: l is NaN then)
      L += none ? (M == -INFINITY ? sl[i][t] : 0.f) : f * sl[i][t];
      sm[i][t] = f;
    }
    s_m[t] = M;
    s_l[t] = L;
  }
  __syncthreads();
  constexpr int kQuads = D / 4;  // 4 dimensions of a row to a thread
  auto joined = [&](int r, int d) {
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kFewWaves; ++i) o += sm[i][r] * *(const f32x4*)&sacc[i][r][d];
    return o;
  };
  auto row_of = [&](int r, int* token) {
    const int rr = row0 + r;
    *token = q.row + rr / p.group;
    return head * p.group + rr % p.group;
  };
  auto finish = [&](int r, int d, f32x4 o, float L) {
    int token;
    const int qhead = row_of(r, &token);
    if (L == 0.f) o = f32x4{0.f, 0.f, 0.f, 0.f};
    else o = o / L;
    *(u32x2*)((uint16_t*)p.out + (long long)token * p.ldo + qhead * D + d) =
        u32x2{A::pack(o[0], o[1]), A::pack(o[2], o[3])};
  };
  if (nchunk == 1) {
    for (int i = t; i < rows * kQuads; i += 64 * kFewWaves) {
      const int r = i / kQuads, d = i % kQuads * 4;
      finish(r, d, joined(r, d), s_l[r]);
    }
    return;
  }
  // partials: o [rows][splits][D], then (m, l) [rows][splits]
  const uint32_t all_rows = (uint32_t)p.seqs.n_tokens * p.heads;
  const uint32_t ml_at = all_rows * p.splits * D;
  const auto part = partials(p.part, all_rows * p.splits * (D + 2) * 4);
  auto slot = [&](int r, int k) {
    int token;
    const int qhead = row_of(r, &token);
    return ((uint32_t)token * p.heads + qhead) * p.splits + k;
  };
  for (int i = t; i < rows * kQuads; i += 64 * kFewWaves) {
    const int r = i / kQuads, d = i % kQuads * 4;
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, joined(r, d)), part, (slot(r, c) * D + d) * 4, 0,
                                           kThrough);
  }
  if (t < rows)
    __builtin_amdgcn_raw_buffer_store_b64(u32x2{bits_of(s_m[t]), bits_of(s_l[t])}, part, (ml_at + slot(t, c) * 2) * 4, 0,
                                          kThrough);
  __builtin_amdgcn_s_waitcnt(0);  // this thread's partials are in memory
  __syncthreads();
  if (t == 0) {
    uint32_t* cnt = p.cnt + it.counter * p.kv.heads + head;
    const uint32_t prev = __hip_atomic_fetch_add(cnt, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    s_last = prev == (uint32_t)(nchunk - 1);
    if (s_last) __hip_atomic_store(cnt, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  if (!s_last) return;
  // join the chunks, in order: N lanes share a row's (m, l), whose weights go to LDS, while the
  // first partials are on their way
  constexpr int N = 64 * kFewWaves / R, kPer = kPagedMaxSplits / N, kAhead = 8;
  float* weight = &sacc[0][0][0];  // [R][kPagedMaxSplits]
  static_assert(kPagedMaxSplits <= kFewWaves * OS, "chunk weights");
  const int mr = t / N, mk = t % N;
  u32x2 ml[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i)
    ml[i] = mr < rows && mk + N * i < nchunk
                ? __builtin_amdgcn_raw_buffer_load_b64(part, (ml_at + slot(mr, mk + N * i) * 2) * 4, 0, kThrough)
                : u32x2{0xFF800000u, 0u};
  u32x4 ahead[kAhead];
  auto request = [&](int i, int k0) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (i < rows * kQuads && k0 + u < nchunk)
        ahead[u] = __builtin_amdgcn_raw_buffer_load_b128(
            part, (slot(i / kQuads, k0 + u) * D + i % kQuads * 4) * 4, 0, kThrough);
  };
  request(t, 0);
  {
    float M = -INFINITY, L = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) M = fmaxf(M, as_float(ml[i][0]));
    M = over_lanes<N>(M, [](float x, float y) { return fmaxf(x, y); });
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const float m_i = as_float(ml[i][0]), l_i = as_float(ml[i][1]);
      const bool none = m_i == -INFINITY;
      const float f = none ? 0.f : exp2_hw(m_i - M);
      L += none ? (M == -INFINITY ? l_i : 0.f) : f * l_i;
      weight[mr * kPagedMaxSplits + mk + N * i] = f;
    }
    L = over_lanes<N>(L, [](float x, float y) { return x + y; });
    if (mk == 0) s_l[mr] = L;
  }
  __syncthreads();
  for (int i = t; i < rows * kQuads; i += 64 * kFewWaves) {
    const int r = i / kQuads;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int k0 = 0; k0 < nchunk; k0 += kAhead) {
      if (i != t || k0 > 0) request(i, k0);
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (k0 + u < nchunk) o += weight[r * kPagedMaxSplits + k0 + u] * __builtin_bit_cast(f32x4, ahead[u]);
    }
    finish(r, i % kQuads * 4, o, s_l[r]);
  }
}

// ---- many rows: prompts and chunks of them ----
//
// Workgroup (tile of 128 rows, key/value head, share of the positions) of four wavefronts of 32
// rows each; 64 positions at a time go through LDS, one buffer being filled while the other is
// multiplied: 16-bit pages by loads that write to LDS themselves (the pages' order is the operands'
// order already), 8-bit ones through registers, where they become fp16.  Every operand read from
// LDS feeds two products.  The scores of the next step are computed beside the weights of this one,
// so that matrix cores and vector units have work at the same time, and a step has one barrier.
// When there are few tiles, several workgroups share a tile's positions and a second kernel joins
// their partials.  The softmax's vector work beside the products bounds it: prompts of 2048 and 7000
// tokens, 32 heads of 128, bf16, 464 to 505 us (863 to 939 TFLOP/s; a large library product 1214).
constexpr int kManyWaves = 4;
constexpr int kManyShift = 7;  // rows per tile: 128
constexpr int kManyKeys = 64;  // positions at a time
constexpr int kManyMaxSplits = 16;
constexpr int kManyWorkgroups = 512;  // two for each of the 256 CUs
constexpr long long kMaxManyPartials = 2LL * kManyWorkgroups << kManyShift;  // rows of all shares

// Shares of a tile's positions [0, kend): `per` steps of kManyKeys each, *used of them.
__device__ __forceinline__ int many_share(int kend, int splits, int* used) {
  const int steps = (kend + kManyKeys - 1) / kManyKeys;
  const int per = max((steps + splits - 1) / splits, 1);
  *used = max((steps + per - 1) / per, 1);
  return per;
}

template <class A, int FMT, int D>
__global__ __launch_bounds__(64 * kManyWaves, 2) void paged_many_kernel(PagedAttnParams p) {
  typedef typename Compute<A, FMT>::type T;
  constexpr int ES = FMT == KV_SAME ? 2 : 1;
  constexpr int KK = D / 32, DT = D / 16, U = 2;
  constexpr int KT = kManyKeys / 16;             // key tiles of a step
  constexpr int kSide = kManyKeys * D * 2;       // bytes of a step's keys (or values) in LDS
  constexpr int NL = kManyKeys * D * ES * 2 / 1024 / kManyWaves;  // loads of a step, per wavefront
  // Scores are a step ahead of weights where there are registers for that: 8-bit pages on their way
  // to LDS and their scales take them.  Keys come a step before their scores.
  constexpr bool kAhead = FMT == KV_SAME;
  __shared__ __align__(16) char keys0[kSide], keys1[kSide], values0[kSide], values1[kSide];
  __shared__ float scales[2][FMT == KV_SAME ? 1 : 2 * kManyKeys];  // of keys, then of values, by step % 2
  __shared__ int s_odd;

  const int head = blockIdx.x % p.kv.heads, tile = blockIdx.x / p.kv.heads;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, g = lane >> 4;
  int local;
  PagedSeq q;
  const int s = paged_find(p.seqs, p.kv.page_shift, tile, p.group, kManyShift, 1, &local, &q);
  if (s < 0) return;
  if ((long long)q.n * p.group <= p.min_rows) return;
  const int all = q.done * p.group;
  local = ((all + (1 << kManyShift) - 1) >> kManyShift) - 1 - local;  // the rows that see most come first
  if (local < 0) return;
  const int row0 = local << kManyShift;
  const int rows = min(all - row0, 1 << kManyShift);
  const int kend = max(min(q.held, q.first + (row0 + rows - 1) / p.group + 1), 0);
  int used;
  const int per = many_share(kend, p.splits, &used);
  const int c = blockIdx.y;
  if (c >= used) return;
  const int j0 = c * per * kManyKeys, j1 = min(j0 + per * kManyKeys, kend);
  const int nsteps = (max(j1 - j0, 0) + kManyKeys - 1) / kManyKeys;

  // this wavefront's rows
  const int wrow = row0 + 32 * wave, wrows = min(rows - 32 * wave, 32);
  const int wmin = q.first + wrow / p.group;                                       // its first row sees to here,
  const int wmax = wrows > 0 ? q.first + (wrow + wrows - 1) / p.group : -1;        // its last one to here
  u32x4 qf[U][KK];
  float mult[U];
  int mypos[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int row = wrow + 16 * u + col;
    const bool ok = 16 * u + col < wrows;
    mypos[u] = ok ? q.first + row / p.group : -1;
    load_query<A, FMT, D>((const uint16_t*)p.q + (long long)(q.row + row / p.group) * p.ldq +
                              (head * p.group + row % p.group) * D + 8 * g,
                          ok, p.scale, qf[u], &mult[u]);
  }

  const long long P = p.kv.page_size;
  const int pmask = p.kv.page_size - 1;
  const char* base = (const char*)p.kv.pages + (long long)head * p.kv.record;
  const long long page_bytes = p.kv.record * p.kv.heads;

  f32x4 O[U][DT];
  f32x4 lsum[U];  // 16-bit pages: the sums of weights come from a product with ones, alike in all elements
  float m[U], l[U];
  uint32_t seen[U];
  int ve;
  int pages = -1;  // lane i: the page of the i-th 32 positions from the last look-up on
  u32x4 raw[NL];   // 8-bit pages on their way to LDS
  float raw_scale = 0.f;
  struct Halves {
    int a, b;  // pages of a step's 32-position halves (-1: none)
  };
  const int half = wave & 1, side = wave >> 1;  // a wavefront brings one half's keys (0) or values (1)

  // of a step, in order of steps
  auto halves = [&](int step) {
    const int i = 2 * (step & 31);
    if (i == 0) {
      const int j = j0 + kManyKeys * step + 32 * lane;
      pages = j < j1 ? paged_page(p.seqs, p.kv, s, j) : -1;
    }
    return Halves{__builtin_amdgcn_readlane(pages, i), __builtin_amdgcn_readlane(pages, i + 1)};
  };
  auto issue = [&](char* keys, char* values, int step, Halves pg) {
    const int j = j0 + kManyKeys * step + 32 * half;
    const char* rec = base + max(half ? pg.b : pg.a, 0) * page_bytes;
    const char* src = rec + (side * P + (j & pmask)) * D * ES + lane * 16;
    if (FMT == KV_SAME) {
      char* dst = (side ? values : keys) + half * (kSide / 2);
#pragma unroll
      for (int i = 0; i < NL; ++i)
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(src + i * 1024),
                                         (__attribute__((address_space(3))) void*)(dst + i * 1024), 16, 0, 0);
    } else {
#pragma unroll
      for (int i = 0; i < NL; ++i) raw[i] = load16(src + i * 1024);
      if (lane < 32) raw_scale = ((const float*)(rec + 2 * P * D))[side * P + (j & pmask) + lane];
    }
  };
  auto commit = [&](char* keys, char* values, int step) {
    if (FMT != KV_SAME) {
      char* dst = (side ? values : keys) + half * (kSide / 2) + lane * 16;
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        *(u32x4*)(dst + 2 * i * 1024) = codes_f16<FMT>(raw[i][0], raw[i][1]);
        *(u32x4*)(dst + (2 * i + 1) * 1024) = codes_f16<FMT>(raw[i][2], raw[i][3]);
      }
      if (lane < 32) scales[step & 1][side * kManyKeys + 32 * half + lane] = raw_scale;
    }
  };
  auto score = [&](const char* keys, int step, f32x4(&sc)[KT][U]) {
#pragma unroll
    for (int t = 0; t < KT; ++t) {
#pragma unroll
      for (int u = 0; u < U; ++u) sc[t][u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KK; ++k) {
        const u32x4 kf = *(const u32x4*)(keys + lane * 16 + (t * KK + k) * 1024);
#pragma unroll
        for (int u = 0; u < U; ++u) sc[t][u] = T::mfma(kf, qf[u][k], sc[t][u]);
      }
      if (FMT != KV_SAME) {
        const f32x4 ks = *(const f32x4*)&scales[step & 1][16 * t + 4 * g];
#pragma unroll
        for (int u = 0; u < U; ++u) sc[t][u] *= ks;
      }
    }
  };
  // what lies behind a sequence's end was never written and may be anything: zeros for its values
  auto blank = [&](char* values, int step, Halves pg) {
    for (int i = threadIdx.x; i < kSide / 16; i += 64 * kManyWaves) {
      const int h = i >= kSide / 32, vg = (i & 63) >> 4;
      const int top = ((h ? pg.b : pg.a) >= 0 ? q.held - 1 : -1) - (j0 + kManyKeys * step + 32 * h + 4 * vg);
      u32x4* at = (u32x4*)values + i;
      u32x4 v = *at;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const int to = top - (16 * (w >> 1) + 2 * (w & 1));
        v[w] &= (to >= 0 ? 0xFFFFu : 0u) | (to >= 1 ? 0xFFFF0000u : 0u);
      }
      *at = v;
    }
  };
  // one step.  kAhead: sc are its scores, and those of the next step's keys afterwards; otherwise
  // its scores are computed here
  auto compute = [&](const char* keys, const char* values, int step, Halves pg, f32x4(&sc)[KT][U], auto again) {
    constexpr bool careful = decltype(again)::value;
    const int jb = j0 + kManyKeys * step;
    if (jb > wmax) return;
    if (!kAhead) score(keys, step, sc);
    const bool whole = pg.a >= 0 && pg.b >= 0 && jb + kManyKeys <= q.held;
    const bool full = whole && jb + kManyKeys - 1 <= wmin;
    // last position of either half that is in the cache
    const int top[2] = {pg.a >= 0 ? q.held - 1 : -1, pg.b >= 0 ? q.held - 1 : -1};
    const int jl = jb + 4 * g;  // element i of key tile t is position jl + 16 t + i
    uint32_t vis[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      vis[u] = 0xFFFFu;
      if (!full) {
        vis[u] = 0u;
#pragma unroll
        for (int t = 0; t < KT; ++t) {
          const int to = min(mypos[u], top[t >> 1]) - (jl + 16 * t);  // elements up to here are seen
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            vis[u] |= (i <= to ? 1u : 0u) << (4 * t + i);
            sc[t][u][i] = i <= to ? sc[t][u][i] : -INFINITY;
          }
        }
      }
      seen[u] |= vis[u];
    }
    // values' scales, relative to the largest so far
    f32x4 vs[KT];
    int e2 = ve;
    if (FMT != KV_SAME) {
      uint32_t most = 0;
#pragma unroll
      for (int t = 0; t < KT; ++t) {
        vs[t] = *(const f32x4*)&scales[step & 1][kManyKeys + 16 * t + 4 * g];
#pragma unroll
        for (int i = 0; i < 4; ++i) most = max(most, bits_of(vs[t][i]));
      }
      if (!whole || __ballot(most >= kInfBits)) {
        most = 0;
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) most = max(most, i <= top[t >> 1] - (jl + 16 * t) ? finite_bits(vs[t][i]) : 0u);
      }
      e2 = max(ve, (int)(groups_umax(most) >> 23) - 126);
      const float to = __builtin_amdgcn_ldexpf(1.f, -e2);
#pragma unroll
      for (int t = 0; t < KT; ++t) vs[t] *= to;
    }
    // The running maximum m only has to keep weights in range: it follows when a score passes it by
    // more than 8 (weights of up to 2^8), so that the sums are seldom scaled.
    float ms[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float mx = sc[0][u][0];
#pragma unroll
      for (int e = 1; e < 4 * KT; ++e) mx = max_of(mx, sc[e >> 2][u][e & 3]);
      mx = groups_max(mx) * mult[u];
      if (__ballot(mx > m[u] + 8.f) || (FMT != KV_SAME && e2 != ve)) {
        mx = fmaxf(m[u], mx);
        float al = exp2_hw(m[u] - (mx == -INFINITY ? 0.f : mx));
        m[u] = mx;
        l[u] *= al;
        lsum[u] *= al;
        al = __builtin_amdgcn_ldexpf(al, ve - e2);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) O[u][dt] *= al;
      }
      ms[u] = m[u] == -INFINITY ? 0.f : m[u];
    }
    ve = e2;
    __builtin_amdgcn_s_setprio(1);  // the other wavefront's vector work fits between these products
    f32x4 next[KT][U];
    if (kAhead) score(keys, step + 1, next);
    // weights, rounded to 16 bits once: their errors average out over the positions
    u32x4 pf[U][KT / 2];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float w[KT * 4];
#pragma unroll
      for (int e = 0; e < 4 * KT; ++e) w[e] = exp2_hw(fmaf(sc[e >> 2][u][e & 3], mult[u], -ms[u]));
      if (FMT != KV_SAME) {
#pragma unroll
        for (int e = 0; e < 4 * KT; ++e) {
          l[u] += w[e];
          w[e] *= vs[e >> 2][e & 3];
        }
        if (!full) {
#pragma unroll
          for (int e = 0; e < 4 * KT; ++e) w[e] = vis[u] >> e & 1u ? w[e] : 0.f;
        }
      }
#pragma unroll
      for (int h = 0; h < KT / 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) pf[u][h][i] = T::pack(w[8 * h + 2 * i], w[8 * h + 2 * i + 1]);
    }
    const uint32_t one = (uint32_t)T::from_f32(1.f) * 0x00010001u;
#pragma unroll
    for (int h = 0; h < KT / 2; ++h) {
      u32x4 sees[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        sees[u] = seen_keys<T>(vis[u] >> (8 * h));
        if (FMT == KV_SAME) lsum[u] = T::mfma(u32x4{one, one, one, one}, pf[u][h], lsum[u]);
      }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        u32x4 vf = *(const u32x4*)(values + lane * 16 + h * (kSide / 2) + dt * 1024);
        if (careful) {
          f32x4* const o[2] = {&O[0][dt], &O[1][dt]};
          take_nonfinite<T, U>(vf, sees, o);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) O[u][dt] = T::mfma(vf, pf[u][h], O[u][dt]);
      }
    }
    __builtin_amdgcn_s_setprio(0);
    if (kAhead) {
#pragma unroll
      for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int u = 0; u < U; ++u) sc[t][u] = next[t][u];
    }
  };

  auto walk = [&](auto again) {
    ve = -126;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      m[u] = -INFINITY;
      l[u] = 0.f;
      lsum[u] = f32x4{0.f, 0.f, 0.f, 0.f};
      seen[u] = 0;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) O[u][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    if (nsteps == 0) return;
    // before step 0: its keys and values are in LDS (kAhead: its scores known, the next keys on their way)
    Halves pg0 = halves(0), pg1{-1, -1};
    issue(keys0, values0, 0, pg0);
    commit(keys0, values0, 0);
    if (nsteps > 1) pg1 = halves(1);
    f32x4 sc[KT][U];
    if (kAhead) {
      __builtin_amdgcn_s_waitcnt(0);
      __syncthreads();
      if (nsteps > 1 && side == 0) issue(keys1, values1, 1, pg1);
      score(keys0, 0, sc);
    }
    // a step: behind its barrier its values and keys (kAhead: the next keys) are in LDS, and nobody
    // reads the other two buffers, which take the keys after those and the next values
    const int lead = kAhead && side == 0 ? 2 : 1;
    auto turn = [&](char* next_keys, char* keys, char* values, char* next_values, int step) {
      __builtin_amdgcn_s_waitcnt(0);
      __syncthreads();
      Halves pg2{-1, -1};
      if (step + 2 < nsteps) pg2 = halves(step + 2);
      char* const to = kAhead ? keys : next_keys;
      const bool more = step + lead < nsteps;
      if (more) issue(to, next_values, step + lead, lead == 2 ? pg2 : pg1);
      if (pg0.a < 0 || pg0.b < 0 || j0 + kManyKeys * (step + 1) > q.held) {
        blank(values, step, pg0);
        __syncthreads();
      }
      compute(kAhead ? next_keys : keys, values, step, pg0, sc, again);
      if (more) commit(to, next_values, step + lead);
      pg0 = pg1;
      pg1 = pg2;
    };
    for (int step = 0; step < nsteps; step += 2) {
      turn(keys1, keys0, values0, values1, step);
      if (step + 1 < nsteps) turn(keys0, keys1, values1, values0, step + 1);
    }
    __syncthreads();
  };
  walk(std::false_type{});
  if (FMT == KV_SAME) {
    bool odd = false;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) odd |= !(fabsf(O[u][dt][i]) < INFINITY);
    // the wavefronts share the buffers, so they walk again together
    if (threadIdx.x == 0) s_odd = 0;
    __syncthreads();
    if (__ballot(odd) && lane == 0) s_odd = 1;
    __syncthreads();
    if (s_odd) walk(std::true_type{});
  }

#pragma unroll
  for (int u = 0; u < U; ++u) {
    l[u] = FMT == KV_SAME ? lsum[u][0] : groups_sum(l[u]);
    if (m[u] == -INFINITY && groups_umax(seen[u]) != 0) l[u] = NAN;
    const int row = wrow + 16 * u + col;
    if (16 * u + col >= wrows) continue;
    const long long token = q.row + row / p.group;
    const int qhead = head * p.group + row % p.group;
    if (used == 1) {
      const float r = l[u] == 0.f ? 0.f : 1.f / l[u];
      uint16_t* out = (uint16_t*)p.out + token * p.ldo + qhead * D + 4 * g;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        f32x4 o = O[u][dt];
        if (FMT != KV_SAME) {
#pragma unroll
          for (int i = 0; i < 4; ++i) o[i] = __builtin_amdgcn_ldexpf(o[i], ve);
        }
        if (l[u] == 0.f) o = f32x4{0.f, 0.f, 0.f, 0.f};
        *(u32x2*)(out + 16 * dt) = u32x2{A::pack(o[0] * r, o[1] * r), A::pack(o[2] * r, o[3] * r)};
      }
    } else {
      const long long at = (token * p.heads + qhead) * p.splits + c;
      float* o_at = p.part + at * D + 4 * g;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        f32x4 o = O[u][dt];
        if (FMT != KV_SAME) {
#pragma unroll
          for (int i = 0; i < 4; ++i) o[i] = __builtin_amdgcn_ldexpf(o[i], ve);
        }
        *(f32x4*)(o_at + 16 * dt) = o;
      }
      if (g == 0) {
        float* ml = p.part + (long long)p.seqs.n_tokens * p.heads * p.splits * D + at * 2;
        ml[0] = m[u];
        ml[1] = l[u];
      }
    }
  }
}

// out = the joined partials of a token's rows, a workgroup to a token, 4 dimensions to a thread.
// Memory bounds it, and a chain of three round trips when there is little to join: the token's
// sequence, the shares' (m, l), their sums.  513 tokens of 32 heads of 128 in 3 shares: 9.0 us.
template <class A, int D>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedAttnParams p) {
  constexpr int kQuads = D / 4;
  const int token = blockIdx.x;
  int local;
  PagedSeq q;
  if (paged_find(p.seqs, p.kv.page_shift, token, 1, 0, 0, &local, &q) < 0) return;
  const int t = token - q.row;
  if (t < 0 || t >= q.done || (long long)q.n * p.group <= p.min_rows) return;
  const float* ml_all = p.part + (long long)p.seqs.n_tokens * p.heads * p.splits * D;
  for (int i = threadIdx.x; i < p.heads * kQuads; i += 256) {
    const int qhead = i / kQuads, d = i % kQuads * 4;
    // the tile's positions, as the kernel above shared them out
    const int tile0 = (t * p.group + qhead % p.group) >> kManyShift << kManyShift;
    const int rows = min(q.done * p.group - tile0, 1 << kManyShift);
    const int kend = max(min(q.held, q.first + (tile0 + rows - 1) / p.group + 1), 0);
    int used;
    many_share(kend, p.splits, &used);
    if (used == 1) continue;  // written already
    const long long at = ((long long)token * p.heads + qhead) * p.splits;
    u32x2 ml[kManyMaxSplits];
#pragma unroll
    for (int k = 0; k < kManyMaxSplits; ++k)
      ml[k] = k < used ? *(const u32x2*)(ml_all + (at + k) * 2) : u32x2{0xFF800000u, 0u};
    float M = -INFINITY, L = 0.f;
#pragma unroll
    for (int k = 0; k < kManyMaxSplits; ++k) M = fmaxf(M, as_float(ml[k][0]));
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k0 = 0; k0 < kManyMaxSplits; k0 += 4) {
      if (k0 >= used) break;
      f32x4 part[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (k0 + k < used) part[k] = *(const f32x4*)(p.part + (at + k0 + k) * D + d);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (k0 + k >= used) continue;
        const bool none = as_float(ml[k0 + k][0]) == -INFINITY;
        const float f = none ? 0.f : exp2_hw(as_float(ml[k0 + k][0]) - M), l = as_float(ml[k0 + k][1]);
        L += none ? (M == -INFINITY ? l : 0.f) : f * l;
        o += f * part[k];
      }
    }
    o = L == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : o / L;
    *(u32x2*)((uint16_t*)p.out + (long long)token * p.ldo + qhead * D + d) =
        u32x2{A::pack(o[0], o[1]), A::pack(o[2], o[3])};
  }
}

template <class A, int FMT, int D>
hipError_t few_t(PagedAttnParams p, bool wide, unsigned items, hipStream_t st) {
  const dim3 grid(items);
  if (wide) hipLaunchKernelGGL((paged_few_kernel<A, FMT, D, 2>), grid, dim3(64 * kFewWaves), 0, st, p);
  else hipLaunchKernelGGL((paged_few_kernel<A, FMT, D, 1>), grid, dim3(64 * kFewWaves), 0, st, p);
  return hipGetLastError();
}

template <class A>
hipError_t few_a(const PagedAttnParams& p, bool wide, unsigned items, hipStream_t st) {
  const bool d128 = p.kv.head_dim == 128;
  switch (p.kv.format) {
    case KV_SAME: return d128 ? few_t<A, KV_SAME, 128>(p, wide, items, st) : few_t<A, KV_SAME, 64>(p, wide, items, st);
    case KV_I8: return d128 ? few_t<A, KV_I8, 128>(p, wide, items, st) : few_t<A, KV_I8, 64>(p, wide, items, st);
  }
  return d128 ? few_t<A, KV_E4M3, 128>(p, wide, items, st) : few_t<A, KV_E4M3, 64>(p, wide, items, st);
}

template <class A, int FMT, int D>
hipError_t many_t(const PagedAttnParams& p, const dim3& grid, hipStream_t st) {
  hipLaunchKernelGGL((paged_many_kernel<A, FMT, D>), grid, dim3(64 * kManyWaves), 0, st, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  hipLaunchKernelGGL((paged_join_kernel<A, D>), dim3((unsigned)p.seqs.n_tokens), dim3(256), 0, st, p);
  return hipGetLastError();
}

template <class A>
hipError_t many_a(const PagedAttnParams& p, const dim3& grid, hipStream_t st) {
  const bool wide = p.kv.head_dim == 128;
  switch (p.kv.format) {
    case KV_SAME: return wide ? many_t<A, KV_SAME, 128>(p, grid, st) : many_t<A, KV_SAME, 64>(p, grid, st);
    case KV_I8: return wide ? many_t<A, KV_I8, 128>(p, grid, st) : many_t<A, KV_I8, 64>(p, grid, st);
  }
  return wide ? many_t<A, KV_E4M3, 128>(p, grid, st) : many_t<A, KV_E4M3, 64>(p, grid, st);
}

// A sequence's rows per key/value head (new tokens x heads of the group) up to which the kernel for few
// rows takes it.  16 sequences of 2500 positions, 8 heads of 128: at 36 rows 45 us (the other kernel
// 62), at 64 rows 44 (55), at 96 rows 64 (60); four sequences with a key head per query head: 48 rows
// 40 (50), 90 rows 59 (54).
constexpr int kFewRows = 64;

// How the kernel for few rows deals a batch: as many pieces as workgroups run at a time on 256
// CUs (their registers allow 2 to 4 on each), as far as the partials (kMaxPartials rows of all
// pieces) and the counters go.  Returns the number of workgroups.
constexpr long long kMaxPartials = 1 << 18;
long long few_splits(PagedAttnParams* p, long long tiles, bool wide, long long rows_each) {
  const long long cap = (long long)p->seqs.max_pages << p->kv.page_shift;
  const long long rows = (long long)p->seqs.n_tokens * p->heads;
  const int heads = p->kv.heads, n_seq = p->seqs.n_seq;
  p->tiles_each = (int)((rows_each + (wide ? 31 : 15)) / (wide ? 32 : 16));
  const long long counters = n_seq > kPagedDense ? tiles : (long long)n_seq * p->tiles_each * heads;
  const long long room = counters > kPagedCounters ? 1 : std::max<long long>(1, kMaxPartials / rows);
  p->want = 256 * (p->kv.head_dim == 128 ? (wide ? 2 : 3) : (wide ? 3 : 4));
  p->most = (int)std::min<long long>(room, kPagedMaxSplits);
  p->splits = paged_most_pieces(cap, heads, p->want, p->most);
  if (n_seq > kPagedDense) {
    p->splits = (int)std::min<long long>(p->splits, ((cap + 127) / 128 + kPagedMaxUnit - 1) / kPagedMaxUnit);
    return tiles * p->splits;
  }
  return heads * paged_most_items(cap, n_seq, p->tiles_each, heads, p->want, p->most);
}

// Workgroups that share a tile of the kernel for many rows: no more than kManyWorkgroups in all, as
// those run at a time, and four steps each at least.  The tiles are taken to be those of one
// sequence, with a token of each other one left to the kernel for few rows when that runs, too.  513
// tokens over 9217 positions, 32 heads on 8 (17 tiles of 8 heads): 3 shares 119 us, 4 144; 1024 tokens
// over 3000 beside 23 single ones, heads of 64, int8 (32 tiles): 1 share 95 us, 2 80.
int many_splits(const PagedCache& kv, const PagedSeqs& b, int heads, bool few) {
  const long long rows = (long long)std::max(1, b.n_tokens - (few ? b.n_seq - 1 : 0)) * (heads / kv.heads);
  const long long tiles = ((rows + (1 << kManyShift) - 1) >> kManyShift) * kv.heads;
  const long long cap = (long long)b.max_pages << kv.page_shift;
  const long long most = std::min<long long>(kManyMaxSplits, (cap + 4 * kManyKeys - 1) / (4 * kManyKeys));
  const long long room = kMaxManyPartials / ((long long)b.n_tokens * heads);
  return (int)std::max<long long>(1, std::min({most, room, kManyWorkgroups / tiles}));
}

}  // namespace

size_t paged_ws_bytes(const PagedCache& kv, const PagedSeqs& b, int heads) {
  const long long cap = (long long)b.max_pages << kv.page_shift;
  const long long chunks = std::min<long long>((cap + 127) / 128, kPagedMaxSplits);
  const long long rows = (long long)b.n_tokens * heads;
  const long long few = std::min(rows * chunks, kMaxPartials);
  const long long many = std::min(rows * kManyMaxSplits, kMaxManyPartials);
  return kPagedCounters * sizeof(uint32_t) + (size_t)std::max(few, many) * (kv.head_dim + 2) * sizeof(float);
}

hipError_t launch_paged_attention(PagedAttnParams p, double scale, void* ws, hipStream_t stream) {
  const PagedSeqs& b = p.seqs;
  if (b.n_tokens < 1 || b.n_seq < 1) return hipSuccess;
  p.group = p.heads / p.kv.heads;
  p.scale = (float)(scale * (double)kLog2e);
  p.cnt = (uint32_t*)ws;
  p.part = (float*)(p.cnt + kPagedCounters);
  // Rows of the longest sequence, and, if every row belongs to one, of the shortest: a batch of
  // short ones only or of long ones only takes one kernel.
  const long long longest = (long long)std::min(b.max_new, b.n_tokens) * p.group;
  const long long shortest = (b.n_tokens - (b.n_seq - 1LL) * b.max_new) * p.group;
  const bool many = longest > kFewRows, few = !many || shortest <= kFewRows;
  hipError_t e = hipSuccess;
  if (few) {
    // (beside a kernel for many rows it is single tokens, as a rule)
    const bool wide = (many ? p.group : longest) > 16;
    const long long tiles = paged_tiles(b, p.group, wide ? kFewShift<2> : kFewShift<1>, 1) * p.kv.heads;
    const unsigned items = (unsigned)few_splits(&p, tiles, wide, std::min(longest, (long long)kFewRows));
    p.min_rows = 0;
    p.max_rows = many ? kFewRows : 0x7FFFFFFF;
    e = p.kv.dtype == 1 ? few_a<BF16>(p, wide, items, stream) : few_a<F16>(p, wide, items, stream);
  }
  if (e == hipSuccess && many) {
    p.splits = many_splits(p.kv, b, p.heads, few);
    p.min_rows = few ? kFewRows : 0;
    const dim3 grid((unsigned)(paged_tiles(b, p.group, kManyShift, 1) * p.kv.heads), (unsigned)p.splits);
    e = p.kv.dtype == 1 ? many_a<BF16>(p, grid, stream) : many_a<F16>(p, grid, stream);
  }
  return e;
}

}  // namespace hg

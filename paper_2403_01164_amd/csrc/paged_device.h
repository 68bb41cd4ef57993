// Device helpers shared by the paged cache's kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "paged.h"

namespace hg {
namespace {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// The 16-bit types: conversions, and the 16x16x32 product of two operands of 8 elements a lane.
struct F16 {
  static constexpr uint32_t kExp = 0x7C007C00u;  // exponent bits of two packed values
  static constexpr uint32_t kExpLow = 0x04000400u;  // the lowest of them
  static __device__ __forceinline__ float to_f32(uint32_t h) { return (float)__builtin_bit_cast(_Float16, (uint16_t)h); }
  static __device__ __forceinline__ uint16_t from_f32(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    const f16x2 v = {(_Float16)a, (_Float16)b};
    return __builtin_bit_cast(uint32_t, v);
  }
  static __device__ __forceinline__ f32x4 mfma(const u32x4& a, const u32x4& b, const f32x4& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
};

struct BF16 {
  static constexpr uint32_t kExp = 0x7F807F80u;
  static constexpr uint32_t kExpLow = 0x00800080u;
  static __device__ __forceinline__ float to_f32(uint32_t h) { return __builtin_bit_cast(float, h << 16); }
  static __device__ __forceinline__ uint16_t from_f32(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    const bf16x2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, v);
  }
  static __device__ __forceinline__ f32x4 mfma(const u32x4& a, const u32x4& b, const f32x4& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};

template <class T>
__device__ __forceinline__ void unpack8(const u32x4& v, float* f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = T::to_f32(v[i] & 0xFFFFu);
    f[2 * i + 1] = T::to_f32(v[i] >> 16);
  }
}

// Loads through the global address space; pages are read once by a workgroup.
__device__ __forceinline__ u32x4 load16(const void* p) {
  return *(const __attribute__((address_space(1))) u32x4*)p;
}
__device__ __forceinline__ u32x4 load16_nt(const void* p) {
  return __builtin_nontemporal_load((const __attribute__((address_space(1))) u32x4*)p);
}
__device__ __forceinline__ int load_i32(const int32_t* p) { return *(const __attribute__((address_space(1))) int32_t*)p; }

// Largest and sum over the four lanes l % 16 + 16 g, in each of them: the two results of a swap
// of a register with itself are the lane's own value and its partner's.  (Elements of the result
// are copied out before they are reinterpreted: the compiler takes element 0 for any otherwise.)
template <class V, class F>
__device__ __forceinline__ V over_groups(V v, F op) {
  const auto a = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
  const uint32_t a0 = a[0], a1 = a[1];
  v = op(__builtin_bit_cast(V, a0), __builtin_bit_cast(V, a1));
  const auto b = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
  const uint32_t b0 = b[0], b1 = b[1];
  return op(__builtin_bit_cast(V, b0), __builtin_bit_cast(V, b1));
}
__device__ __forceinline__ float groups_max(float v) {
  return over_groups(v, [](float x, float y) { return fmaxf(x, y); });
}
__device__ __forceinline__ uint32_t groups_umax(uint32_t v) {
  return over_groups(v, [](uint32_t x, uint32_t y) { return x > y ? x : y; });
}
__device__ __forceinline__ float groups_sum(float v) {
  return over_groups(v, [](float x, float y) { return x + y; });
}

// Sum over the wavefront, in every lane (below 2^32).
__device__ __forceinline__ uint32_t wave_sum(uint32_t v) {
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, false);   // lane ^ 1
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, false);   // lane ^ 2
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, false);  // mirrored half row
  v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, false);  // mirrored row of 16
  return __builtin_amdgcn_readfirstlane(over_groups(v, [](uint32_t x, uint32_t y) { return x + y; }));
}

// Sum over the lanes up to this one.
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);  // from 1, 2, 4 and 8 lanes below, within 16
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);  // lane 15 of the row below, to rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);  // lane 31, to rows 2 and 3
  return v;
}

// Sequence of a tile (see paged_tile_base), the same in every lane of the wavefront: the last
// one whose tiles begin at or before it, or -1; *local the tile's number within it, *seq its
// rows and positions.  64 sequences at a time, in one round of loads.
__device__ __forceinline__ int paged_find(const PagedSeqs& b, int page_shift, int tile, int unit, int shift, int extra,
                                          int* local, PagedSeq* seq) {
  const int lane = threadIdx.x & 63;
  int s = -1, start = 0, end = 0, len = 0;
  for (int i0 = 0; i0 < b.n_seq; i0 += 64) {
    const int i = min(i0 + lane, b.n_seq - 1);
    const int st = load_i32(b.start + i), en = load_i32(b.start + i + 1), ln = load_i32(b.len + i);
    const bool before = i0 + lane < b.n_seq && paged_tile_base(st, i, b.n_tokens, unit, shift, extra) <= tile;
    const int c = __popcll(__ballot(before));
    if (c > 0) {
      s = i0 + c - 1;
      start = __builtin_amdgcn_readlane(st, c - 1);
      end = __builtin_amdgcn_readlane(en, c - 1);
      len = __builtin_amdgcn_readlane(ln, c - 1);
    }
    if (c < 64) break;
  }
  if (s < 0) return -1;
  *local = tile - paged_tile_base(start, s, b.n_tokens, unit, shift, extra);
  if (*local < 0) return -1;  // (only where new_start decreases)
  *seq = paged_seq(start, end, len, b, page_shift);
  return s;
}

// A table entry, -1 where it names no page, and the page of position j (j < held) of sequence s.
__device__ __forceinline__ int paged_entry(const PagedCache& kv, int p) { return p >= 0 && p < kv.n_pages ? p : -1; }
__device__ __forceinline__ int paged_page(const PagedSeqs& b, const PagedCache& kv, int s, int j) {
  return paged_entry(kv, load_i32(b.table + (size_t)s * b.max_pages + (j >> kv.page_shift)));
}

}  // namespace
}  // namespace hg

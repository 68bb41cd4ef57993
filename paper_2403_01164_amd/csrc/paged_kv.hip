// Writing a paged KV cache and reading it back, on gfx950.
//
// write, 16-bit: the row is stored as it is.  8-bit, for each token and head, keys and values
// apart: c = max_d |x_d| * (1 / Q) (Q = 127 for int8, 448 for e4m3; 1 / Q rounded to binary32),
// code_d = round(x_d / c), half to even, in binary32; c is kept as binary32.  A row of zeros has c = 0; a row that holds an
// infinity or a NaN has c infinite or NaN and codes 0, so that it reads back as NaN and the
// matrix products that multiply its codes with weights of 0 stay finite.
// read: code_d * c, rounded once to the 16-bit type (half to even).
//
// Both move every byte once, so memory bounds them (the launch, for single tokens): 65536 positions of
// 40 heads of 128, int8, written in 469 us (4.3 TB/s) and read in 466 (4.4; a large copy reaches 4.83),
// one token of 8 sequences, 16-bit, in 3.2 and 3.6.  A workgroup
// takes the 32 positions of one value tile (two key tiles) of one head: wavefronts 0 and 1 the
// keys, whose 16-byte pieces only change places, 2 and 3 the values, which pass through LDS to
// bring 8 positions of one dimension together.  Lane (position, group of 8 dimensions) holds
// D / 4 dimensions of its row, so the row's largest value takes two cross-lane steps.
#include "paged_device.h"

namespace hg {
namespace {

constexpr int kThreads = 256;
constexpr int kTile = 32;  // positions per workgroup

// One position's D / 4 dimensions of a lane, as 16-bit values.
template <int D>
struct Row {
  u32x4 x[D / 32];
};

template <class T, int FMT>
struct Quant {
  static constexpr float kMax = FMT == KV_I8 ? 127.f : 448.f;
  // 8 values / c -> 8 codes.  The quotients are rounded as a division rounds: y = x r with the
  // rounded reciprocal r, then y + (x - y c) r, the remainder exact (Markstein's correction), is the
  // rounded x / c as long as nothing underflows; a division for each bound the kernel (3711
  // tokens of 32 heads of 128 to int8: 29.4 us, now 24.5).  Scales out of that range are divided by.
  static __device__ __forceinline__ u32x2 codes(const u32x4& v, float c, float r) {
    float f[8];
    unpack8<T>(v, f);
    u32x2 w = {0u, 0u};
    if (!(c > 0.f) || !(c < INFINITY)) return w;
    if (c > 0x1p-60f && c < 0x1p60f) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float y = f[i] * r;
        f[i] = copysignf(fmaf(fmaf(-y, c, f[i]), r, y), f[i]);  // (the correction loses the sign of -0)
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = fminf(fmaxf(f[i] / c, -kMax), kMax);  // a subnormal c is short of bits
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float* q = f + 4 * h;
      if (FMT == KV_I8) {
        // 1.5 * 2^23 + q has the integer nearest to q, half to even, in its low bits
        uint32_t n[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) n[i] = __builtin_bit_cast(uint32_t, q[i] + 12582912.f);
        const uint32_t lo = __builtin_amdgcn_perm(n[1], n[0], 0x0C0C0400u), hi = __builtin_amdgcn_perm(n[3], n[2], 0x04000C0Cu);
        w[h] = lo | hi;
      } else {
        const int n = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
        w[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], n, true);
      }
    }
    return w;
  }
  // 8 codes * c -> 8 values
  static __device__ __forceinline__ u32x4 values(const u32x2& w, float c) {
    float f[8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (FMT == KV_I8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[4 * h + i] = (float)((int32_t)(w[h] << (24 - 8 * i)) >> 24) * c;
      } else {
        const auto a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w[h], 1.0f, false);
        const auto b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w[h], 1.0f, true);
        f[4 * h] = (float)a[0] * c;
        f[4 * h + 1] = (float)a[1] * c;
        f[4 * h + 2] = (float)b[0] * c;
        f[4 * h + 3] = (float)b[1] * c;
      }
    }
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = T::pack(f[2 * i], f[2 * i + 1]);
    return r;
  }
};

// The scale of a row from the 16-bit patterns: their magnitudes compare as integers, infinity
// above every number and NaN above infinity.
template <class T, int D, int FMT>
__device__ __forceinline__ float row_scale(const Row<D>& r) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t w = r.x[i][j] & 0x7FFF7FFFu;
      m = max(m, max(w & 0xFFFFu, w >> 16));
    }
  return T::to_f32(groups_umax(m)) * (1.f / Quant<T, FMT>::kMax);
}

// The 32 positions of a workgroup (see PagedTile), its position in the page and its record there
// (nullptr: the table names no page).
struct Tile {
  int row, lo, hi, off;
  char* rec;
};

__device__ __forceinline__ bool find_tile(const PagedCopyParams& p, int head, Tile* t) {
  int local;
  PagedSeq q;
  const int s = paged_find(p.seqs, p.kv.page_shift, blockIdx.x, 1, 5, 2, &local, &q);
  if (s < 0) return false;
  const PagedTile u = paged_tile(q, local);
  if (u.hi <= u.lo) return false;
  t->row = u.row;
  t->lo = u.lo;
  t->hi = u.hi;
  t->off = u.j0 & (p.kv.page_size - 1);
  // a tile lies in one page, and on one side of `held` unless the sequence ends in it
  const int page = u.j0 < q.held ? paged_page(p.seqs, p.kv, s, u.j0) : -1;
  t->rec = page < 0 ? nullptr : (char*)p.kv.pages + ((long long)page * p.kv.heads + head) * p.kv.record;
  return true;
}

template <class T, int FMT, int D>
__global__ __launch_bounds__(kThreads) void paged_write_kernel(PagedCopyParams p) {
  constexpr int ES = FMT == KV_SAME ? 2 : 1;
  constexpr int RS = D * ES + 16;  // LDS bytes per position
  __shared__ __align__(16) char lds[kTile * RS];
  const int head = blockIdx.y, lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Tile t;
  if (!find_tile(p, head, &t) || !t.rec) return;
  const bool values = wave >= 2;
  const int half = wave & 1, pos = lane & 15, g = lane >> 4, i = 16 * half + pos;
  const bool mine = i >= t.lo && i < t.hi;
  const long long P = p.kv.page_size;
  char* data = t.rec + (values ? P * D * ES : 0) + (long long)t.off * D * ES;  // the tile's positions
  Row<D> r;
  if (mine) {
    const uint16_t* src = (const uint16_t*)(values ? p.v : p.k) + (long long)(t.row + i) * p.ld + head * D + 8 * g;
#pragma unroll
    for (int k = 0; k < D / 32; ++k) r.x[k] = load16_nt(src + 32 * k);
  } else {
#pragma unroll
    for (int k = 0; k < D / 32; ++k) r.x[k] = u32x4{0u, 0u, 0u, 0u};
  }
  float c = 1.f, rc = 1.f;
  if (FMT != KV_SAME) {
    c = row_scale<T, D, FMT>(r);
    float* scales = (float*)(t.rec + 2 * P * D) + (values ? P : 0) + t.off;
    if (mine && g == 0) scales[i] = c;
    rc = 1.f / c;
  }
  if (!values) {
    char* dst = data + half * (16 * D * ES) + lane * 16;
    if (FMT == KV_SAME) {
#pragma unroll
      for (int k = 0; k < D / 32; ++k)
        if (mine) *(u32x4*)(dst + k * 1024) = r.x[k];
    } else {
#pragma unroll
      for (int k = 0; k < D / 64; ++k) {
        const u32x2 a = Quant<T, FMT>::codes(r.x[2 * k], c, rc), b = Quant<T, FMT>::codes(r.x[2 * k + 1], c, rc);
        if (mine) *(u32x4*)(dst + k * 1024) = u32x4{a[0], a[1], b[0], b[1]};
      }
    }
  } else {
#pragma unroll
    for (int k = 0; k < D / 32; ++k) {
      char* at = lds + i * RS + (32 * k + 8 * g) * ES;
      if (FMT == KV_SAME) *(u32x4*)at = r.x[k];
      else *(u32x2*)at = Quant<T, FMT>::codes(r.x[k], c, rc);
    }
  }
  __syncthreads();
  // values: 16 bytes of the tile a thread at a time, 8 positions of one dimension (or of two)
  char* vdata = t.rec + P * D * ES + (long long)t.off * D * ES;
  const bool whole = t.lo == 0 && t.hi == kTile;
  for (int u = threadIdx.x; u < kTile * D * ES / 16; u += kThreads) {
    const int l = u & 63, d0 = (u >> 6) * (16 * 2 / ES) + (l & 15), vg = l >> 4;
    if (FMT == KV_SAME) {
      uint16_t e[8];
#pragma unroll
      for (int x = 0; x < 8; ++x) e[x] = *(const uint16_t*)(lds + (16 * (x >> 2) + 4 * vg + (x & 3)) * RS + 2 * d0);
      if (whole) {
        u32x4 w;
#pragma unroll
        for (int x = 0; x < 4; ++x) w[x] = e[2 * x] | (uint32_t)e[2 * x + 1] << 16;
        *(u32x4*)(vdata + u * 16) = w;
      } else {
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          const int j = 16 * (x >> 2) + 4 * vg + (x & 3);
          if (j >= t.lo && j < t.hi) *(uint16_t*)(vdata + u * 16 + 2 * x) = e[x];
        }
      }
    } else {
      uint8_t e[16];
#pragma unroll
      for (int x = 0; x < 16; ++x)
        e[x] = *(const uint8_t*)(lds + (16 * ((x & 7) >> 2) + 4 * vg + (x & 3)) * RS + d0 + 16 * (x >> 3));
      if (whole) {
        u32x4 w;
#pragma unroll
        for (int x = 0; x < 4; ++x)
          w[x] = e[4 * x] | (uint32_t)e[4 * x + 1] << 8 | (uint32_t)e[4 * x + 2] << 16 | (uint32_t)e[4 * x + 3] << 24;
        *(u32x4*)(vdata + u * 16) = w;
      } else {
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          const int j = 16 * ((x & 7) >> 2) + 4 * vg + (x & 3);
          if (j >= t.lo && j < t.hi) *(uint8_t*)(vdata + u * 16 + x) = e[x];
        }
      }
    }
  }
}

template <class T, int FMT, int D>
__global__ __launch_bounds__(kThreads) void paged_read_kernel(PagedCopyParams p) {
  constexpr int ES = FMT == KV_SAME ? 2 : 1;
  constexpr int RS = D * ES + 16;
  __shared__ __align__(16) char lds[kTile * RS];
  const int head = blockIdx.y, lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Tile t;
  if (!find_tile(p, head, &t)) return;
  const bool values = wave >= 2;
  const int half = wave & 1, pos = lane & 15, g = lane >> 4, i = 16 * half + pos;
  const bool mine = i >= t.lo && i < t.hi;
  const long long P = p.kv.page_size;
  constexpr int kLoads = D * ES / 64;                    // of a position's keys
  constexpr int kChunks = kTile * D * ES / 16 / kThreads;  // of the tile's values, per thread
  static_assert(kChunks * kThreads * 16 == kTile * D * ES || D * ES == 64, "values");
  u32x4 kw[kLoads], vw[kChunks > 0 ? kChunks : 1];
  float c = 1.f;
  if (t.rec) {
    // everything that the tile needs is requested at once
    const char* kdata = t.rec + (long long)t.off * D * ES + half * (16 * D * ES) + lane * 16;
    const char* vdata = t.rec + P * D * ES + (long long)t.off * D * ES;
#pragma unroll
    for (int k = 0; k < kLoads; ++k)
      if (!values) kw[k] = load16_nt(kdata + k * 1024);
    if (FMT != KV_SAME) c = ((const float*)(t.rec + 2 * P * D) + (values ? P : 0) + t.off)[i];
#pragma unroll
    for (int n = 0; n < (kChunks > 0 ? kChunks : 1); ++n) {
      const int u = threadIdx.x + n * kThreads;
      if (u < kTile * D * ES / 16) vw[n] = load16_nt(vdata + u * 16);
    }
#pragma unroll
    for (int n = 0; n < (kChunks > 0 ? kChunks : 1); ++n) {
      const int u = threadIdx.x + n * kThreads;
      if (u >= kTile * D * ES / 16) continue;
      const int l = u & 63, d0 = (u >> 6) * (16 * 2 / ES) + (l & 15), vg = l >> 4;
      const u32x4 w = vw[n];
      if (FMT == KV_SAME) {
#pragma unroll
        for (int x = 0; x < 8; ++x)
          *(uint16_t*)(lds + (16 * (x >> 2) + 4 * vg + (x & 3)) * RS + 2 * d0) = (uint16_t)(w[x >> 1] >> (16 * (x & 1)));
      } else {
#pragma unroll
        for (int x = 0; x < 16; ++x)
          *(uint8_t*)(lds + (16 * ((x & 7) >> 2) + 4 * vg + (x & 3)) * RS + d0 + 16 * (x >> 3)) =
              (uint8_t)(w[x >> 2] >> (8 * (x & 3)));
      }
    }
  }
  __syncthreads();
  if (!mine) return;
  uint16_t* dst = (uint16_t*)(values ? p.v : p.k) + (long long)(t.row + i) * p.ld + head * D + 8 * g;
#pragma unroll
  for (int k = 0; k < D / 32; ++k) {
    u32x4 x = {0u, 0u, 0u, 0u};
    if (t.rec) {
      if (FMT == KV_SAME) {
        x = values ? *(const u32x4*)(lds + i * RS + (32 * k + 8 * g) * ES) : kw[k];
      } else {
        const u32x4& w = kw[k >> 1];
        x = Quant<T, FMT>::values(values ? *(const u32x2*)(lds + i * RS + 32 * k + 8 * g)
                                         : u32x2{w[2 * (k & 1)], w[2 * (k & 1) + 1]}, c);
      }
    }
    *(u32x4*)(dst + 32 * k) = x;
  }
}

template <class T, int FMT, int D>
hipError_t copy_t(const PagedCopyParams& p, bool write, const dim3& grid, hipStream_t st) {
  if (write) hipLaunchKernelGGL((paged_write_kernel<T, FMT, D>), grid, dim3(kThreads), 0, st, p);
  else hipLaunchKernelGGL((paged_read_kernel<T, FMT, D>), grid, dim3(kThreads), 0, st, p);
  return hipGetLastError();
}

template <class T>
hipError_t copy_f(const PagedCopyParams& p, bool write, hipStream_t st) {
  const dim3 grid((unsigned)paged_tiles(p.seqs, 1, 5, 2), p.kv.heads);
  const bool wide = p.kv.head_dim == 128;
  switch (p.kv.format) {
    case KV_SAME: return wide ? copy_t<T, KV_SAME, 128>(p, write, grid, st) : copy_t<T, KV_SAME, 64>(p, write, grid, st);
    case KV_I8: return wide ? copy_t<T, KV_I8, 128>(p, write, grid, st) : copy_t<T, KV_I8, 64>(p, write, grid, st);
  }
  return wide ? copy_t<T, KV_E4M3, 128>(p, write, grid, st) : copy_t<T, KV_E4M3, 64>(p, write, grid, st);
}

hipError_t copy(const PagedCopyParams& p, bool write, hipStream_t st) {
  if (p.seqs.n_tokens < 1 || p.seqs.n_seq < 1) return hipSuccess;
  return p.kv.dtype == 1 ? copy_f<BF16>(p, write, st) : copy_f<F16>(p, write, st);
}

}  // namespace

hipError_t launch_paged_write(const PagedCopyParams& p, hipStream_t stream) { return copy(p, true, stream); }
hipError_t launch_paged_read(const PagedCopyParams& p, hipStream_t stream) { return copy(p, false, stream); }

}  // namespace hg

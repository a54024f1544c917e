// The 8-bit paged KV cache: what its kernels and its host side share.
//
// A tile is 32 slots of one page and KV head: 32 * dh bytes of keys laid out
// [dh / 16][32 slots][16 dims] and 32 * dh bytes of values laid out
// [dh][32 slots], e4m3, and one exponent each; a stored x stands for
// x * 2^exponent.  In both layouts a wave's 16 bytes per lane are one
// contiguous 1 KB piece of the tile and the operand of the matrix cores that
// the attention needs, without a transpose.  Tile t of a sequence is tile
// t % tpp of page table[b][t / tpp]; tiles of a pool are numbered
// (page * Hkv + head) * tpp + tile.
//
// The exponents are powers of two and not general scales, so that the tile's
// earlier numbers stay exact when a later token raises the exponent (only
// what falls below the smallest subnormal's half step is lost), and so that
// applying one is an exponent of a conversion or of a score's factor.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_common.h"

namespace griffin {

constexpr int PAGED_E_MIN = -110;  // exponent of a tile of zeros; 2^(E_MIN - 9) is a normal fp32

// bits of the optional status word
enum PagedStatus : int { PAGED_BAD_PAGE = 1, PAGED_BAD_LENGTH = 2, PAGED_BAD_ROW = 4 };

enum PagedType : int { PT_BF16 = 0, PT_F16 = 1, PT_F32 = 2 };

struct PagedPool {
  uint8_t *k, *v;      // e4m3 tiles
  int8_t *ke, *ve;     // exponents, one per tile
  int n_pages, tpp, Hkv, dh;
};

struct PagedTable {
  const int32_t* pages;  // [batch][stride]
  int stride, cols;
  const int32_t* lengths;  // [batch] cached slots
  int most;                // the longest that a length may be
};

struct PagedRows {       // [batch][rows][heads][dh], unit stride in dh
  const void* p;
  long long sb, sr, sh;  // strides of sequence, row and head, in elements
  int vec;               // 1: every 8 consecutive values are aligned to their size (16 or 32 bytes)
};

struct PagedAppend {
  PagedPool pool;
  PagedTable tab;
  const int32_t* counts;  // [batch] or null: max_new each
  int counts_stride, counts_add;  // count of sequence b: counts[b * stride] + add
  const int32_t* path;    // [batch][path_stride] source rows, or null: row j
  int path_stride;
  int path_first;         // 1: the first appended row is row 0 and path gives the ones after it
  PagedRows k, v;
  int dtype, batch, rows, max_new;
  int rotate;
  double inv_rev[64];     // rotary frequencies in revolutions per position: base^(-2i/dh) / (2 pi)
  int layers;             // the same append for several layers:
  long long pool_layer;   // tiles between two layers' pools
  long long rows_layer;   // elements between two layers' source rows
  int heads_per_wg;
  int32_t* status;
};
hipError_t launch_paged_append(PagedAppend a, hipStream_t s);

// Workgroups of a launch at most: 2^32 threads of 512 each, and room for rounding
// up.
constexpr long long PAGED_MAX_GROUPS = 1 << 22;

// Work cut of an attention call.  The cached tiles that some node of a sequence
// sees are dealt to units, numbered sequence by sequence (unit_at); each unit is
// one partial result per row, joined by paged_combine_kernel.
struct PagedCut {
  int window, sinks;
  int target;  // units wanted in all: workgroups that fit the chip at once
  int least;   // tiles per unit at least
  int full;    // tiles per unit from which on all of the target is used
};

struct PagedAttn {
  PagedPool pool;
  PagedTable tab;
  const int32_t* counts;  // [batch] or null: nodes each
  const uint64_t* anc;    // [batch][nodes], or null: a chain
  PagedRows q, q_lo, k, v;  // q_lo: low parts of a split bf16 q, or p null
  void* out;              // [batch][nodes][Hq][dh], strides below; packed: see out_ks
  long long ob, orow, oh;
  int out_vec;
  int out_ks;             // > 0: out is the split bf16 packed operand of a projection (xpack_off), out_ks K steps
  int dtype, batch, nodes, Hq;
  int stride;             // nodes of a sequence in anc and in the packed operand, >= nodes
  float scale_log2;       // log2(e) * scale
  PagedCut cut;
  int units;              // upper bound of the units (grid)
  float* part_o;          // [units][Hkv][G * nodes][dh]
  float* part_ml;         // [units][Hkv][G * nodes][2]
  int2* first_unit;       // [batch] first unit and units of a sequence that has any
  // the kernel (paged_plan).  thin: row tiles of 16, fused: whole sequences, nothing to join; else
  // wide: waves of a workgroup of the wide kernel, or 0
  int thin, fused, wide;
  int32_t* status;
};
hipError_t launch_paged_attention(const PagedAttn& a, hipStream_t s);
hipError_t launch_paged_thin(const PagedAttn& a, hipStream_t s);

// Shape of the call, from host values alone: fills a.cut, a.units and the
// workgroup's shape.  Not 0: too many tiles.
int paged_plan(PagedAttn& a, int max_length);
// Lays the call's workspace out at `base` and returns its bytes.
size_t paged_workspace(PagedAttn& a, void* base);

// ------------------------------------------------------------- device helpers

__device__ __forceinline__ float pow2i(int e) {  // 2^e, e clamped to the normal range
  return __uint_as_float((uint32_t)(min(max(e, -126), 127) + 127) << 23);
}

// 8 consecutive 16-bit values
__device__ __forceinline__ u32x4 load8_raw(const void* p, long long at, int vec) {
  const uint16_t* h = static_cast<const uint16_t*>(p) + at;
  if (vec) return ld_u4(h);
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = h[2 * i] | (uint32_t)h[2 * i + 1] << 16;
  return w;
}

// 8 consecutive values as fp32
__device__ __forceinline__ void load8(const void* p, long long at, int dtype, int vec, float (&x)[8]) {
  if (dtype == PT_F32) {
    const float* f = static_cast<const float*>(p) + at;
    if (vec) {
      const float4 a = *reinterpret_cast<const float4*>(f), b = *reinterpret_cast<const float4*>(f + 4);
      x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = f[i];
    }
    return;
  }
  const u32x4 w = load8_raw(p, at, vec);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint16_t u = w[i / 2] >> (16 * (i & 1));
    x[i] = dtype == PT_BF16 ? bf16_to_f32(u) : (float)__builtin_bit_cast(_Float16, u);
  }
}

// 4 consecutive values: as they are, and as fp32
template <int DT>
struct QuadOf {
  typedef uint2 type;
};
template <>
struct QuadOf<PT_F32> {
  typedef float4 type;
};
template <int DT>
__device__ __forceinline__ typename QuadOf<DT>::type load_quad(const void* p, long long at, int vec) {
  if constexpr (DT == PT_F32) {
    const float* f = static_cast<const float*>(p) + at;
    if (vec) return *reinterpret_cast<const float4*>(f);
    return make_float4(f[0], f[1], f[2], f[3]);
  } else {
    const uint16_t* h = static_cast<const uint16_t*>(p) + at;
    if (vec) return *reinterpret_cast<const uint2*>(h);
    return make_uint2(h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16);
  }
}
template <int DT>
__device__ __forceinline__ float4 quad_f32(const typename QuadOf<DT>::type& w) {
  if constexpr (DT == PT_F32) {
    return w;
  } else if constexpr (DT == PT_BF16) {
    return make_float4(bf16_to_f32(w.x & 0xffff), bf16_to_f32(w.x >> 16), bf16_to_f32(w.y & 0xffff), bf16_to_f32(w.y >> 16));
  } else {
    auto f = [](uint32_t u) { return (float)__builtin_bit_cast(_Float16, (uint16_t)u); };
    return make_float4(f(w.x), f(w.x >> 16), f(w.y), f(w.y >> 16));
  }
}
}  // namespace griffin

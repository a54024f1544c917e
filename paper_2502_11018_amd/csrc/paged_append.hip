// Appending keys and values to the 8-bit paged cache (paged.h).
//
// New row j of sequence b goes to slot s = length_b + j.  Its key is rotated
// by the angle of position s on the way (k_i cos - k_{i+dh/2} sin, k_{i+dh/2}
// cos + k_i sin; the angle in fp64, reduced to a fraction of a turn there, its
// sine and cosine in fp32).  A tile's exponent is the smallest e with |x| <=
// 448 * 2^e for all its new finite values, and not below the one that its
// earlier slots have; where it rises those are rounded again.  The numbers are
// rounded to e4m3 once, to nearest even, from fp32; an infinity becomes the
// largest number, a NaN stays one.
//
// A workgroup owns a tile (every slot of it that this call writes or rounds
// again) for some heads, one after the other, so that no two workgroups write
// one tile and the 32 * dh / 2 sines are computed once for all its heads.
// Later slots of the tile keep their bytes.
//
// What bounds it: 30011 tokens of 8 heads of 128 in bf16 move 184 MB in 45 us,
// 4.1 TB/s, where a large copy moves 4.85.  With a slot's keys across a wave's
// lanes (32 rows a load) and 4-byte stores of the values it took 54 us, with
// three instead of four waves per SIMD 52; loads of the next head ahead of this
// one's stores gained nothing beside four waves.

#include <algorithm>
#include <type_traits>

#include "paged.h"

namespace griffin {

namespace {

// Smallest e with amax <= 448 * 2^e (448 = 1.75 * 2^8), at least PAGED_E_MIN.
__device__ __forceinline__ int exponent_for(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffff) > 0x600000 ? 1 : 0);
  return max(e, PAGED_E_MIN);  // subnormal and zero: far below
}

__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a <= 3.402823466e38f ? a : 0.f;
}

// The conversion to e4m3 turns what is above 448 into a NaN.  Finite numbers
// are within it by their tile's exponent; infinities are clamped where a tile
// has any (a NaN passes).
template <bool INF>
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  auto sat = [](float x) { return !INF ? x : x > 448.f ? 448.f : x < -448.f ? -448.f : x; };
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(sat(a), sat(b), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(sat(c), sat(d), lo, true);
}

__device__ __forceinline__ uint32_t rescale_e4m3(uint32_t w, float f) {
  return pack_e4m3<false>(__builtin_amdgcn_cvt_f32_fp8(w, 0) * f, __builtin_amdgcn_cvt_f32_fp8(w, 1) * f,
                          __builtin_amdgcn_cvt_f32_fp8(w, 2) * f, __builtin_amdgcn_cvt_f32_fp8(w, 3) * f);
}

// What a thread reads of one head.
template <int DT>
struct HeadRows {
  typedef typename QuadOf<DT>::type Quad;
  Quad k[4], v[4];
};

// Bytes of a word for the lowest 4 bits of `b`.
__device__ __forceinline__ uint32_t byte_mask(uint32_t b) { return ((b & 15) * 0x00204081u & 0x01010101u) * 0xffu; }

// Threads: DH * 2.  Reading, a wave's lanes lie along the dims of a few rows.
// Keys: thread t has slot t / (DH / 16) and of it the dims 8 j .. and DH / 2 + 8
// j .., j = t % (DH / 16), which are rotated together.  Values: slots 4 vg ..,
// dims 4 vd .., (vg, vd) = (t / (DH / 4), t % (DH / 4)); they go to their tile
// through LDS, from which thread t takes 16 slots of dim t / 2.
template <int DH, int DT>
__global__ __launch_bounds__(DH * 2, 4) void paged_append_kernel(PagedAppend a) {
  constexpr int NT = DH * 2, NW = NT / 64, HALF = DH / 2, ROW = 9;  // words of a dim in LDS, one of padding
  typedef typename QuadOf<DT>::type Quad;
  __shared__ float red[2][2][NW];
  __shared__ uint32_t turn[DH * ROW];
  const int t = threadIdx.x;
  const int groups = (a.pool.Hkv + a.heads_per_wg - 1) / a.heads_per_wg;
  const int tiles_max = (a.max_new + 31) / 32 + 1;
  int id = blockIdx.x;
  const int g = id % groups;
  id /= groups;
  const int tl = id % tiles_max;
  id /= tiles_max;
  const int b = id % a.batch, layer = id / a.batch;

  const int len = a.tab.lengths[b];
  int n = a.counts ? a.counts[(long long)b * a.counts_stride] + a.counts_add : a.max_new;
  const bool odd = len < 0 || n < 0 || n > a.max_new || (long long)len + n > a.tab.most;
  if (odd) {  // nothing of such a sequence is written
    if (a.status && t == 0) atomicOr(a.status, PAGED_BAD_LENGTH);
    return;
  }
  const int tile = len / 32 + tl;
  const int s0 = tile * 32;
  if (n == 0 || s0 >= len + n) return;
  const int page = a.tab.pages[(long long)b * a.tab.stride + tile / a.pool.tpp];
  const int h0 = g * a.heads_per_wg, h1 = min(h0 + a.heads_per_wg, a.pool.Hkv);

  // source row of a slot: -1 none (an earlier or a later slot), -2 out of range
  auto row_of = [&](int slot) -> int {
    const int j = slot - len;
    if (j < 0 || j >= n) return -1;
    if (!a.path) return j;
    if (a.path_first && j == 0) return 0;
    const int r = a.path[(long long)b * a.path_stride + j - a.path_first];
    return r >= 0 && r < a.rows ? r : -2;
  };
  const int slot = s0 + t / (DH / 16), j = t % (DH / 16);
  const int krow = row_of(slot);
  const int vg = t / (DH / 4), vd = t % (DH / 4);
  int vrow[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) vrow[i] = row_of(s0 + 4 * vg + i);
  const long long kb = layer * a.rows_layer + b * a.k.sb + 8 * j, vb = layer * a.rows_layer + b * a.v.sb + 4 * vd;
  auto read = [&](int h, HeadRows<DT>& r) {
#pragma unroll
    for (int i = 0; i < 4; ++i) r.k[i] = r.v[i] = Quad{};
    if (krow >= 0) {
      const long long at = kb + krow * a.k.sr + h * a.k.sh;
#pragma unroll
      for (int i = 0; i < 4; ++i) r.k[i] = load_quad<DT>(a.k.p, at + (i / 2) * HALF + 4 * (i % 2), a.k.vec);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (vrow[i] >= 0) r.v[i] = load_quad<DT>(a.v.p, vb + vrow[i] * a.v.sr + h * a.v.sh, a.v.vec);
  };
  HeadRows<DT> now;
  read(h0, now);  // asked for before the page is known
  // the tile's slots that get a row, and its earlier ones
  const int lrow = row_of(s0 + t % 32);
  const uint32_t fresh = (uint32_t)__ballot(lrow >= 0 && t % 64 < 32);
  const uint32_t older = s0 >= len ? 0u : len - s0 >= 32 ? ~0u : (1u << (len - s0)) - 1;
  if (a.status && lrow == -2) atomicOr(a.status, PAGED_BAD_ROW);
  if (page < 0 || page >= a.pool.n_pages) {  // uniform
    if (a.status && t == 0) atomicOr(a.status, PAGED_BAD_PAGE);
    return;
  }
  const long long tile0 = layer * a.pool_layer + (long long)page * a.pool.Hkv * a.pool.tpp + tile % a.pool.tpp;

  float cs[8], sn[8];
  if (a.rotate) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      double rev = slot * a.inv_rev[8 * j + i];
      rev -= rint(rev);
      sincospif(2.f * (float)rev, &sn[i], &cs[i]);
    }
  }
  for (int h = h0; h < h1; ++h) {
    if (h > h0) read(h, now);
    const long long ti = tile0 + (long long)h * a.pool.tpp;
    int ke = PAGED_E_MIN, ve = PAGED_E_MIN;
    if (older) ke = a.pool.ke[ti], ve = a.pool.ve[ti];
    float x[8], y[8], z[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 k = quad_f32<DT>(now.k[i]), v = quad_f32<DT>(now.v[i]);
      float* d = i < 2 ? x + 4 * i : y + 4 * (i - 2);
      d[0] = k.x, d[1] = k.y, d[2] = k.z, d[3] = k.w;
      z[i][0] = v.x, z[i][1] = v.y, z[i][2] = v.z, z[i][3] = v.w;
    }
    if (a.rotate) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float u = x[i], w = y[i];
        x[i] = u * cs[i] - w * sn[i];
        y[i] = w * cs[i] + u * sn[i];
      }
    }
    float mk = 0.f, mv = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) mk = fmaxf(mk, fmaxf(fabsf(x[i]), fabsf(y[i])));
#pragma unroll
    for (int i = 0; i < 16; ++i) mv = fmaxf(mv, fabsf(z[i / 4][i % 4]));
    // the workgroup's maxima; two sets, so that the next head's do not meet
    // this one's readers
    auto meet = [&](int set) {
      float(&rd)[2][NW] = red[set];
      mk = wave_max(mk), mv = wave_max(mv);
      if ((t & 63) == 0) rd[0][t >> 6] = mk, rd[1][t >> 6] = mv;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < NW; ++i) mk = fmaxf(mk, rd[0][i]), mv = fmaxf(mv, rd[1][i]);
    };
    meet(h & 1);
    const bool inf = mk == INFINITY || mv == INFINITY;  // uniform; rare
    if (inf) {
      mk = mv = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) mk = fmaxf(mk, fmaxf(finite_abs(x[i]), finite_abs(y[i])));
#pragma unroll
      for (int i = 0; i < 16; ++i) mv = fmaxf(mv, finite_abs(z[i / 4][i % 4]));
      __syncthreads();
      meet(h & 1);
      __syncthreads();
    }
    const int ken = max(ke, exponent_for(mk)), ven = max(ve, exponent_for(mv));
    uint8_t* kt = a.pool.k + ti * 32 * DH;
    uint8_t* vt = a.pool.v + ti * 32 * DH;
    auto put = [&](auto infinities) {
      constexpr bool INF = decltype(infinities)::value;
      // keys: [DH / 16][32][16]
      uint2* k0 = reinterpret_cast<uint2*>(kt + (j / 2 * 32 + slot - s0) * 16 + 8 * (j % 2));
      uint2* k1 = reinterpret_cast<uint2*>(kt + ((j / 2 + DH / 32) * 32 + slot - s0) * 16 + 8 * (j % 2));
      if (krow >= 0) {
        const float f = pow2i(-ken);
        auto four = [&](const float* d) { return pack_e4m3<INF>(d[0] * f, d[1] * f, d[2] * f, d[3] * f); };
        *k0 = make_uint2(four(x), four(x + 4));
        *k1 = make_uint2(four(y), four(y + 4));
      } else if (slot < len && ken > ke) {
        const float f = pow2i(ke - ken);
        const uint2 u = *k0, w = *k1;
        *k0 = make_uint2(rescale_e4m3(u.x, f), rescale_e4m3(u.y, f));
        *k1 = make_uint2(rescale_e4m3(w.x, f), rescale_e4m3(w.y, f));
      }
      // values: words of 4 slots of a dim
      const float f = pow2i(-ven);
#pragma unroll
      for (int d = 0; d < 4; ++d)
        turn[(4 * vd + d) * ROW + vg] = pack_e4m3<INF>(z[0][d] * f, z[1][d] * f, z[2][d] * f, z[3][d] * f);
    };
    if (inf) put(std::true_type{});
    else put(std::false_type{});
    __syncthreads();
    // .. and 16 slots of a dim, [DH][32]
    {
      const int half = t % 2;
      uint4* w = reinterpret_cast<uint4*>(vt + t / 2 * 32 + 16 * half);
      uint32_t u[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) u[i] = turn[t / 2 * ROW + 4 * half + i];
      const uint32_t fh = fresh >> (16 * half) & 0xffff, oh = older >> (16 * half) & 0xffff;
      if (fh == 0xffff) {
        *w = make_uint4(u[0], u[1], u[2], u[3]);
      } else if (fh || (oh && ven > ve)) {
        const uint4 was4 = *w;
        const uint32_t was[4] = {was4.x, was4.y, was4.z, was4.w};
        const float f_old = pow2i(ve - ven);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t mine = byte_mask(fh >> (4 * i)), old = byte_mask(oh >> (4 * i));
          const uint32_t kept = ven > ve ? (was[i] & ~old) | (rescale_e4m3(was[i], f_old) & old) : was[i];
          u[i] = (u[i] & mine) | (kept & ~mine);
        }
        *w = make_uint4(u[0], u[1], u[2], u[3]);
      }
    }
    if (t == 0) a.pool.ke[ti] = (int8_t)ken, a.pool.ve[ti] = (int8_t)ven;
  }
}

template <int DH>
void launch_dh(const PagedAppend& a, unsigned grid, hipStream_t s) {
  if (a.dtype == PT_F32) hipLaunchKernelGGL((paged_append_kernel<DH, PT_F32>), dim3(grid), dim3(DH * 2), 0, s, a);
  else if (a.dtype == PT_F16) hipLaunchKernelGGL((paged_append_kernel<DH, PT_F16>), dim3(grid), dim3(DH * 2), 0, s, a);
  else hipLaunchKernelGGL((paged_append_kernel<DH, PT_BF16>), dim3(grid), dim3(DH * 2), 0, s, a);
}

}  // namespace

hipError_t launch_paged_append(PagedAppend a, hipStream_t s) {
  const long long tiles = (long long)a.layers * a.batch * ((a.max_new + 31) / 32 + 1);
  // One head per workgroup until there are enough of them, then two, four ..,
  // which share the tile's sines (30011 tokens: 69 us with one head each, 45
  // with four).
  a.heads_per_wg = 1;
  while (a.heads_per_wg < a.pool.Hkv && tiles * a.pool.Hkv / (2 * a.heads_per_wg) >= 1024) a.heads_per_wg *= 2;
  const long long grid = tiles * ((a.pool.Hkv + a.heads_per_wg - 1) / a.heads_per_wg);
  if (grid > 0x7fffffffLL) return hipErrorInvalidValue;
  if (a.pool.dh == 128) launch_dh<128>(a, (unsigned)grid, s);
  else if (a.pool.dh == 64) launch_dh<64>(a, (unsigned)grid, s);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace griffin

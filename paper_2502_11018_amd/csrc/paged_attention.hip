// Attention of draft-tree nodes over the 8-bit paged cache (paged.h).
//
// Node i of sequence b (bits anc[i]; a chain: nodes 0 .. i) stands at position
// p = length + |anc[i] without i|.  It sees the cached slots s < length with
// window == 0, p - s < window or s < sinks, and the nodes of anc[i], the r-th
// of which stands at position length + r, by the same window.
//
// paged_attention_kernel computes the cached part in units: some of the tiles
// of one sequence, a KV head, and 32 rows of the head group (row = head * N +
// node).  Its four waves take every fourth tile each and meet in LDS at the
// end.  Per tile a wave loads 16 bytes a lane and piece, which are the matrix
// operands as they stand, and computes S^T = K Q^T and O^T += V^T P^T with
// v_mfma_f32_32x32x16_f16, so that a lane owns a query row and the softmax is
// lane-local:
//  * e4m3 is exact in fp16.  Keys are converted as they are, their tile's
//    exponent goes into the score's factor; values are converted relative to
//    the largest exponent the wave has met (E), which is uniform over the wave
//    and rarely rises; the accumulators follow it when it does.
//  * Keys meet the matrix cores in a permuted row order, so that accumulator
//    register r of lane half h holds slot 16 h + r: the P operand is the lane's
//    own registers and the V operand 16 consecutive slots of a dim.
//  * q is scaled by a power of two per row to fill fp16 (exact for bf16 and
//    fp16 inputs); fp32 inputs enter as high and low parts (22 bits), and so
//    do their probabilities.  The others' probabilities are rounded to fp16,
//    2^-12 relative: an eighth of the rounding of a bf16 output.
//  * The maximum that the probabilities refer to follows the scores only where
//    a lane's sum of a tile passes 2^14 (fp16 ends at 65504), so no maximum is
//    formed for most tiles.
//
// paged_combine_kernel joins a row's units in their order, adds the nodes of
// its own root path in fp32, and writes the row.

#include <algorithm>

#include "griffin_internal.h"
#include "paged.h"

namespace griffin {

namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// The cached tiles that some node of a sequence of `len` slots sees: the first
// `sink` ones, then those from `lo` on; n in all.
struct SeqTiles {
  int n, sink, lo;
};
__host__ __device__ inline SeqTiles seq_tiles(int len, const PagedCut& c) {
  const int all = (int)(((long long)len + 31) >> 5);
  if (c.window == 0) return {all, 0, 0};
  const int lo = max(0, len - c.window + 1) >> 5;  // the root's window starts first
  const int sink = min((int)(((long long)c.sinks + 31) >> 5), lo);
  return {sink + all - lo, sink, lo};
}

// A sequence's length as the kernels use it: 0 where it is out of range.
__device__ __forceinline__ int checked_len(const PagedTable& t, int b, bool* bad) {
  const int len = t.lengths[b];
  const bool ok = len >= 0 && len <= t.most;
  if (!ok) *bad = true;
  return ok ? len : 0;
}

// Tiles per unit: the same for every workgroup of both kernels (whole waves
// call these).
__device__ int tiles_per_unit(const PagedAttn& a) {
  const int lane = threadIdx.x & 63;
  long long total = 0;
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    bool bad = false;
    const int b = b0 + lane;
    int n = b < a.batch ? seq_tiles(checked_len(a.tab, b, &bad), a.cut).n : 0;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o, 64);
    total += n;
  }
  const long long per = (total + a.cut.target - 1) / a.cut.target;
  return (int)max((long long)a.cut.least, per);
}

// First unit of sequence `b` and the sequence's units.
struct Units {
  int first, n;
};
__device__ Units units_of(const PagedAttn& a, int per, int b) {
  const int lane = threadIdx.x & 63;
  int first = 0;
  for (int b0 = 0;; b0 += 64) {
    bool bad = false;
    const int x = b0 + lane;
    const int n = x < a.batch ? (seq_tiles(checked_len(a.tab, x, &bad), a.cut).n + per - 1) / per : 0;
    int before = x < b ? n : 0;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) before += __shfl_xor(before, o, 64);
    first += before;
    if (b < b0 + 64) return {first, __shfl(n, b - b0, 64)};
  }
}
// The sequence of unit u: {sequence (-1: none), split, splits}.
struct UnitAt {
  int b, split, n;
};
__device__ UnitAt unit_at(const PagedAttn& a, int per, int u) {
  const int lane = threadIdx.x & 63;
  int first = 0;
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    bool bad = false;
    const int x = b0 + lane;
    const int n = x < a.batch ? (seq_tiles(checked_len(a.tab, x, &bad), a.cut).n + per - 1) / per : 0;
    int end = n;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(end, o, 64);
      if (lane >= o) end += y;
    }
    const unsigned long long in = __ballot(u >= first + end - n && u < first + end);
    if (in) {
      const int l = __builtin_ctzll(in);
      return {b0 + l, u - first - __shfl(end - n, l, 64), __shfl(n, l, 64)};
    }
    first += __shfl(end, 63, 64);
  }
  return {-1, 0, 0};
}

// 8 e4m3 of two words as fp16, times 2^e of the factor `s`
__device__ __forceinline__ f16x8 cvt8(uint32_t a, uint32_t b, float s) {
  const f16x2 p = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, s, false), q = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, s, true);
  const f16x2 r = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, s, false), t = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, s, true);
  return f16x8{p.x, p.y, q.x, q.y, r.x, r.y, t.x, t.y};
}

// nodes that node i sees, and its position behind the cached slots
__device__ __forceinline__ uint64_t anc_of(const PagedAttn& a, int b, int i) {
  return a.anc ? a.anc[(long long)b * a.nodes + i] & (~0ull >> (64 - a.nodes)) : (2ull << i) - 1;
}
__device__ __forceinline__ int depth_of(uint64_t anc, int i) { return __builtin_popcountll(anc & ~(1ull << i)); }

constexpr float NO_MAX = -3e38f;  // reference of a row that has seen no key

template <int DH, bool SPLIT>
__global__ __launch_bounds__(256, 2) void paged_attention_kernel(PagedAttn a) {
  constexpr int NW = 4;
  constexpr int KP = DH / 32;  // 1 KB pieces of a tile's keys, two MFMAs each
  constexpr int DB = DH / 32;  // 1 KB pieces of its values: 32 dims each
  __shared__ float so[NW][32 * DH];
  __shared__ float sm[NW][32], sl[NW][32];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int col = lane & 31, hh = lane >> 5;
  const int G = a.Hq / a.pool.Hkv, R = G * a.nodes, rtiles = (R + 31) / 32;

  // XCD-aware decode: workgroups go round-robin over the 8 XCDs, so the row
  // tiles of one (unit, KV head) get the same id % 8 and share its L2
  const int id = blockIdx.x, rest = id >> 3;
  const int rt = rest % rtiles;
  const int st = (rest / rtiles) * 8 + (id & 7);
  const int hk = st % a.pool.Hkv, u = st / a.pool.Hkv;
  const int per = tiles_per_unit(a);
  const UnitAt at = unit_at(a, per, u);
  if (at.b < 0) return;  // uniform
  const int b = at.b;
  bool bad = false;
  const int len = checked_len(a.tab, b, &bad);
  const SeqTiles seq = seq_tiles(len, a.cut);
  const int i0 = (int)((long long)seq.n * at.split / at.n), i1 = (int)((long long)seq.n * (at.split + 1) / at.n);
  const int count = a.counts ? a.counts[b] : a.nodes;

  // row of this lane
  const int row = rt * 32 + col, rowc = min(row, R - 1);
  const int node = rowc % a.nodes, hq = hk * G + rowc / a.nodes;
  int pos = 0;
  if (a.cut.window) pos = len + depth_of(anc_of(a, b, node), node);

  // Q^T operands: piece x, half u holds dims 32 x + 16 hh + 8 u ..
  f16x8 qh[KP][2], ql[SPLIT ? KP : 1][2];
  float fac;  // scale_log2 and the row's power of two
  {
    float x[KP][2][8];
    const long long o = b * a.q.sb + node * a.q.sr + hq * a.q.sh + 16 * hh;
#pragma unroll
    for (int p = 0; p < KP; ++p)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        load8(a.q.p, o + 32 * p + 8 * h, a.q_lo.p ? PT_BF16 : a.dtype, a.q.vec, x[p][h]);
        if (SPLIT && a.q_lo.p) {
          float y[8];
          load8(a.q_lo.p, o + 32 * p + 8 * h, PT_BF16, a.q.vec, y);
#pragma unroll
          for (int e = 0; e < 8; ++e) x[p][h][e] += y[e];
        }
      }
    float mx = 0.f;
#pragma unroll
    for (int p = 0; p < KP; ++p)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 8; ++e) mx = fmaxf(mx, fabsf(x[p][h][e]));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    // to [2^8, 2^9); subnormal rows stay near zero, infinite ones infinite
    const int ex = min(max((int)(__float_as_uint(mx) >> 23) - 127, -110), 118);
    const float f = pow2i(8 - ex);
    fac = a.scale_log2 * pow2i(ex - 8);
#pragma unroll
    for (int p = 0; p < KP; ++p)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float v = x[p][h][e] * f;
          const _Float16 hi = (_Float16)v;
          qh[p][h][e] = hi;
          if constexpr (SPLIT) ql[p][h][e] = (_Float16)(v - (float)hi);
        }
  }

  float m = NO_MAX, l = 0.f;
  int E = PAGED_E_MIN;
  f32x16 oacc[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[d][r] = 0.f;

  // MFMA row -> slot of the tile: row 8q + 4h + e holds slot 16h + 4q + e
  const int krow = 16 * ((col >> 2) & 1) + 4 * (col >> 3) + (col & 3);
  const uint32_t ko = (hh * 32 + krow) * 16, vo = col * 32 + 16 * hh;
  const int wu = __builtin_amdgcn_readfirstlane(w);

  // The wave's tiles i0 + w, i0 + w + 4, ..: lane j looks up the j-th of 64.
  for (int base = i0 + wu; base < i1; base += 64 * NW) {
    int my_tile = 0, my_at = 0, my_ke = 0, my_ve = 0;
    const int my = base + NW * lane;
    if (my < i1) {
      my_tile = my < seq.sink ? my : my - seq.sink + seq.lo;
      int page = a.tab.pages[(long long)b * a.tab.stride + my_tile / a.pool.tpp];
      if (page < 0 || page >= a.pool.n_pages) {
        bad = true;
        if (a.status) atomicOr(a.status, PAGED_BAD_PAGE);
        page = 0;
      }
      my_at = (page * a.pool.Hkv + hk) * a.pool.tpp + my_tile % a.pool.tpp;
      my_ke = a.pool.ke[my_at];
      my_ve = a.pool.ve[my_at];
    }
    const int cnt = min(64, (i1 - base + NW - 1) / NW);
    u32x4 kf[KP], vf[DB];
    auto load = [&](int i, u32x4 (&kr)[KP], u32x4 (&vr)[DB]) {
      const long long o = (long long)__builtin_amdgcn_readlane(my_at, i) * (32 * DH);
      const uint8_t *kp = a.pool.k + o, *vp = a.pool.v + o;
#pragma unroll
      for (int x = 0; x < KP; ++x) kr[x] = *reinterpret_cast<const u32x4*>(kp + 1024 * x + ko);
#pragma unroll
      for (int x = 0; x < DB; ++x) vr[x] = *reinterpret_cast<const u32x4*>(vp + 1024 * x + vo);
    };
    load(0, kf, vf);
    for (int i = 0; i < cnt; ++i) {
      u32x4 kn[KP], vn[DB];
      load(min(i + 1, cnt - 1), kn, vn);
      const int tile = __builtin_amdgcn_readlane(my_tile, i), s0 = tile * 32;
      const int ke = __builtin_amdgcn_readlane(my_ke, i), ve = __builtin_amdgcn_readlane(my_ve, i);
      f32x16 s, s2;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = s2[r] = 0.f;
#pragma unroll
      for (int x = 0; x < KP; ++x)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const f16x8 k8 = cvt8(kf[x][2 * h], kf[x][2 * h + 1], 1.f);
          s = __builtin_amdgcn_mfma_f32_32x32x16_f16(k8, qh[x][h], s, 0, 0, 0);
          if constexpr (SPLIT) s2 = __builtin_amdgcn_mfma_f32_32x32x16_f16(k8, ql[x][h], s2, 0, 0, 0);
        }
      if constexpr (SPLIT) s += s2;
      // a tile that not every row sees whole: the last one, those at the
      // windows' starts, and the last one of the sinks
      const bool edge = s0 + 32 > len || (a.cut.window && s0 + 32 > a.cut.sinks && s0 < len + a.nodes - a.cut.window);
      bool nan_v = false;
      if (edge) {  // uniform
        const int lo = a.cut.window ? pos - a.cut.window : -1;  // slots above it are seen
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int slot = s0 + 16 * hh + r;
          if (!(slot < len && (slot > lo || slot < a.cut.sinks))) s[r] = -INFINITY;
        }
      }
      // never 0, which times a masked -inf would be a NaN
      const float f = fmaxf(fac * pow2i(ke), 0x1p-126f);
      float p[16];
      auto probs = [&]() {
        float t[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) t[r] = p[r] = __builtin_amdgcn_exp2f(fmaf(s[r], f, -m));
#pragma unroll
        for (int o = 8; o > 0; o >>= 1)
#pragma unroll
          for (int r = 0; r < o; ++r) t[r] += t[r + o];
        return t[0];
      };
      float sum = probs();
      if (__any(sum > 16384.f)) {
        float mx = -INFINITY;
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[r]);
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * f;
        const float mn = fmaxf(m, mx), al = __builtin_amdgcn_exp2f(m - mn);
        m = mn;
        l *= al;
#pragma unroll
        for (int d = 0; d < DB; ++d) oacc[d] *= al;
        sum = probs();
      }
      l += sum;
      if (ve > E) {  // uniform
        const float al = pow2i(E - ve);
        E = ve;
#pragma unroll
        for (int d = 0; d < DB; ++d) oacc[d] *= al;
      }
      const float vs = pow2i(ve - E);
      if (edge) {
        // what lies in slots that a row does not see must not reach it, NaN
        // included: bytes that no row sees become 0 ..
        const int lo0 = a.cut.window ? len - a.cut.window : -1;
#pragma unroll
        for (int x = 0; x < DB; ++x)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            uint32_t keep = 0;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const int slot = s0 + 16 * hh + 4 * e + c;
              if (slot < len && (slot > lo0 || slot < a.cut.sinks)) keep |= 0xffu << (8 * c);
            }
            const uint32_t v = vf[x][e] & keep;
            vf[x][e] = v;
            nan_v |= (((v & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0;
          }
        // .. and a NaN that only some rows see is given to those (rare: a
        // product of their 0 / 1 masks with the NaNs' places)
        if (a.cut.window && __any(nan_v)) {
#pragma unroll
          for (int x = 0; x < DB; ++x) {
            f32x16 hit;
#pragma unroll
            for (int r = 0; r < 16; ++r) hit[r] = 0.f;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              f16x8 is, sees;
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const uint32_t byte = vf[x][2 * t + e / 4] >> (8 * (e % 4)) & 0x7f;
                is[e] = byte == 0x7f ? (_Float16)1.f : (_Float16)0.f;
                sees[e] = s[8 * t + e] == -INFINITY ? (_Float16)0.f : (_Float16)1.f;
              }
              hit = __builtin_amdgcn_mfma_f32_32x32x16_f16(is, sees, hit, 0, 0, 0);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r)
              if (hit[r] > 0.f) oacc[x][r] = __builtin_nanf("");
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
              for (int c = 0; c < 4; ++c)
                if ((vf[x][e] >> (8 * c) & 0x7f) == 0x7f) vf[x][e] &= ~(0xffu << (8 * c));
          }
        }
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        f16x8 ph, pl;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const _Float16 hi = (_Float16)p[8 * t + e];
          ph[e] = hi;
          if constexpr (SPLIT) pl[e] = (_Float16)(p[8 * t + e] - (float)hi);
        }
#pragma unroll
        for (int x = 0; x < DB; ++x) {
          const f16x8 v8 = cvt8(vf[x][2 * t], vf[x][2 * t + 1], vs);
          oacc[x] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v8, ph, oacc[x], 0, 0, 0);
          if constexpr (SPLIT) oacc[x] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v8, pl, oacc[x], 0, 0, 0);
        }
      }
#pragma unroll
      for (int x = 0; x < KP; ++x) kf[x] = kn[x];
#pragma unroll
      for (int x = 0; x < DB; ++x) vf[x] = vn[x];
    }
  }
  l += __shfl_xor(l, 32, 64);
  if (__any(bad)) l = __builtin_nanf("");  // a tile that is not there: the rows become NaN

  // ---- the waves' results meet in LDS: row `col` at so[w][col * DH ..], its
  // 16-byte chunk c at c ^ (col & 7)
  {
    const float fe = pow2i(E);
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int rg = 0; rg < 4; ++rg) {
        const int c = 8 * d + 2 * rg + hh;
        *reinterpret_cast<float4*>(&so[w][col * DH + 4 * (c ^ (col & 7))]) =
            make_float4(oacc[d][4 * rg] * fe, oacc[d][4 * rg + 1] * fe, oacc[d][4 * rg + 2] * fe, oacc[d][4 * rg + 3] * fe);
      }
    if (hh == 0) sm[w][col] = m, sl[w][col] = l;
  }
  __syncthreads();
  constexpr int CH = DH / 4;
  const long long prow = ((long long)u * a.pool.Hkv + hk) * R + rt * 32;
  const int live = min(32, R - rt * 32);
  for (int i = threadIdx.x; i < live * CH; i += 256) {
    const int r = i / CH, c = i % CH;
    if ((rt * 32 + r) % a.nodes >= count) continue;  // an absent node
    float M = sm[0][r];
#pragma unroll
    for (int x = 1; x < NW; ++x) M = fmaxf(M, sm[x][r]);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    float L = 0.f;
#pragma unroll
    for (int x = 0; x < NW; ++x) {
      const float f = __builtin_amdgcn_exp2f(sm[x][r] - M);
      const float4 v = *reinterpret_cast<const float4*>(&so[x][r * DH + 4 * (c ^ (r & 7))]);
      o.x += f * v.x, o.y += f * v.y, o.z += f * v.z, o.w += f * v.w;
      L += f * sl[x][r];
    }
    *reinterpret_cast<float4*>(a.part_o + (prow + r) * DH + 4 * c) = o;
    if (c == 0) a.part_ml[(prow + r) * 2] = M, a.part_ml[(prow + r) * 2 + 1] = L;
  }
}

// A thread: 4 dims of a head of one node.
__global__ __launch_bounds__(256) void paged_combine_kernel(PagedAttn a) {
  const int dh = a.pool.dh, quads = dh / 4;
  const int b = blockIdx.x / a.nodes, i = blockIdx.x % a.nodes;
  const int t = blockIdx.y * 256 + threadIdx.x;
  const int per = tiles_per_unit(a);
  const Units un = units_of(a, per, b);
  const int G = a.Hq / a.pool.Hkv, R = G * a.nodes;
  bool bad = false;
  const int len = checked_len(a.tab, b, &bad);
  int count = a.counts ? a.counts[b] : a.nodes;
  if (count < 0 || count > a.nodes) bad = true, count = min(max(count, 0), a.nodes);
  if (bad && a.status && threadIdx.x == 0) atomicOr(a.status, PAGED_BAD_LENGTH);
  if (t >= a.Hq * quads) return;  // whole heads: 64 threads of a wave hold 2 or 4
  const int h = t / quads, d = t % quads * 4, hk = h / G;
  const bool live = i < count;
  if (!live && a.out_ks == 0) return;
  float4 out = make_float4(0.f, 0.f, 0.f, 0.f);
  if (live) {  // uniform over the workgroup
    float4 q = load4(a.q.p, b * a.q.sb + i * a.q.sr + h * a.q.sh + d, a.q_lo.p ? PT_BF16 : a.dtype, a.q.vec);
    if (a.q_lo.p) {
      const float4 y = load4(a.q_lo.p, b * a.q.sb + i * a.q.sr + h * a.q.sh + d, PT_BF16, a.q.vec);
      q.x += y.x, q.y += y.y, q.z += y.z, q.w += y.w;
    }
    // nodes of the root path, eight at a time
    uint64_t anc = anc_of(a, b, i);
    const int dep = depth_of(anc, i);
    float m = -INFINITY, l = 0.f;
    float4 o = out;
    const long long kb = b * a.k.sb + hk * a.k.sh + d, vb = b * a.v.sb + hk * a.v.sh + d;
    int r = 0;  // rank of the next node
    while (anc) {
      constexpr int TB = 8;
      float sc[TB];
      float4 v4[TB];
      int n = 0;
#pragma unroll
      for (int x = 0; x < TB; ++x) {
        const bool ok = anc != 0;
        const int j = ok ? __builtin_ctzll(anc) : 0;
        anc &= anc - 1;
        const bool sees = ok && (!a.cut.window || dep - r < a.cut.window || (long long)len + r < a.cut.sinks);
        r += ok;
        sc[x] = -INFINITY;
        v4[x] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (sees) {  // uniform
          const float4 k = load4(a.k.p, kb + j * a.k.sr, a.dtype, a.k.vec);
          v4[x] = load4(a.v.p, vb + j * a.v.sr, a.dtype, a.v.vec);
          sc[x] = q.x * k.x + q.y * k.y + q.z * k.z + q.w * k.w;
        }
        n |= sees << x;
      }
      for (int s = quads >> 1; s > 0; s >>= 1)
#pragma unroll
        for (int x = 0; x < TB; ++x) sc[x] += __shfl_xor(sc[x], s, 64);
      float mn = m;
#pragma unroll
      for (int x = 0; x < TB; ++x) mn = fmaxf(mn, sc[x] *= a.scale_log2);
      if (mn == -INFINITY && n == 0) continue;
      const float al = m == -INFINITY ? 0.f : exp2f(m - mn);
      l *= al;
      o.x *= al, o.y *= al, o.z *= al, o.w *= al;
#pragma unroll
      for (int x = 0; x < TB; ++x)
        if (n >> x & 1) {
          const float e = exp2f(sc[x] - mn);
          l += e;
          o.x += e * v4[x].x, o.y += e * v4[x].y, o.z += e * v4[x].z, o.w += e * v4[x].w;
        }
      m = mn;
    }
    // the cached part's units, in their order
    for (int s = 0; s < un.n; ++s) {
      const long long row = ((long long)(un.first + s) * a.pool.Hkv + hk) * R + (h % G) * a.nodes + i;
      const float mu = a.part_ml[row * 2], lu = a.part_ml[row * 2 + 1];
      const float4 ou = *reinterpret_cast<const float4*>(a.part_o + row * dh + d);
      if (mu == NO_MAX && lu == 0.f) continue;  // no slot of it is seen
      const float mn = fmaxf(m, mu);
      const float al = m == -INFINITY ? 0.f : exp2f(m - mn), e = exp2f(mu - mn);
      l = l * al + lu * e;
      o.x = o.x * al + ou.x * e, o.y = o.y * al + ou.y * e, o.z = o.z * al + ou.z * e, o.w = o.w * al + ou.w * e;
      m = mn;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;  // a row that sees nothing is 0
    out = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
    if (bad) out.x = out.y = out.z = out.w = __builtin_nanf("");
  }
  if (a.out_ks) {
    uint16_t* dst = static_cast<uint16_t*>(a.out) + xpack_off((long long)b * a.nodes + i, h * dh + d, a.out_ks);
    const Hilo2 p0 = pack_hilo2(out.x, out.y), p1 = pack_hilo2(out.z, out.w);
    *reinterpret_cast<uint2*>(dst) = make_uint2(p0.hi, p1.hi);
    *reinterpret_cast<uint2*>(dst + XPACK_LO) = make_uint2(p0.lo, p1.lo);
    return;
  }
  const long long at = b * a.ob + i * a.orow + h * a.oh + d;
  if (a.dtype == PT_F32) {
    float* f = static_cast<float*>(a.out) + at;
    if (a.out_vec) *reinterpret_cast<float4*>(f) = out;
    else f[0] = out.x, f[1] = out.y, f[2] = out.z, f[3] = out.w;
    return;
  }
  uint2 w;
  if (a.dtype == PT_BF16) {
    w = make_uint2(pack_bf16x2(out.x, out.y), pack_bf16x2(out.z, out.w));
  } else {
    auto f = [](float x) { return (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)x); };
    w = make_uint2(f(out.x) | f(out.y) << 16, f(out.z) | f(out.w) << 16);
  }
  uint16_t* p = static_cast<uint16_t*>(a.out) + at;
  if (a.out_vec) *reinterpret_cast<uint2*>(p) = w;
  else p[0] = w.x, p[1] = w.x >> 16, p[2] = w.y, p[3] = w.y >> 16;
}

}  // namespace

void paged_plan(PagedAttn& a, int max_length) {
  const int G = a.Hq / a.pool.Hkv, rtiles = (G * a.nodes + 31) / 32;
  // two workgroups on each of 256 CUs
  const int streams = a.pool.Hkv * rtiles;
  a.cut.target = std::max(1, 512 / streams);
  a.cut.least = 4;  // a tile for each wave
  // tiles of a sequence: all, or those that window - 1 slots can touch and the sinks
  int most = (int)(((long long)max_length + 31) >> 5);
  if (a.cut.window)
    most = (int)std::min<long long>(most, ((long long)a.cut.window + 30) / 32 + 1 + ((long long)a.cut.sinks + 31) / 32);
  // units of a sequence of n tiles: ceil(n / per) with per >= least and >= total / target
  const long long by_len = (long long)a.batch * ((most + a.cut.least - 1) / a.cut.least);
  a.units = (int)std::min<long long>(by_len, (long long)a.cut.target + a.batch);
}

size_t paged_workspace_floats(const PagedAttn& a) {
  const size_t rows = (size_t)a.units * a.Hq * a.nodes;
  return rows * (a.pool.dh + 2);
}

hipError_t launch_paged_attention(const PagedAttn& a, hipStream_t s) {
  const int G = a.Hq / a.pool.Hkv, rtiles = (G * a.nodes + 31) / 32;
  const bool split = a.dtype == PT_F32 || a.q_lo.p;
  if (a.units > 0) {
    const long long streams = ((long long)a.units * a.pool.Hkv + 7) / 8 * 8;
    if (streams * rtiles > 0x7fffffffLL) return hipErrorInvalidValue;
    const dim3 grid((unsigned)(streams * rtiles));
    if (a.pool.dh == 128 && split) hipLaunchKernelGGL((paged_attention_kernel<128, true>), grid, dim3(256), 0, s, a);
    else if (a.pool.dh == 128) hipLaunchKernelGGL((paged_attention_kernel<128, false>), grid, dim3(256), 0, s, a);
    else if (a.pool.dh == 64 && split) hipLaunchKernelGGL((paged_attention_kernel<64, true>), grid, dim3(256), 0, s, a);
    else if (a.pool.dh == 64) hipLaunchKernelGGL((paged_attention_kernel<64, false>), grid, dim3(256), 0, s, a);
    else return hipErrorInvalidValue;
  }
  const dim3 grid(a.batch * a.nodes, (a.Hq * (a.pool.dh / 4) + 255) / 256);
  hipLaunchKernelGGL(paged_combine_kernel, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace griffin

// Attention of draft-tree nodes over the 8-bit paged cache (paged.h).
//
// Node i of sequence b (bits anc[i]; a chain: nodes 0 .. i) stands at position
// p = length + |anc[i] without i|.  It sees the cached slots s < length with
// window == 0, p - s < window or s < sinks, and the nodes of anc[i], the r-th
// of which stands at position length + r, by the same window.
//
// The cached part is computed in units: some of the tiles of one sequence, a KV
// head, and a block of the head group's rows (row = head * N + node), as many
// units as fill the chip (paged_plan, unit_at).  Three kernels for it: row tiles
// of 32 here, of 16 for few rows and short calls (paged_thin.hip), and
// paged_wide_kernel for many rows over long sequences.
//
// Per tile a wave loads 16 bytes a lane and piece, which are the matrix operands
// as they stand, and computes S^T = K Q^T and O^T += V^T P^T with
// v_mfma_f32_32x32x16, so that a lane owns a query row and the softmax is
// lane-local:
//  * e4m3 is exact in fp16 and bf16.  Keys are converted as they are, their
//    tile's exponent goes into the score's factor; values are converted relative
//    to the largest exponent the wave has met (E), which is uniform over the wave
//    and rarely rises; the accumulators follow it when it does.
//  * Keys meet the matrix cores in a permuted row order, so that accumulator
//    register r of lane half h holds slot 16 h + r: the P operand is the lane's
//    own registers and the V operand 16 consecutive slots of a dim.
//  * bf16 and fp16 queries are operands as they are; fp32 ones, scaled by a power
//    of two per row to fill fp16, enter as high and low parts (22 bits).  So do
//    their and fp16 inputs' probabilities; bf16 inputs' are rounded to fp16,
//    2^-12 relative: an eighth of the rounding of a bf16 output.
//  * What the probabilities refer to follows the scores only where a lane's sum
//    of a tile passes 2^P_TOP, so no maximum is formed for most tiles.
//
// paged_combine_kernel joins a row's units in their order, adds the nodes of
// its own root path in fp32, and writes the row.

#include <algorithm>

#include "paged_device.h"

namespace griffin {

namespace {

// A tile in a wave's registers, as it is stored: 1 KB pieces, 16 bytes a lane.
template <int DH>
struct Keys {
  u32x4 r[DH / 32];
};
template <int DH>
struct Vals {
  u32x4 r[DH / 32];
};

// Q^T operand of a row tile: lane (row col, half hh) holds, of piece x and
// half h, dims 32 x + 16 hh + 8 h .. (Q_FP8: pieces 2 y and 2 y + 1 together).
template <int DH, int QF>
struct Query {
  static constexpr int KP = DH / 32;
  u32x4 a[QF == Q_FP8 ? 1 : KP][2], b[QF == Q_SPLIT ? KP : 1][2];
  i32x8 e[QF == Q_FP8 ? KP / 2 : 1][2];
  float fac;  // the scores' scale in the log2 domain, and the power of two that the row was scaled by

  __device__ __forceinline__ void take(const SplitRows<DH, 32>& rows, int col, int hh) {
    fac = rows.fac[col];
#pragma unroll
    for (int x = 0; x < KP; ++x)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        a[x][h] = rows.get(0, col, 4 * x + 2 * hh + h);
        b[x][h] = rows.get(1, col, 4 * x + 2 * hh + h);
      }
  }
  __device__ __forceinline__ void load(const PagedAttn& p, long long at) {
    fac = p.scale_log2;
    if constexpr (QF == Q_BF16 || QF == Q_F16) {
#pragma unroll
      for (int x = 0; x < KP; ++x)
#pragma unroll
        for (int h = 0; h < 2; ++h) a[x][h] = load8_raw(p.q.p, at + 32 * x + 8 * h, p.q.vec);
    } else {
      float v[KP][2][8], mx = load_query<KP, 2, 32, QF == Q_SPLIT>(p, at, v);
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      constexpr int TOP = QF == Q_FP8 ? 7 : 8;  // the row's largest value to [2^TOP, 2^(TOP + 1))
      const int ex = scale_exponent(mx);
      const float f = pow2i(TOP - ex);
      fac *= pow2i(ex - TOP);
#pragma unroll
      for (int x = 0; x < KP; ++x)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 8; i += 2) {
            const float v0 = v[x][h][i] * f, v1 = v[x][h][i + 1] * f;
            if constexpr (QF == Q_SPLIT) {
              const Hilo2 parts = split_f16(v0, v1);
              a[x][h][i / 2] = parts.hi;
              b[x][h][i / 2] = parts.lo;
            } else {
              // word i / 4 of the half, its lower or upper pair; the low part
              // 2^4 up, which its product's scale takes back
              const int at8 = 4 * (x % 2) + 2 * h + i / 4;
              if (i % 4 == 0) {
                const int w = __builtin_amdgcn_cvt_pk_fp8_f32(v0, v1, 0, false);
                const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
                e[x / 2][0][at8] = w;
                e[x / 2][1][at8] = __builtin_amdgcn_cvt_pk_fp8_f32((v0 - hi.x) * 16.f, (v1 - hi.y) * 16.f, 0, false);
              } else {
                const int w = __builtin_amdgcn_cvt_pk_fp8_f32(v0, v1, e[x / 2][0][at8], true);
                const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
                e[x / 2][0][at8] = w;
                e[x / 2][1][at8] = __builtin_amdgcn_cvt_pk_fp8_f32((v0 - hi.x) * 16.f, (v1 - hi.y) * 16.f, e[x / 2][1][at8], true);
              }
            }
          }
    }
  }

  // S^T = K Q^T: what step g of STEPS adds to hi (and lo, the low part's sum
  // of Q_SPLIT), given the keys and, of those that have to be converted, piece
  // g / PER's halves
  static constexpr int STEPS = QF == Q_FP8 ? KP : QF == Q_SPLIT ? 4 * KP : 2 * KP;
  __device__ __forceinline__ void step(int g, const Keys<DH>& k, const u32x4& k16, f32x16& hi, f32x16& lo) const {
    if constexpr (QF == Q_FP8) {
      const i32x8 k8 = __builtin_bit_cast(i32x8, KeyPair{k.r[g / 2 * 2], k.r[g / 2 * 2 + 1]});
      hi = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(k8, e[g / 2][g % 2], hi, 0, 0, 0, 0x7f7f7f7f, 0,
                                                           g % 2 ? 0x7b7b7b7b : 0x7f7f7f7f);
    } else if constexpr (QF == Q_BF16) {
      hi = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(k16), as_bf16x8(a[g / 2][g % 2]), hi, 0, 0, 0);
    } else if constexpr (QF == Q_F16) {
      hi = __builtin_amdgcn_mfma_f32_32x32x16_f16(as_f16x8(k16), as_f16x8(a[g / 2][g % 2]), hi, 0, 0, 0);
    } else if (g % 2 == 0) {
      hi = __builtin_amdgcn_mfma_f32_32x32x16_f16(as_f16x8(k16), as_f16x8(a[g / 4][g / 2 % 2]), hi, 0, 0, 0);
    } else {
      lo = __builtin_amdgcn_mfma_f32_32x32x16_f16(as_f16x8(k16), as_f16x8(b[g / 4][g / 2 % 2]), lo, 0, 0, 0);
    }
  }
  // the converted keys of step g (the same for a Q_SPLIT pair)
  static __device__ __forceinline__ u32x4 convert(int g, const Keys<DH>& k) {
    const int c = QF == Q_SPLIT ? g / 2 : g;
    const uint32_t x = k.r[c / 2][2 * (c % 2)], y = k.r[c / 2][2 * (c % 2) + 1];
    if constexpr (QF == Q_BF16) return __builtin_bit_cast(u32x4, cvt8_bf16(x, y));
    else return __builtin_bit_cast(u32x4, cvt8(x, y, 1.f));
  }
  __device__ __forceinline__ f32x16 scores(const Keys<DH>& k) const {
    f32x16 hi = f32x16(0.f), lo = f32x16(0.f);
    u32x4 k16 = zero_u4();
#pragma unroll
    for (int g = 0; g < STEPS; ++g) {
      if (QF != Q_FP8 && (QF != Q_SPLIT || g % 2 == 0)) k16 = convert(g, k);
      step(g, k, k16, hi, lo);
    }
    if constexpr (QF == Q_SPLIT) hi += lo;
    return hi;
  }
};

// Running softmax and output of a row tile: lane col's row (both halves hold
// it), dims 32 d + 8 (r / 4) + 4 hh + r % 4 of it in o[d][r], times 2^(V_LIFT - E).
template <int DH>
struct State {
  float m, l;
  int E;  // uniform
  f32x16 o[DH / 32];

  __device__ __forceinline__ void clear() {
    m = NO_MAX;
    l = 0.f;
    E = PAGED_E_MIN;
#pragma unroll
    for (int d = 0; d < DH / 32; ++d) o[d] = f32x16(0.f);
  }
  __device__ __forceinline__ void scale(float f) {
#pragma unroll
    for (int d = 0; d < DH / 32; ++d) o[d] *= f;
  }
  // raise the reference towards the scores' maximum (both halves')
  __device__ __forceinline__ void follow(const f32x16& s, float f) {
    float mx = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[r]);
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * f;
    const float mn = fmaxf(m, mx - P_LIFT), al = __builtin_amdgcn_exp2f(m - mn);
    m = mn;
    l *= al;
    scale(al);
  }
  // raise E to a tile's exponent
  __device__ __forceinline__ void reach(int ve) {
    if (ve > E) {  // uniform
      scale(pow2i(E - ve));
      E = ve;
    }
  }
};

// Softmax of one tile's scores and O^T += V^T P^T.  EDGE: a tile (first slot
// s0) that not every row sees whole; this lane's row stands at `pos`, the
// first node at sight.len.
template <int DH, int QF, class EDGE>
__device__ __forceinline__ void attend(State<DH>& st, f32x16 s, Vals<DH> v, float f, int ve, EDGE, const Sight& sight,
                                       int s0, int pos) {
  constexpr int DB = DH / 32;
  const int hh = threadIdx.x >> 5 & 1;
  if constexpr (EDGE::value) {
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (!sight.of(s0 + 16 * hh + r, pos)) s[r] = -INFINITY;
  }
  float p[16], sum;
  auto probs = [&]() {
    float x[8];
#pragma unroll
    for (int r = 0; r < 16; ++r) p[r] = __builtin_amdgcn_exp2f(fmaf(s[r], f, -st.m));
#pragma unroll
    for (int r = 0; r < 8; ++r) x[r] = p[r] + p[r + 8];
#pragma unroll
    for (int o = 4; o > 0; o >>= 1)
#pragma unroll
      for (int r = 0; r < o; ++r) x[r] += x[r + o];
    sum = x[0];
  };
  probs();
  if (__any(sum > pow2i(P_TOP))) {
    st.follow(s, f);
    probs();
  }
  st.l += sum;
  st.reach(ve);
  const float vs = value_factor(ve, st.E);
  if constexpr (EDGE::value) {
    // what lies in slots that a row does not see must not reach it, NaN
    // included: bytes that no row sees become 0 ..
    bool nan_v = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      uint32_t keep = 0;
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (sight.of(s0 + 16 * hh + 4 * e + c, sight.len)) keep |= 0xffu << (8 * c);
#pragma unroll
      for (int x = 0; x < DB; ++x) {
        const uint32_t y = v.r[x][e] & keep;
        v.r[x][e] = y;
        nan_v |= (((y & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0;
      }
    }
    // .. and a NaN that only some rows see is given to those (rare: a product
    // of their 0 / 1 masks with the NaNs' places)
    if (sight.window && __any(nan_v)) {
#pragma unroll
      for (int x = 0; x < DB; ++x) {
        f32x16 hit = f32x16(0.f);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          f16x8 is, sees;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const uint32_t byte = v.r[x][2 * h + e / 4] >> (8 * (e % 4)) & 0x7f;
            is[e] = byte == 0x7f ? (_Float16)1.f : (_Float16)0.f;
            sees[e] = s[8 * h + e] == -INFINITY ? (_Float16)0.f : (_Float16)1.f;
          }
          hit = __builtin_amdgcn_mfma_f32_32x32x16_f16(is, sees, hit, 0, 0, 0);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (hit[r] > 0.f) st.o[x][r] = __builtin_nanf("");
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int c = 0; c < 4; ++c)
            if ((v.r[x][e] >> (8 * c) & 0x7f) == 0x7f) v.r[x][e] &= ~(0xffu << (8 * c));
      }
    }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    u32x4 ph, pl;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float x = p[8 * h + 2 * e], y = p[8 * h + 2 * e + 1];
      const f16x2 hi = __builtin_convertvector(f32x2{x, y}, f16x2);
      ph[e] = __builtin_bit_cast(uint32_t, hi);
      if constexpr (probs_split(QF))
        pl[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x - (float)hi.x, y - (float)hi.y}, f16x2));
    }
#pragma unroll
    for (int x = 0; x < DB; ++x) {
      const f16x8 v8 = cvt8(v.r[x][2 * h], v.r[x][2 * h + 1], vs);
      st.o[x] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v8, as_f16x8(ph), st.o[x], 0, 0, 0);
      if constexpr (probs_split(QF)) st.o[x] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v8, as_f16x8(pl), st.o[x], 0, 0, 0);
    }
  }
}

// MFMA row -> slot of the tile: row 8q + 4h + e holds slot 16h + 4q + e
__device__ __forceinline__ int slot_of_row(int col) { return 16 * ((col >> 2) & 1) + 4 * (col >> 3) + (col & 3); }

template <int DH>
__device__ __forceinline__ void load_keys(const PagedAttn& a, long long at, int col, int hh, Keys<DH>& k) {
  const uint8_t* p = a.pool.k + at * (32 * DH) + (hh * 32 + slot_of_row(col)) * 16;
#pragma unroll
  for (int x = 0; x < DH / 32; ++x) k.r[x] = *reinterpret_cast<const u32x4*>(p + 1024 * x);
}
template <int DH>
__device__ __forceinline__ void load_vals(const PagedAttn& a, long long at, int col, int hh, Vals<DH>& v) {
  const uint8_t* p = a.pool.v + at * (32 * DH) + col * 32 + 16 * hh;
#pragma unroll
  for (int x = 0; x < DH / 32; ++x) v.r[x] = *reinterpret_cast<const u32x4*>(p + 1024 * x);
}

// The first `rows` rows of a row tile's output to LDS: row r at buf[r * DH ..], its 16-byte chunk c at
// c ^ (r & 7) (conflict-free here and where rows are read).
template <int DH>
__device__ __forceinline__ void put_rows(const State<DH>& st, int col, int hh, int rows, float* buf) {
  if (col >= rows) return;
  const float fe = out_factor(st.E);
#pragma unroll
  for (int d = 0; d < DH / 32; ++d)
#pragma unroll
    for (int rg = 0; rg < 4; ++rg) {
      const int c = 8 * d + 2 * rg + hh;
      *reinterpret_cast<float4*>(buf + col * DH + 4 * (c ^ (col & 7))) =
          make_float4(st.o[d][4 * rg] * fe, st.o[d][4 * rg + 1] * fe, st.o[d][4 * rg + 2] * fe, st.o[d][4 * rg + 3] * fe);
    }
}

// One row tile per workgroup, whose four waves take every fourth tile of the
// unit each and meet in LDS; two workgroups per CU, the next tile's loads in
// flight while one is computed.  (One workgroup of eight waves for a whole
// sequence, with the join, is slower down to 200 slots: 61 nodes 14.8 us against
// 9.4 + 5.4.)
template <int DH, int QF>
__global__ __launch_bounds__(256, 2) void paged_attention_kernel(PagedAttn a) {
  constexpr int NW = 4;
  __shared__ __align__(16) float so[NW][32 * DH];
  __shared__ float sm[NW][32], sl[NW][32];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, hh = lane >> 5;
  const int G = a.Hq / a.pool.Hkv, R = G * a.nodes;
  Place p;
  if (!place_of(a, (R + 31) / 32, p)) return;
  const int count = a.counts ? a.counts[p.b] : a.nodes;

  // lane j looks up the j-th of 64 of the wave's tiles i0 + w, i0 + w + NW, ..
  const int mine = p.i1 - p.i0 - w > 0 ? (p.i1 - p.i0 - w + NW - 1) / NW : 0;
  int my_tile = 0, my_at = 0, my_ke = 0, my_ve = 0;
  auto look = [&](int base) {
    if (base + lane < mine) {
      const TileAt t = look_up(a, p, p.i0 + w + NW * (base + lane));
      my_tile = t.tile;
      my_at = t.at;
      my_ke = a.pool.ke[t.at];
      my_ve = a.pool.ve[t.at];
    }
  };
  look(0);
  const int node = min(p.rb * 32 + col, R - 1) % a.nodes;
  const int pos = a.cut.window ? p.sight.len + depth_of(anc_of(a, p.b, node), node) : 0;
  Query<DH, QF> q;
  if constexpr (QF == Q_SPLIT) {
    auto& rows = *reinterpret_cast<SplitRows<DH, 32>*>(so);
    static_assert(sizeof(rows) <= sizeof(so));
    rows.fill(a, [&](int r) { return query_row(a, p, p.rb * 32 + r); });
    q.take(rows, col, hh);
  } else {
    q.load(a, query_row(a, p, p.rb * 32 + col) + 16 * hh);
  }
  State<DH> st;
  st.clear();
  for (int base = 0; base < mine; base += 64) {
    if (base) look(base);
    // tiles that not every row sees whole (the last one, those at the windows'
    // starts, the last one of the sinks) come first
    const int s0 = my_tile * 32;
    const bool edge = s0 + 32 > p.sight.len ||
                      (a.cut.window && s0 + 32 > a.cut.sinks && s0 < p.sight.len + a.nodes - a.cut.window);
    const unsigned long long all = __ballot(base + lane < mine);
    unsigned long long todo = all & __ballot(edge), rest = all & ~todo;
    Keys<DH> k0, k1;
    Vals<DH> v0, v1;
    auto load = [&](int i, Keys<DH>& k, Vals<DH>& v) {
      const long long at = __builtin_amdgcn_readlane(my_at, i);
      load_keys<DH>(a, at, col, hh, k);
      load_vals<DH>(a, at, col, hh, v);
    };
    auto tile = [&](auto kind, int i, const Keys<DH>& k, const Vals<DH>& v) {
      const f32x16 s = q.scores(k);
      attend<DH, QF>(st, s, v, score_factor(q.fac, __builtin_amdgcn_readlane(my_ke, i)),
                     __builtin_amdgcn_readlane(my_ve, i), kind, p.sight, __builtin_amdgcn_readlane(my_tile, i) * 32, pos);
    };
    while (todo) {
      const int i = __builtin_ctzll(todo);
      todo &= todo - 1;
      load(i, k0, v0);
      tile(Edge{}, i, k0, v0);
    }
    if (!rest) continue;
    int left = __builtin_popcountll(rest);
    auto next = [&](int i) {  // the next of the others, or the last one again
      const unsigned long long r = rest;
      rest &= rest - 1;
      return r ? (int)__builtin_ctzll(r) : i;
    };
    int i = next(0);
    load(i, k0, v0);
    for (;;) {
      const int n = next(i);
      load(n, k1, v1);
      tile(Whole{}, i, k0, v0);
      if (--left == 0) break;
      i = next(n);
      load(i, k0, v0);
      tile(Whole{}, n, k1, v1);
      if (--left == 0) break;
    }
  }
  if constexpr (QF == Q_SPLIT) __syncthreads();  // every wave has its queries
  float l = st.l + __shfl_xor(st.l, 32, 64);
  if (__any(p.bad)) l = __builtin_nanf("");  // a tile that is not there: the rows become NaN
  put_rows<DH>(st, col, hh, R - p.rb * 32, so[w]);
  const float2 ml = out_sums(st.m, l);
  if (hh == 0) sm[w][col] = ml.x, sl[w][col] = ml.y;
  __syncthreads();
  constexpr int CH = DH / 4;
  const long long prow = ((long long)p.u * a.pool.Hkv + p.hk) * R + p.rb * 32;
  for (int i = threadIdx.x; i < 32 * CH; i += 256) {
    const int r = i / CH, c = i % CH, gr = p.rb * 32 + r;
    if (gr >= R || (count < a.nodes && gr % a.nodes >= count)) continue;  // an absent node
    float m = sm[0][r];
#pragma unroll
    for (int x = 1; x < NW; ++x) m = fmaxf(m, sm[x][r]);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    float L = 0.f;
#pragma unroll
    for (int x = 0; x < NW; ++x) {
      const float f = __builtin_amdgcn_exp2f(sm[x][r] - m);
      const float4 v = *reinterpret_cast<const float4*>(&so[x][r * DH + 4 * (c ^ (r & 7))]);
      o.x += f * v.x, o.y += f * v.y, o.z += f * v.z, o.w += f * v.w;
      L += f * sl[x][r];
    }
    *reinterpret_cast<float4*>(a.part_o + (prow + r) * DH + 4 * c) = o;
    if (c == 0) *reinterpret_cast<float2*>(a.part_ml + (prow + r) * 2) = make_float2(m, L);
  }
}

// Row tiles side by side: NW waves of one row tile each over the same tiles,
// which the workgroup stages into an LDS ring once (each wave an equal share of
// a tile's 1 KB pieces, which are MFMA operands as they stand).  Two waves per
// SIMD; a step over tile i is written as a sequence of MFMAs with their share
// of everything else, held by sched_barrier, so that matrix and vector work
// overlap:
//   the scores of tile i + 1, between the softmax of tile i;
//   O += V P of tile i, between the conversion of its values, the reads of tile
//   i + 2's keys and the maximum of tile i + 1's scores, which decides whether
//   a reference has to rise: no branch stands inside a step.  At a higher
//   priority, so that one wave's matrix work goes before the other's softmax
//   (148 -> 142 us for 8 x 61 nodes over 16384 slots).
// The workgroup meets once in two tiles (2 p, 2 p + 1): then every wave has its
// share of pair p + 2 and is done with pair p, whose slots pair p + D / 2 gets.
// Tiles that not every row sees whole are computed one by one before.
template <int DH, int QF, int NW>
__global__ __launch_bounds__(64 * NW, 2) void paged_wide_kernel(PagedAttn a) {
  constexpr int KP = DH / 32, DB = DH / 32, PIECES = KP + DB, D = 2 * NW;  // ring slots
  constexpr int STAGERS = PIECES < NW ? PIECES : NW, PPW = PIECES / STAGERS;  // waves that stage, pieces of each
  static_assert(PIECES % STAGERS == 0 && PPW * D < 64 && D % 2 == 0 && D >= 8, "ring shape");
  constexpr int LDS = D * PIECES * 1024 > NW * 32 * DH * 4 ? D * PIECES * 1024 : NW * 32 * DH * 4;
  __shared__ u32x4 lds[LDS / 16];
  u32x4(*ring)[PIECES][64] = reinterpret_cast<u32x4(*)[PIECES][64]>(lds);
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, hh = lane >> 5;
  const int G = a.Hq / a.pool.Hkv, R = G * a.nodes;
  Place p;
  if (!place_of(a, (R + 32 * NW - 1) / (32 * NW), p)) return;
  const int count = a.counts ? a.counts[p.b] : a.nodes;
  const int row0 = (p.rb * NW + w) * 32;

  // The unit's tiles that every row sees whole: list entries [i0, e0) and
  // [w0, w1); the others are [e0, w0) and [w1, i1).
  int e0 = p.i0, w0 = p.i0, w1 = p.i1;
  {
    const int len = p.sight.len;
    if (a.cut.window) {
      e0 = min(max(min(p.seq.sink, a.cut.sinks >> 5), p.i0), p.i1);
      const int clear = max(0, len + a.nodes - a.cut.window);  // slots from here on are in every window
      w0 = max(p.seq.sink, ((clear + 31) >> 5) - p.seq.lo + p.seq.sink);
      w0 = min(max(w0, e0), p.i1);
    }
    w1 = min(max(p.seq.n - ((len & 31) != 0), w0), p.i1);
  }
  const int n0 = e0 - p.i0, whole = n0 + w1 - w0, edges = p.i1 - p.i0 - whole;
  auto whole_at = [&](int j) { return j < n0 ? p.i0 + j : w0 + j - n0; };
  auto edge_at = [&](int j) { return j < w0 - e0 ? e0 + j : w1 + j - (w0 - e0); };

  const int row = min(row0 + col, R - 1), node = row % a.nodes, hq = p.hk * G + row / a.nodes;
  const int pos = a.cut.window ? p.sight.len + depth_of(anc_of(a, p.b, node), node) : 0;
  Query<DH, QF> q;
  q.load(a, p.b * a.q.sb + node * a.q.sr + hq * a.q.sh + 16 * hh);
  State<DH> st;
  st.clear();
  for (int j = 0; j < edges; ++j) {
    const TileAt x = look_up(a, p, edge_at(j));
    Keys<DH> k;
    Vals<DH> v;
    load_keys<DH>(a, x.at, col, hh, k);
    load_vals<DH>(a, x.at, col, hh, v);
    const int ke = __builtin_amdgcn_readfirstlane(a.pool.ke[x.at]), ve = __builtin_amdgcn_readfirstlane(a.pool.ve[x.at]);
    attend<DH, QF>(st, q.scores(k), v, score_factor(q.fac, ke), ve, Edge{}, p.sight, x.tile * 32, pos);
  }

  if (whole > 0) {  // uniform over the workgroup
    // tile j's pool number, and 2^ke (a float) with ve in its low byte: lane
    // j % 64 of one of two banks
    int at0 = 0, at1 = 0, ex0 = 0, ex1 = 0;
    auto fill = [&](int c) {  // tiles 64 c .. into bank c % 2
      const int j = 64 * c + lane;
      int at = 0, e = 0;
      if (j < whole) {
        at = look_up(a, p, whole_at(j)).at;
        e = (int)(__float_as_uint(pow2i(a.pool.ke[at])) | (uint8_t)a.pool.ve[at]);
      }
      at0 = c & 1 ? at0 : at;
      ex0 = c & 1 ? ex0 : e;
      at1 = c & 1 ? at : at1;
      ex1 = c & 1 ? e : ex1;
    };
    fill(0);
    fill(1);
    auto of = [](int x0, int x1, int j) {
      const int y0 = __builtin_amdgcn_readlane(x0, j & 63), y1 = __builtin_amdgcn_readlane(x1, j & 63);
      return j >> 6 & 1 ? y1 : y0;
    };
    // this lane's byte offset inside a tile, for each piece this wave stages
    const bool stager = w < STAGERS;
    uint32_t goff[PPW];
#pragma unroll
    for (int x = 0; x < PPW; ++x) {
      const int pc = w * PPW + x;
      goff[x] = pc < KP ? 1024 * pc + (hh * 32 + slot_of_row(col)) * 16 : 1024 * (pc - KP) + col * 32 + 16 * hh;
    }
    auto issue = [&](int slot, int j) {
      const long long at = of(at0, at1, min(j, whole - 1));
      if (stager) {  // uniform over the wave
#pragma unroll
        for (int x = 0; x < PPW; ++x) {
          const int pc = w * PPW + x;
          const uint8_t* t = (pc < KP ? a.pool.k : a.pool.v) + at * (32 * DH);
          __builtin_amdgcn_global_load_lds((const void*)(t + goff[x]), (lds_void*)&ring[slot][pc][0], 16, 0, 0);
        }
      }
    };
#pragma unroll
    for (int i = 0; i < D; ++i) issue(i, i);

    constexpr int SQ = Query<DH, QF>::STEPS;
    Keys<DH> kf;
    auto read_k = [&](int slot) {
#pragma unroll
      for (int x = 0; x < KP; ++x) kf.r[x] = ring[slot][x][lane];
    };
    // a tile's factor of the scores, and whether its scores or its values'
    // exponent go beyond what the state refers to
    auto factor = [&](int ex) { return fmaxf(q.fac * __int_as_float(ex & 0x7f800000), 0x1p-126f); };
    auto beyond = [&](float mx, float f, int ex) { return __any(fmaf(mx, f, -st.m) > P_TOP) || (int8_t)ex > st.E; };
    f32x16 sa, sb;
    wait_vmcnt_lds<(D - 4) * PPW>();  // pairs 0 and 1
    __builtin_amdgcn_s_barrier();
    read_k(0);
    sa = q.scores(kf);
    int ex = of(ex0, ex1, 0);  // of the current tile
    float f = factor(ex);
    bool far;
    {
      float mx = sa[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) mx = fmaxf(mx, sa[r]);
      far = beyond(mx, f, ex);
    }
    read_k(1);  // of a single tile: a repeat of it
    int slot = 0;  // i % D
    // tile i: scores s in, the next tile's out; its values in the ring's slot
    auto step = [&](const f32x16& s, f32x16& sn, int i) {
      if (far) {
        st.follow(s, f);
        st.reach((int8_t)ex);
      }
      const float vs = value_factor((int8_t)ex, st.E);
      const int s1 = slot + 1 == D ? 0 : slot + 1, s2 = s1 + 1 == D ? 0 : s1 + 1;
      const int exn = of(ex0, ex1, min(i + 1, whole - 1));
      const float fn = factor(exn);
      float pr[16], part[4], mx = 0.f;
      u32x4 ph[2], pl[2];  // halves of the lane's slots
      Vals<DH> v;
      // softmax of slot r: the sum as a tree over the 16
      auto prob = [&](int r) {
        pr[r] = __builtin_amdgcn_exp2f(fmaf(s[r], f, -st.m));
        float x = pr[r];
        int level = 0;
#pragma unroll
        for (; r >> level & 1; ++level) x = part[level] + x;
        if (level == 4) st.l += x;
        else part[level] = x;
        if (r & 1) {
          const f16x2 hi = __builtin_convertvector(f32x2{pr[r - 1], pr[r]}, f16x2);
          ph[r / 8][r / 2 % 4] = __builtin_bit_cast(uint32_t, hi);
          if constexpr (probs_split(QF))
            pl[r / 8][r / 2 % 4] =
                __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{pr[r - 1] - (float)hi.x, pr[r] - (float)hi.y}, f16x2));
        }
      };
      f32x16 lo = f32x16(0.f);
      sn = f32x16(0.f);
      u32x4 k16 = zero_u4();
#pragma unroll
      for (int g = 0; g < SQ; ++g) {
        if (QF != Q_FP8 && (QF != Q_SPLIT || g % 2 == 0)) k16 = Query<DH, QF>::convert(g, kf);
        q.step(g, kf, k16, sn, lo);
#pragma unroll
        for (int x = g * DB / SQ; x < (g + 1) * DB / SQ; ++x) v.r[x] = ring[slot][KP + x][lane];
#pragma unroll
        for (int r = g * 16 / SQ; r < (g + 1) * 16 / SQ; ++r) prob(r);
        __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (QF == Q_SPLIT) sn += lo;
      __builtin_amdgcn_s_setprio(1);
      constexpr int PL = probs_split(QF) ? 2 : 1, S2 = 2 * DB * PL;  // O += V P: half, dims, part
      constexpr int S3 = S2 - 2;                                     // the maximum is there two MFMAs before the end
      u32x4 v16 = zero_u4();
#pragma unroll
      for (int g = 0; g < S2; ++g) {
        const int h = g / (DB * PL), d = g / PL % DB;
        if (g % PL == 0) v16 = __builtin_bit_cast(u32x4, cvt8(v.r[d][2 * h], v.r[d][2 * h + 1], vs));
        st.o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(as_f16x8(v16), as_f16x8(g % PL ? pl[h] : ph[h]), st.o[d], 0, 0, 0);
        if (g < KP) kf.r[g] = ring[s2][g][lane];
        if (g < S3) {
#pragma unroll
          for (int y = g * 16 / S3; y < (g + 1) * 16 / S3; ++y) mx = y ? fmaxf(mx, sn[y]) : sn[0];
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      __builtin_amdgcn_s_setprio(0);
      far = beyond(mx, fn, exn);
      f = fn;
      ex = exn;
      slot = s1;
    };
    for (int i = 0;; i += 2) {
      // every tile that is still to be issued, and the current ones, are in the banks
      if ((i & 63) == 0 && i > 0) fill((i >> 6) + 1);
      step(sa, sb, i);
      if (i + 1 >= whole) break;
      step(sb, sa, i + 1);
      if (i + 2 >= whole) break;
      wait_vmcnt_lds<(D - 6) * PPW>();
      __builtin_amdgcn_s_barrier();
      const int s0 = slot >= 2 ? slot - 2 : slot + D - 2;
      issue(s0, i + D);
      issue(s0 + 1, i + 1 + D);
    }
    wait_vmcnt_lds<0>();
  }
  const bool hurt = __any(p.bad);
  constexpr int CH = DH / 4, RPI = 64 / CH;  // 16-byte chunks of a row, rows per wave-wide store
  const long long prow = ((long long)p.u * a.pool.Hkv + p.hk) * R + row0;
  float* buf = reinterpret_cast<float*>(lds) + w * 32 * DH;
  __syncthreads();  // every wave has left the ring
  float l = st.l + __shfl_xor(st.l, 32, 64);
  if (hurt) l = __builtin_nanf("");
  put_rows<DH>(st, col, hh, R - row0, buf);
  auto live = [&](int r) { return row0 + r < R && (count >= a.nodes || (row0 + r) % a.nodes < count); };
  if (hh == 0 && live(col)) *reinterpret_cast<float2*>(a.part_ml + (prow + col) * 2) = out_sums(st.m, l);
#pragma unroll 4
  for (int n = 0; n < 32 / RPI; ++n) {
    const int r = n * RPI + lane / CH, c = lane % CH;
    if (live(r))
      *reinterpret_cast<float4*>(a.part_o + (prow + r) * DH + 4 * c) =
          *reinterpret_cast<const float4*>(buf + r * DH + 4 * (c ^ (r & 7)));
  }
}

// Joins a row's units and the nodes of its own root path: a thread holds 4 dims
// of a head of one node.  SG groups of threads share a head where there are few
// rows: group g takes units and nodes g, g + SG, .., and they meet in LDS.  What
// a group needs is asked for before any of it is used.
template <int DT, int SG>
__global__ __launch_bounds__(256) void paged_combine_kernel(PagedAttn a) {
  constexpr int TB = SG == 1 ? 2 : 8;  // units at a time
  constexpr int TN = 4;                // nodes at a time
  __shared__ float4 so[SG > 1 ? 256 : 1];
  __shared__ float2 sml[SG > 1 ? 256 : 1];
  const int dh = a.pool.dh, quads = dh / 4, heads = 256 / SG / quads;  // heads of a workgroup
  const int b = blockIdx.x / a.stride, i = blockIdx.x % a.stride;
  const int G = a.Hq / a.pool.Hkv, R = G * a.nodes;
  const int grp = SG == 1 ? 0 : threadIdx.x / (256 / SG), t = SG == 1 ? threadIdx.x : threadIdx.x % (256 / SG);
  const int h = min((int)blockIdx.y * heads + t / quads, a.Hq - 1), d = t % quads * 4, hk = h / G;
  const bool mine = blockIdx.y * heads + t / quads < a.Hq;
  if (i >= a.nodes) {  // uniform: a row of the operand behind the nodes
    if (a.out_ks && grp == 0 && mine) store_row<DT>(a, b, i, h, d, make_float4(0.f, 0.f, 0.f, 0.f));
    return;
  }
  const uint64_t anc = anc_of(a, b, i);
  const int2 un = a.units > 0 ? a.first_unit[b] : make_int2(0, 0);
  bool bad = false;
  const int len = checked_len(a.tab, b, &bad);
  int count = a.counts ? a.counts[b] : a.nodes;
  const float4 q = query_quad<DT>(a, b * a.q.sb + i * a.q.sr + h * a.q.sh + d);
  if (count < 0 || count > a.nodes) bad = true, count = min(max(count, 0), a.nodes);
  if (bad && a.status && threadIdx.x == 0) atomicOr(a.status, PAGED_BAD_LENGTH);
  const bool live = i < count;
  if (!live && a.out_ks == 0) return;  // uniform
  float4 out = make_float4(0.f, 0.f, 0.f, 0.f);
  if (live) {
    float m = -INFINITY, l = 0.f;
    float4 o = out;
    // a sequence without tiles has no units (and nobody wrote their place)
    const int units = seq_tiles(len, a.cut).n > 0 ? un.y : 0;
    const long long row = ((long long)un.x * a.pool.Hkv + hk) * R + (h % G) * a.nodes + i;
    const long long step = (long long)a.pool.Hkv * R;
    float2 ml[TB];
    float4 ou[TB];
    auto ask = [&](int s) {
#pragma unroll
      for (int x = 0; x < TB; ++x)
        if (s + x * SG < units) {  // uniform over the group
          const long long at = row + (s + x * SG) * step;
          ml[x] = *reinterpret_cast<const float2*>(a.part_ml + at * 2);
          ou[x] = *reinterpret_cast<const float4*>(a.part_o + at * dh + d);
        }
    };
    RootPath<DT, TN> path;
    ask(grp);
    path.start(a, b, hk, d, anc, SG == 1 ? ~0ull : 0x1111111111111111ull << grp, depth_of(anc, i), len);
    for (int s = grp; s < units; s += TB * SG) {
      if (s != grp) ask(s);
      float mn = m;
#pragma unroll
      for (int x = 0; x < TB; ++x)
        if (s + x * SG < units && !(ml[x].x == NO_MAX && ml[x].y == 0.f)) mn = fmaxf(mn, ml[x].x);
      if (mn == -INFINITY) continue;  // no slot of them is seen
      const float al = __builtin_amdgcn_exp2f(m - mn);
      l *= al;
      o.x *= al, o.y *= al, o.z *= al, o.w *= al;
#pragma unroll
      for (int x = 0; x < TB; ++x)
        if (s + x * SG < units) {
          const float e = __builtin_amdgcn_exp2f(ml[x].x - mn);
          l += e * ml[x].y;
          o.x += e * ou[x].x, o.y += e * ou[x].y, o.z += e * ou[x].z, o.w += e * ou[x].w;
        }
      m = mn;
    }
    path.add(a, q, quads, m, l, o);
    if constexpr (SG > 1) {
      so[threadIdx.x] = o;
      sml[threadIdx.x] = make_float2(m, l);
      __syncthreads();
      if (grp == 0) {
        float mn = m;
#pragma unroll
        for (int g = 1; g < SG; ++g) mn = fmaxf(mn, sml[g * (256 / SG) + t].x);
        const float al = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
        l *= al;
        o.x *= al, o.y *= al, o.z *= al, o.w *= al;
#pragma unroll
        for (int g = 1; g < SG; ++g) {
          const float2 x = sml[g * (256 / SG) + t];
          const float4 v = so[g * (256 / SG) + t];
          const float e = x.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x.x - mn);
          l += e * x.y;
          o.x += e * v.x, o.y += e * v.y, o.z += e * v.z, o.w += e * v.w;
        }
      }
    }
    out = row_output(l, o, bad);
  }
  if (grp == 0 && mine) store_row<DT>(a, b, i, h, d, out);
}

}  // namespace

constexpr int UNIT_LEAST = 8;  // tiles: two for each of a workgroup's four waves

int paged_plan(PagedAttn& a, int max_length) {
  const int R = a.Hq / a.pool.Hkv * a.nodes;
  // tiles of a sequence: all, or those that window - 1 slots can touch and the sinks
  long long most = ((long long)max_length + 31) >> 5;
  if (a.cut.window)
    most = std::min(most, ((long long)a.cut.window + 30) / 32 + 1 + ((long long)a.cut.sinks + 31) / 32);
  if (most * a.batch > 0x7fffffffLL) return -1;
  // The wide kernel where a KV head has more than two row tiles and either half
  // of the CUs get a whole sequence each (32 x 61 nodes of 4 x 8 heads over 512
  // slots: 36 us against 58, 8 of them 24 against 22), or its units are long: at
  // least 32 tiles for each of the 256 workgroups that then fill the chip.
  const int nw = R > 128 ? 8 : 4, wide_blocks = (R + 32 * nw - 1) / (32 * nw), thin_blocks = (R + 15) / 16;
  const long long whole = (long long)a.batch * a.pool.Hkv * wide_blocks;
  a.wide = R > 64 && (whole >= 128 || most * whole >= 32 * 256) ? nw : 0;
  // Row tiles of 16 where one holds all rows, and where all workgroups fit the
  // chip at once, as a wave then has half of the work: 61 nodes of 4 heads over
  // 500 slots 8 us against 10 (256 workgroups), over 2077 13 against 12 (1152).
  const long long by_len = (long long)a.batch * ((most + UNIT_LEAST - 1) / UNIT_LEAST);
  a.thin = R <= 16 || by_len * a.pool.Hkv * thin_blocks <= 1024;
  // One workgroup of eight waves for all of a (sequence, KV head), which reads
  // about 100 GB/s: up to 72 tiles while that leaves half of the CUs idle (a token
  // over 2077 slots 12.5 us against 7 + 5 and a second launch, over 4096 18
  // against 7 + 5), else up to 160 (16 chains over up to 2048 slots 14 us against
  // 13 + 5, 16 tokens with a window of 4096 28 against 26 + 5).
  const long long wgs = (long long)a.batch * a.pool.Hkv;
  a.fused = R <= 16 && most <= (wgs < 128 ? 72 : 160);
  const int streams = a.pool.Hkv * (a.wide ? wide_blocks : a.thin ? thin_blocks : (R + 31) / 32);
  // workgroups that fit the 256 CUs at once
  a.cut.target = std::max(1, (a.thin ? 1024 : a.wide == 8 ? 256 : 512) / streams);
  a.cut.least = UNIT_LEAST;
  a.cut.full = a.wide ? 0 : a.thin ? 64 : 32;
  // units of a sequence of n tiles: ceil(n / per) with per >= least and >= all tiles / target
  a.units = a.fused ? 0 : (int)std::min<long long>(by_len, (long long)a.cut.target + a.batch);
  return (a.units + 8LL) * streams <= PAGED_MAX_GROUPS ? 0 : -1;
}

size_t paged_workspace(PagedAttn& a, void* base) {
  const size_t rows = (size_t)a.units * a.Hq * a.nodes;
  a.part_o = static_cast<float*>(base);
  a.part_ml = a.part_o + rows * a.pool.dh;
  a.first_unit = reinterpret_cast<int2*>(a.part_ml + rows * 2);
  return rows * (a.pool.dh + 2) * sizeof(float) + (a.units > 0 ? a.batch * sizeof(int2) : 0);
}

template <int DH, int QF>
static void launch_tiles(const PagedAttn& a, dim3 grid, hipStream_t s) {
  if (a.wide == 8) hipLaunchKernelGGL((paged_wide_kernel<DH, QF == Q_BF16 ? Q_FP8 : QF, 8>), grid, dim3(512), 0, s, a);
  else if (a.wide) hipLaunchKernelGGL((paged_wide_kernel<DH, QF == Q_BF16 ? Q_FP8 : QF, 4>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((paged_attention_kernel<DH, QF>), grid, dim3(256), 0, s, a);
}

template <int DH>
static void launch_form(const PagedAttn& a, dim3 grid, hipStream_t s) {
  if (a.q_lo.p || a.dtype == PT_F32) launch_tiles<DH, Q_SPLIT>(a, grid, s);
  else if (a.dtype == PT_F16) launch_tiles<DH, Q_F16>(a, grid, s);
  else launch_tiles<DH, Q_BF16>(a, grid, s);
}

template <int DT>
static void launch_combine(const PagedAttn& a, bool few, hipStream_t s) {
  const int rows = a.batch * a.stride, threads = a.Hq * (a.pool.dh / 4);
  if (few) hipLaunchKernelGGL((paged_combine_kernel<DT, 4>), dim3(rows, (threads + 63) / 64), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((paged_combine_kernel<DT, 1>), dim3(rows, (threads + 255) / 256), dim3(256), 0, s, a);
}

hipError_t launch_paged_attention(const PagedAttn& a, hipStream_t s) {
  const int R = a.Hq / a.pool.Hkv * a.nodes, rows = a.wide ? 32 * a.wide : 32;
  if (a.pool.dh != 64 && a.pool.dh != 128) return hipErrorInvalidValue;
  if (a.thin && (a.fused || a.units > 0)) {
    const hipError_t e = launch_paged_thin(a, s);
    if (e != hipSuccess || a.fused) return e;
  } else if (a.units > 0) {
    const long long wgs = ((long long)a.units * a.pool.Hkv + 7) / 8 * 8 * ((R + rows - 1) / rows);
    if (a.pool.dh == 128) launch_form<128>(a, dim3((unsigned)wgs), s);
    else launch_form<64>(a, dim3((unsigned)wgs), s);
  }
  // Four groups a head while that leaves at most four workgroups for each CU (a
  // chain of 61 nodes of 32 heads 10 us against 16, 40 nodes of a tree 5.3 against
  // 6.0; 4 chains 27 against 24), of fp32 trees, whose groups take more registers,
  // two (61 nodes 7.9 against 5.6; a chain's long paths gain all the same: 12.5
  // against 17.8).
  const int most = a.dtype == PT_F32 && a.anc ? 512 : 1024;
  const bool few = (long long)a.batch * a.stride * a.Hq * (a.pool.dh / 4) <= most * 64;
  if (a.dtype == PT_F32) launch_combine<PT_F32>(a, few, s);
  else if (a.dtype == PT_F16) launch_combine<PT_F16>(a, few, s);
  else launch_combine<PT_BF16>(a, few, s);
  return hipGetLastError();
}

}  // namespace griffin

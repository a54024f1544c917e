// Device side of the paged attention that its kernels share: which tiles a
// sequence's nodes see and how a call's work is cut, conversions of stored
// numbers, and the nodes of a row's own root path.
#pragma once

#include "griffin_internal.h"
#include <type_traits>

#include "paged.h"

namespace griffin {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
struct KeyPair {
  u32x4 a, b;
};
__device__ __forceinline__ f16x8 as_f16x8(const u32x4& v) { return __builtin_bit_cast(f16x8, v); }

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

// Sum over the lanes that hold sequences (uniform; whole waves call these).
__device__ __forceinline__ int lanes_sum(int n, int batch) {
  for (int o = 1; o < 64 && o < batch; o <<= 1) n += __shfl_xor(n, o, 64);
  return __builtin_amdgcn_readfirstlane(n);
}

// The sequence of unit u: {sequence (-1: none), split, splits}.  A unit holds
// at most `per` tiles, and a sequence's units the same number each to one;
// per is at least ceil(all tiles / target), and rises for a few steps while
// the sequences' last units bring their number above the target (workgroups
// that do not fit the chip at once cost a second round: 18.5 -> 14.1 us for 16
// sequences of up to 2048 slots).
struct UnitAt {
  int b, split, n;
};
__device__ UnitAt unit_at(const PagedAttn& a, int u) {
  const int lane = threadIdx.x & 63;
  bool bad = false;
  auto tiles = [&](int b) { return b < a.batch ? seq_tiles(checked_len(a.tab, b, &bad), a.cut).n : 0; };
  const int own = tiles(lane);
  uint32_t total = lanes_sum(own, a.batch);
  for (int b0 = 64; b0 < a.batch; b0 += 64) total += lanes_sum(tiles(b0 + lane), 64);
  // half the target while units are short: a unit's start and join cost more
  // than what the second workgroup of a CU hides
  const uint32_t target = total >= (uint32_t)a.cut.target * a.cut.full ? a.cut.target : (a.cut.target + 1) / 2;
  uint32_t per = max((uint32_t)a.cut.least, (total + target - 1) / target);
  for (int i = 0; i < 4; ++i) {
    uint32_t units = 0;
    for (int b0 = 0; b0 < a.batch; b0 += 64)
      units += lanes_sum(((b0 ? tiles(b0 + lane) : own) + per - 1) / per, b0 ? 64 : a.batch);
    if (units <= target) break;
    per += (per * (units - target) + target - 1) / target;
  }
  int first = 0;
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    const int n = ((b0 ? tiles(b0 + lane) : own) + per - 1) / per;
    int end = n;  // inclusive sum over the lanes
    for (int o = 1; o < 64 && o < a.batch; o <<= 1) {
      const int y = __shfl_up(end, o, 64);
      if (lane >= o) end += y;
    }
    const unsigned long long in = __ballot(u >= first + end - n && u < first + end);
    if (in) {
      const int l = __builtin_ctzll(in);
      return {b0 + l, u - first - __builtin_amdgcn_readlane(end - n, l), __builtin_amdgcn_readlane(n, l)};
    }
    first += __builtin_amdgcn_readlane(end, 63);
  }
  return {-1, 0, 0};
}

// 8 e4m3 of two words as fp16 or bf16 (both exact), times 2^e of the factor `s`
__device__ __forceinline__ f16x8 cvt8(uint32_t a, uint32_t b, float s) {
  const f16x2 p = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, s, false), q = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, s, true);
  const f16x2 r = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, s, false), t = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, s, true);
  return f16x8{p.x, p.y, q.x, q.y, r.x, r.y, t.x, t.y};
}
__device__ __forceinline__ bf16x8 cvt8_bf16(uint32_t a, uint32_t b) {
  const bf16x2 p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, false), q = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, true);
  const bf16x2 r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, false), t = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, true);
  return bf16x8{p.x, p.y, q.x, q.y, r.x, r.y, t.x, t.y};
}

// nodes that node i sees, and its position behind the cached slots
__device__ __forceinline__ uint64_t anc_of(const PagedAttn& a, int b, int i) {
  return a.anc ? a.anc[(long long)b * a.stride + i] & (~0ull >> (64 - a.nodes)) : (2ull << i) - 1;
}
__device__ __forceinline__ int depth_of(uint64_t anc, int i) { return __builtin_popcountll(anc & ~(1ull << i)); }

constexpr float NO_MAX = -3e38f;  // reference of a row that has seen no key
// fp16 holds steps of 2^-24 and ends at 2^16.  A row's largest probability
// stands at 2^P_LIFT or above and follows the scores up to 2^P_TOP, so that what
// is rounded away is at most 2^-(25 + P_LIFT) of it: a lift of 10 made references
// rise more often (8 x 61 nodes over 16384 slots 145 us against 142), one of 0
// loses many small weights beside a large one.  Values of the largest exponent
// met, E, stand at 2^V_LIFT times their bytes (at most 448): bytes are multiples
// of 2^-9, so that tiles down to E - 21 are exact.
constexpr int P_LIFT = 8, P_TOP = 15, V_LIFT = 6;
static_assert(PAGED_E_MIN - V_LIFT - P_LIFT >= -126, "pow2i");
__device__ __forceinline__ float value_factor(int ve, int E) { return pow2i(ve - E + V_LIFT); }
// A wave's result for the join: the lifts taken out
__device__ __forceinline__ float out_factor(int E) { return pow2i(E - V_LIFT - P_LIFT); }
__device__ __forceinline__ float2 out_sums(float m, float l) { return make_float2(m + P_LIFT, l * pow2i(-P_LIFT)); }

// How q enters the matrix cores, by its type and the kernel:
//   Q_BF16   bf16 as it is, keys converted to bf16
//   Q_FP8    bf16 as two e4m3 parts (4 + 4 bits, exact down to 2^-21 of the row's largest value), keys
//            not converted at all: for waves with many tiles, as splitting q costs what converting
//            the keys of a dozen tiles does
//   Q_F16    fp16 as it is
//   Q_SPLIT  fp32 (or bf16 hi + lo) as two fp16 parts
enum QueryForm : int { Q_BF16, Q_FP8, Q_F16, Q_SPLIT };

constexpr bool probs_split(int qf) { return qf == Q_F16 || qf == Q_SPLIT; }  // probabilities as two fp16 parts

// The exponent of a row's largest value; subnormal rows stay near zero,
// infinite ones infinite.
__device__ __forceinline__ int scale_exponent(float mx) {
  return min(max((int)(__float_as_uint(mx) >> 23) - 127, -110), 118);
}

// Dims at + STEP x + 8 h .. of a query row, bf16 (with SPLIT: plus its low part, or
// fp32).  One block per type and alignment, so that all loads are in flight at
// once.  Returns the largest magnitude.
template <int NX, int NH, int STEP, bool SPLIT>
__device__ __forceinline__ float load_query(const PagedAttn& p, long long at, float (&v)[NX][NH][8]) {
  if (!SPLIT || p.q_lo.p) {
    auto rows = [&](const void* q, auto vec, u32x4(&w)[NX][NH]) {
#pragma unroll
      for (int x = 0; x < NX; ++x)
#pragma unroll
        for (int h = 0; h < NH; ++h) w[x][h] = load8_raw(q, at + STEP * x + 8 * h, decltype(vec)::value);
    };
    u32x4 w[NX][NH], y[SPLIT ? NX : 1][NH];
    if (p.q.vec) {
      rows(p.q.p, std::true_type{}, w);
      if constexpr (SPLIT) rows(p.q_lo.p, std::true_type{}, y);
    } else {
      rows(p.q.p, std::false_type{}, w);
      if constexpr (SPLIT) rows(p.q_lo.p, std::false_type{}, y);
    }
#pragma unroll
    for (int x = 0; x < NX; ++x)
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          v[x][h][i] = bf16_to_f32((uint16_t)(w[x][h][i / 2] >> (16 * (i & 1))));
          if constexpr (SPLIT) v[x][h][i] += bf16_to_f32((uint16_t)(y[x][h][i / 2] >> (16 * (i & 1))));
        }
  } else {
    const float* f = static_cast<const float*>(p.q.p) + at;
    auto rows = [&](auto vec) {
#pragma unroll
      for (int x = 0; x < NX; ++x)
#pragma unroll
        for (int h = 0; h < NH; ++h) load8(f, STEP * x + 8 * h, PT_F32, decltype(vec)::value, v[x][h]);
    };
    if (p.q.vec) rows(std::true_type{});
    else rows(std::false_type{});
  }
  float mx = 0.f;
#pragma unroll
  for (int x = 0; x < NX; ++x)
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
      for (int i = 0; i < 8; ++i) mx = fmaxf(mx, fabsf(v[x][h][i]));
  return mx;
}

// Two values as fp16 high and low parts (22 bits)
__device__ __forceinline__ Hilo2 split_f16(float x, float y) {
  const f16x2 h = __builtin_convertvector(f32x2{x, y}, f16x2);
  const f16x2 l = __builtin_convertvector(f32x2{x - (float)h.x, y - (float)h.y}, f16x2);
  return {__builtin_bit_cast(uint32_t, h), __builtin_bit_cast(uint32_t, l)};
}

// A row tile's queries in two fp16 parts, as the waves of a workgroup share
// them: a thread takes 8 dims of a row, so that whole rows are read together and
// split once.  (In the operands' order each wave's loads touch every line of the
// fp32 rows many times: 61 nodes of 32 heads over 1024 slots 17 us against 12.
// 16-bit rows, which are operands as they stand, are read so: 0.5 us less than
// through LDS.)  Chunk c of row r stands at c ^ r.
template <int DH, int ROWS>
struct SplitRows {
  static constexpr int CQ = DH / 8;
  u32x4 part[2][ROWS][CQ];
  float fac[ROWS];  // the scores' scale in the log2 domain, and the power of two that a row was scaled by

  // by all threads; at(r): where row r starts.  Ends with a barrier.
  template <class At>
  __device__ __forceinline__ void fill(const PagedAttn& a, At at) {
    for (int i = threadIdx.x; i < ROWS * CQ; i += blockDim.x) {
      const int r = i / CQ, c = i % CQ, put = c ^ (r % CQ);
      float v[1][1][8];
      float mx = load_query<1, 1, 0, true>(a, at(r) + 8 * c, v);
#pragma unroll
      for (int s = CQ / 2; s > 0; s >>= 1) mx = fmaxf(mx, __shfl_xor(mx, s, 64));
      const int ex = scale_exponent(mx);
      const float f = pow2i(8 - ex);  // the row's largest value to [2^8, 2^9)
      u32x4 hi, lo;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const Hilo2 x = split_f16(v[0][0][2 * e] * f, v[0][0][2 * e + 1] * f);
        hi[e] = x.hi;
        lo[e] = x.lo;
      }
      part[0][r][put] = hi;
      part[1][r][put] = lo;
      if (c == 0) fac[r] = a.scale_log2 * pow2i(ex - 8);
    }
    __syncthreads();
  }
  __device__ __forceinline__ u32x4 get(int x, int r, int c) const { return part[x][r][c ^ (r % CQ)]; }
};

// A score's factor on a tile: never 0, which times a masked -inf would be a NaN.
__device__ __forceinline__ float score_factor(float fac, int ke) { return fmaxf(fac * pow2i(ke), 0x1p-126f); }

// The places of a tile that a row does not see, for lane half hh.
struct Sight {
  int len, window, sinks;
  __device__ __forceinline__ bool of(int slot, int pos) const {
    return slot < len && (window == 0 || slot > pos - window || slot < sinks);
  }
};

struct Edge {
  static constexpr bool value = true;
};
struct Whole {
  static constexpr bool value = false;
};

// Where a workgroup works: unit u (sequence b, the list's tiles [i0, i1)) of KV
// head hk, row block rb.
struct Place {
  int u, b, hk, rb, i0, i1;
  SeqTiles seq;
  Sight sight;
  bool bad;
};
// XCD-aware decode of the workgroup's number: workgroups go round-robin over
// the 8 XCDs, so the row blocks of one (unit or sequence, KV head) get the same
// id % 8 and share its L2.
__device__ __forceinline__ int decode_group(const PagedAttn& a, int blocks, Place& p) {
  const int id = blockIdx.x, rest = id >> 3;
  p.rb = rest % blocks;
  const int st = (rest / blocks) * 8 + (id & 7);
  p.hk = st % a.pool.Hkv;
  return st / a.pool.Hkv;
}
// Where row `row` of the KV head's starts in q (behind the last one: that again)
__device__ __forceinline__ long long query_row(const PagedAttn& a, const Place& p, int row) {
  const int G = a.Hq / a.pool.Hkv;
  row = min(row, G * a.nodes - 1);
  return p.b * a.q.sb + row % a.nodes * a.q.sr + (p.hk * G + row / a.nodes) * a.q.sh;
}
// All of a sequence; false: none (the grid is rounded up).
__device__ __forceinline__ bool whole_sequence(const PagedAttn& a, int blocks, Place& p) {
  p.b = decode_group(a, blocks, p);
  if (p.b >= a.batch) return false;  // uniform
  p.u = 0;
  p.bad = false;
  const int len = checked_len(a.tab, p.b, &p.bad);
  p.seq = seq_tiles(len, a.cut);
  p.i0 = 0;
  p.i1 = p.seq.n;
  p.sight = Sight{len, a.cut.window, a.cut.sinks};
  return true;
}
__device__ __forceinline__ bool place_of(const PagedAttn& a, int blocks, Place& p) {
  p.u = decode_group(a, blocks, p);
  const UnitAt at = unit_at(a, p.u);
  if (at.b < 0) return false;  // uniform
  p.b = at.b;
  p.bad = false;
  const int len = checked_len(a.tab, at.b, &p.bad);
  p.seq = seq_tiles(len, a.cut);
  p.i0 = (int)((long long)p.seq.n * at.split / at.n);
  p.i1 = (int)((long long)p.seq.n * (at.split + 1) / at.n);
  p.sight = Sight{len, a.cut.window, a.cut.sinks};
  // the joining kernel finds a sequence's units here
  if (at.split == 0 && p.hk == 0 && p.rb == 0 && threadIdx.x == 0) a.first_unit[at.b] = make_int2(p.u, at.n);
  return true;
}

// The tile that entry i of a sequence's list is, and its number in the pool.
struct TileAt {
  int tile, at;
};
__device__ __forceinline__ TileAt look_up(const PagedAttn& a, Place& p, int i) {
  TileAt t;
  t.tile = i < p.seq.sink ? i : i - p.seq.sink + p.seq.lo;
  int page = a.tab.pages[(long long)p.b * a.tab.stride + t.tile / a.pool.tpp];
  if (page < 0 || page >= a.pool.n_pages) {
    p.bad = true;
    if (a.status) atomicOr(a.status, PAGED_BAD_PAGE);
    page = 0;
  }
  t.at = (page * a.pool.Hkv + p.hk) * a.pool.tpp + t.tile % a.pool.tpp;
  return t;
}

// Sum over each 16 lanes, in all of them, by lane moves inside the vector unit
// (through LDS the join of 64 x 61 nodes of 32 heads took 60 us instead of 55)
template <int CTRL>
__device__ __forceinline__ float moved(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float row_sum(float x) {
  x += moved<0xb1>(x);   // pairs
  x += moved<0x4e>(x);   // quads
  x += moved<0x141>(x);  // mirrored halves of 16
  return x + moved<0x140>(x);
}
__device__ __forceinline__ float xor16(float x) {
  return __int_as_float(__builtin_amdgcn_ds_swizzle(__float_as_int(x), 0x401f));
}

// Adds the nodes of a row's own root path (bits anc, of a row at `dep` nodes
// behind the `len` cached slots) to the running softmax (m, l, o) of 4 dims (d)
// of head h; the head's threads are neighbours.  TN: nodes at a time.  start()
// asks for the first ones, so that they are under way while something else is
// done.
template <int DT, int TN>
struct RootPath {
  typename QuadOf<DT>::type k4[TN], v4[TN];
  uint64_t path, anc;  // all of the path; what is left of this thread's part of it
  long long kb, vb;
  int dep, len, seen;
  bool any;

  __device__ __forceinline__ void ask(const PagedAttn& a) {
    seen = 0;
#pragma unroll
    for (int x = 0; x < TN; ++x) {
      if (!anc) break;  // uniform
      const int j = __builtin_ctzll(anc), r = __builtin_popcountll(path & ((1ull << j) - 1));
      anc &= anc - 1;
      if (!a.cut.window || dep - r < a.cut.window || (long long)len + r < a.cut.sinks) seen |= 1 << x;
      k4[x] = load_quad<DT>(a.k.p, kb + j * a.k.sr, a.k.vec);
      v4[x] = load_quad<DT>(a.v.p, vb + j * a.v.sr, a.v.vec);
    }
  }
  // part: the bits of the path that are this thread's
  __device__ __forceinline__ void start(const PagedAttn& a, int b, int hk, int d, uint64_t nodes, uint64_t part, int depth, int length) {
    path = nodes;
    anc = nodes & part;
    any = anc != 0;
    dep = depth;
    len = length;
    kb = b * a.k.sb + hk * a.k.sh + d;
    vb = b * a.v.sb + hk * a.v.sh + d;
    ask(a);
  }
  __device__ __forceinline__ void add(const PagedAttn& a, const float4& q, int quads, float& m, float& l, float4& o) {
    while (any) {
      if (seen) {
        float sc[TN];
#pragma unroll
        for (int x = 0; x < TN; ++x) {
          sc[x] = 0.f;
          if (seen >> x & 1) {
            const float4 k = quad_f32<DT>(k4[x]);
            sc[x] = q.x * k.x + q.y * k.y + q.z * k.z + q.w * k.w;
          }
        }
#pragma unroll
        for (int x = 0; x < TN; ++x) sc[x] = row_sum(sc[x]);
        if (quads == 32) {  // uniform
#pragma unroll
          for (int x = 0; x < TN; ++x) sc[x] += xor16(sc[x]);
        }
        float mn = m;
#pragma unroll
        for (int x = 0; x < TN; ++x)
          if (seen >> x & 1) mn = fmaxf(mn, sc[x] *= a.scale_log2);
        const float al = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
        l *= al;
        o.x *= al, o.y *= al, o.z *= al, o.w *= al;
#pragma unroll
        for (int x = 0; x < TN; ++x)
          if (seen >> x & 1) {
            const float e = __builtin_amdgcn_exp2f(sc[x] - mn);
            const float4 v = quad_f32<DT>(v4[x]);
            l += e;
            o.x += e * v.x, o.y += e * v.y, o.z += e * v.z, o.w += e * v.w;
          }
        m = mn;
      }
      any = anc != 0;
      if (any) ask(a);
    }
  }
};

// 4 dims of a head's query as fp32
template <int DT>
__device__ __forceinline__ float4 query_quad(const PagedAttn& a, long long at) {
  if (DT == PT_F32 && a.q_lo.p) {
    float4 q = quad_f32<PT_BF16>(load_quad<PT_BF16>(a.q.p, at, a.q.vec));
    const float4 y = quad_f32<PT_BF16>(load_quad<PT_BF16>(a.q_lo.p, at, a.q.vec));
    q.x += y.x, q.y += y.y, q.z += y.z, q.w += y.w;
    return q;
  }
  return quad_f32<DT>(load_quad<DT>(a.q.p, at, a.q.vec));
}

// The output: the running softmax's quotient (0 where nothing was seen; NaN
// where `bad`), and 4 dims of it stored.
__device__ __forceinline__ float4 row_output(float l, const float4& o, bool bad) {
  const float inv = bad ? __builtin_nanf("") : l == 0.f ? 0.f : 1.f / l;
  return make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
}
template <int DT>
__device__ __forceinline__ void store_row(const PagedAttn& a, int b, int i, int h, int d, const float4& out) {
  if (a.out_ks) {
    uint16_t* dst = static_cast<uint16_t*>(a.out) + xpack_off((long long)b * a.stride + i, h * a.pool.dh + d, a.out_ks);
    const Hilo2 p0 = pack_hilo2(out.x, out.y), p1 = pack_hilo2(out.z, out.w);
    *reinterpret_cast<uint2*>(dst) = make_uint2(p0.hi, p1.hi);
    *reinterpret_cast<uint2*>(dst + XPACK_LO) = make_uint2(p0.lo, p1.lo);
    return;
  }
  const long long at = b * a.ob + i * a.orow + h * a.oh + d;
  if constexpr (DT == PT_F32) {
    float* f = static_cast<float*>(a.out) + at;
    if (a.out_vec) *reinterpret_cast<float4*>(f) = out;
    else f[0] = out.x, f[1] = out.y, f[2] = out.z, f[3] = out.w;
  } else {
    uint2 w;
    if constexpr (DT == PT_BF16) {
      w = make_uint2(pack_bf16x2(out.x, out.y), pack_bf16x2(out.z, out.w));
    } else {
      const f16x2 x = __builtin_convertvector(f32x2{out.x, out.y}, f16x2), y = __builtin_convertvector(f32x2{out.z, out.w}, f16x2);
      w = make_uint2(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, y));
    }
    uint16_t* p = static_cast<uint16_t*>(a.out) + at;
    if (a.out_vec) *reinterpret_cast<uint2*>(p) = w;
    else p[0] = w.x, p[1] = w.x >> 16, p[2] = w.y, p[3] = w.y >> 16;
  }
}

}  // namespace griffin

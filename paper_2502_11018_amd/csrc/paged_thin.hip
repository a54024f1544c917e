// Attention over the 8-bit paged cache (paged.h) in row tiles of 16 (rows: heads
// of the group x nodes): single tokens and short chains, where reading the cache
// is the work (32 tokens over up to 16384 slots: 605 MB in 110 us, 5.5 TB/s), and
// calls too short to fill the chip, where its latency is.
//
// The same products as in paged_attention.hip with v_mfma_f32_16x16x32: S^T =
// K Q^T in two groups of 16 keys, O^T += V^T P^T in groups of 16 dims.  MFMA
// row 4 g + r of key group t holds slot 8 g + 4 t + r, so that lane (row n,
// quarter g) has the scores of slots 8 g .. 8 g + 7, which are its P operand,
// and reads its values' 8 bytes for those slots.  A wave holds half of what a
// 32-row tile needs, so that four fit a SIMD and keep the loads going without
// any ahead of a tile (which measured the same), and has half of the softmax.
//
// Long sequences are cut into units of four waves that paged_combine_kernel
// joins.  Where a sequence's tiles are few (FUSED), one workgroup of eight
// waves takes all of a (sequence, KV head), joins them in LDS, adds the root
// path's nodes and writes the rows: one launch and no partial results.

#include "paged_device.h"

namespace griffin {

namespace {

template <int DH>
struct ThinKeys {
  u32x4 r[2][DH / 64];  // key group; chunks g and g + 4 of 16 dims
};
template <int DH>
struct ThinVals {
  uint2 r[DH / 16];  // slots 8 g .. 8 g + 7 of dim 16 x + n
};

template <int DH>
__device__ __forceinline__ void load_thin(const PagedAttn& a, long long at, int n, int g, ThinKeys<DH>& k, ThinVals<DH>& v) {
  const uint8_t* kp = a.pool.k + at * (32 * DH) + (g * 32 + 8 * (n >> 2) + (n & 3)) * 16;
  const uint8_t* vp = a.pool.v + at * (32 * DH) + n * 32 + 8 * g;
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int j = 0; j < DH / 64; ++j) k.r[t][j] = *reinterpret_cast<const u32x4*>(kp + 2048 * j + 64 * t);
#pragma unroll
  for (int x = 0; x < DH / 16; ++x) v.r[x] = *reinterpret_cast<const uint2*>(vp + 512 * x);
}

// Q^T operand: dims 16 (g + 4 j) + 8 h .. of row n; Q_SPLIT: fp16 parts of the
// row scaled by a power of two
template <int DH, int QF>
struct ThinQuery {
  static constexpr int J = DH / 64;
  u32x4 a[J][2], b[QF == Q_SPLIT ? J : 1][2];
  float fac;

  __device__ __forceinline__ void load(const PagedAttn& p, long long at, int g) {  // the row starts at `at`
    fac = p.scale_log2;
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) a[j][h] = load8_raw(p.q.p, at + 16 * g + 64 * j + 8 * h, p.q.vec);
  }
  __device__ __forceinline__ void take(const SplitRows<DH, 16>& rows, int n, int g) {
    fac = rows.fac[n];
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        a[j][h] = rows.get(0, n, 2 * (g + 4 * j) + h);
        b[j][h] = rows.get(1, n, 2 * (g + 4 * j) + h);
      }
  }

  __device__ __forceinline__ void scores(const ThinKeys<DH>& k, f32x4 (&s)[2]) const {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      f32x4 lo = f32x4(0.f);
      s[t] = f32x4(0.f);
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t x = k.r[t][j][2 * h], y = k.r[t][j][2 * h + 1];
          if constexpr (QF == Q_BF16) {
            s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(cvt8_bf16(x, y), as_bf16x8(a[j][h]), s[t], 0, 0, 0);
          } else {
            const f16x8 k8 = cvt8(x, y, 1.f);
            s[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k8, as_f16x8(a[j][h]), s[t], 0, 0, 0);
            if constexpr (QF == Q_SPLIT) lo = __builtin_amdgcn_mfma_f32_16x16x32_f16(k8, as_f16x8(b[j][h]), lo, 0, 0, 0);
          }
        }
      if constexpr (QF == Q_SPLIT) s[t] += lo;
    }
  }
};

// Running softmax and output: lane (n, g) holds row n's reference, its own
// slots' part of the sum, and dims 16 x + 4 g + r in o[x][r], times
// 2^(V_LIFT - E).
template <int DH>
struct ThinState {
  float m, l;
  int E;  // uniform
  f32x4 o[DH / 16];

  __device__ __forceinline__ void scale(float f) {
#pragma unroll
    for (int x = 0; x < DH / 16; ++x) o[x] *= f;
  }
};

template <int DH, int QF, class EDGE>
__device__ __forceinline__ void attend_thin(ThinState<DH>& st, f32x4 (&s)[2], ThinVals<DH>& v, float f, int ve, EDGE,
                                            const Sight& sight, int s0, int pos, int g) {
  constexpr int DB = DH / 16;
  if constexpr (EDGE::value) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (!sight.of(s0 + 8 * g + i, pos)) s[i / 4][i % 4] = -INFINITY;
  }
  float p[8], sum;
  auto probs = [&]() {
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = __builtin_amdgcn_exp2f(fmaf(s[i / 4][i % 4], f, -st.m));
    sum = ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
  };
  probs();
  if (__any(sum > pow2i(P_TOP))) {  // raise the reference towards the scores' maximum
    float mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < 8; ++i) mx = fmaxf(mx, s[i / 4][i % 4]);
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * f;
    const float mn = fmaxf(st.m, mx - P_LIFT), al = __builtin_amdgcn_exp2f(st.m - mn);
    st.m = mn;
    st.l *= al;
    st.scale(al);
    probs();
  }
  st.l += sum;
  if (ve > st.E) {  // uniform
    st.scale(pow2i(st.E - ve));
    st.E = ve;
  }
  const float vs = value_factor(ve, st.E);
  if constexpr (EDGE::value) {
    // bytes that no row sees become 0, and a NaN that only some rows see is
    // given to those (as in paged_attention.hip)
    bool nan_v = false;
    uint32_t keep[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (sight.of(s0 + 8 * g + i, sight.len)) keep[i / 4] |= 0xffu << (8 * (i % 4));
    auto nan_in = [](uint32_t y) { return (((y & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0; };
#pragma unroll
    for (int x = 0; x < DB; ++x) {
      v.r[x].x &= keep[0];
      v.r[x].y &= keep[1];
      nan_v |= nan_in(v.r[x].x) || nan_in(v.r[x].y);
    }
    if (sight.window && __any(nan_v)) {
#pragma unroll
      for (int x = 0; x < DB; ++x) {
        f16x8 is, sees;
        uint32_t w[2] = {v.r[x].x, v.r[x].y};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const bool nan = (w[i / 4] >> (8 * (i % 4)) & 0x7f) == 0x7f;
          is[i] = nan ? (_Float16)1.f : (_Float16)0.f;
          sees[i] = s[i / 4][i % 4] == -INFINITY ? (_Float16)0.f : (_Float16)1.f;
          if (nan) w[i / 4] &= ~(0xffu << (8 * (i % 4)));
        }
        const f32x4 hit = __builtin_amdgcn_mfma_f32_16x16x32_f16(is, sees, f32x4(0.f), 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (hit[r] > 0.f) st.o[x][r] = __builtin_nanf("");
        v.r[x] = make_uint2(w[0], w[1]);
      }
    }
  }
  u32x4 ph, pl;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (probs_split(QF)) {
      const Hilo2 x = split_f16(p[2 * e], p[2 * e + 1]);
      ph[e] = x.hi;
      pl[e] = x.lo;
    } else {
      ph[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{p[2 * e], p[2 * e + 1]}, f16x2));
    }
  }
#pragma unroll
  for (int x = 0; x < DB; ++x) {
    const f16x8 v8 = cvt8(v.r[x].x, v.r[x].y, vs);
    st.o[x] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v8, as_f16x8(ph), st.o[x], 0, 0, 0);
    if constexpr (probs_split(QF)) st.o[x] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v8, as_f16x8(pl), st.o[x], 0, 0, 0);
  }
}

constexpr int type_of(int qf) { return qf == Q_BF16 ? PT_BF16 : qf == Q_F16 ? PT_F16 : PT_F32; }

// The end of a workgroup that has all of a sequence's cached part of a KV head's
// rows: joined by `join(row, chunk of 4 dims, m, l, o)`, the root path's nodes
// added, and written.
template <int DH, int QF, class Join>
__device__ __forceinline__ void write_rows(const PagedAttn& a, const Place& p, int count, int live, Join join) {
  constexpr int DT = type_of(QF), CH = DH / 4;
  const int G = a.Hq / a.pool.Hkv;
  bool bad = false;
  checked_len(a.tab, p.b, &bad);
  if (count < 0 || count > a.nodes) bad = true, count = min(max(count, 0), a.nodes);
  if (bad && a.status && threadIdx.x == 0) atomicOr(a.status, PAGED_BAD_LENGTH);
  for (int i = threadIdx.x; i < live * CH; i += blockDim.x) {  // whole rows: CH divides 64
    const int r = i / CH, c = i % CH, node = r % a.nodes, h = p.hk * G + r / a.nodes, d = 4 * c;
    if (node >= count) {
      if (a.out_ks) store_row<DT>(a, p.b, node, h, d, make_float4(0.f, 0.f, 0.f, 0.f));
      continue;
    }
    const uint64_t anc = anc_of(a, p.b, node);
    const float4 q = query_quad<DT>(a, p.b * a.q.sb + node * a.q.sr + h * a.q.sh + d);
    RootPath<DT, 4> path;
    path.start(a, p.b, p.hk, d, anc, ~0ull, depth_of(anc, node), p.sight.len);
    float m, l;
    float4 o;
    join(r, c, m, l, o);
    if (m == NO_MAX && l == 0.f) m = -INFINITY;  // no slot is seen
    path.add(a, q, CH, m, l, o);
    store_row<DT>(a, p.b, node, h, d, row_output(l, o, bad));
  }
  if (a.out_ks)  // the operand's rows behind them
    for (int i = threadIdx.x; i < (a.stride - a.nodes) * G * CH; i += blockDim.x)
      store_row<DT>(a, p.b, a.nodes + i / (G * CH), p.hk * G + i / CH % G, i % CH * 4, make_float4(0.f, 0.f, 0.f, 0.f));
}

template <int DH, int QF, int NW, bool FUSED>
__global__ __launch_bounds__(64 * NW, 2) void paged_thin_kernel(PagedAttn a) {
  constexpr int CH = DH / 4;  // 16-byte chunks of a row
  __shared__ float4 so[NW][16 * CH];
  __shared__ float sm[NW][16], sl[NW][16];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, g = lane >> 4;
  const int G = a.Hq / a.pool.Hkv, R = G * a.nodes;
  Place p;
  const int blocks = FUSED ? 1 : (R + 15) / 16;
  if (!(FUSED ? whole_sequence(a, 1, p) : place_of(a, blocks, p))) return;
  const int count = a.counts ? a.counts[p.b] : a.nodes, first = 16 * p.rb, live = min(16, R - first);

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
  const int node = min(first + n, R - 1) % a.nodes;
  const int pos = a.cut.window ? p.sight.len + depth_of(anc_of(a, p.b, node), node) : 0;
  ThinQuery<DH, QF> q;
  if constexpr (QF == Q_SPLIT) {
    __shared__ SplitRows<DH, 16> rows;
    rows.fill(a, [&](int r) { return query_row(a, p, first + r); });
    q.take(rows, n, g);
  } else {
    q.load(a, query_row(a, p, first + n), g);
  }
  ThinState<DH> st;
  st.m = NO_MAX;
  st.l = 0.f;
  st.E = PAGED_E_MIN;
#pragma unroll
  for (int x = 0; x < DH / 16; ++x) st.o[x] = f32x4(0.f);
  for (int base = 0; base < mine; base += 64) {
    if (base) look(base);
    // tiles that not every row sees whole come first
    const int s0 = my_tile * 32;
    const bool edge = s0 + 32 > p.sight.len ||
                      (a.cut.window && s0 + 32 > a.cut.sinks && s0 < p.sight.len + a.nodes - a.cut.window);
    const unsigned long long all = __ballot(base + lane < mine);
    unsigned long long todo = all & __ballot(edge), rest = all & ~todo;
    auto tile = [&](auto kind, int i) {
      ThinKeys<DH> k;
      ThinVals<DH> v;
      load_thin<DH>(a, __builtin_amdgcn_readlane(my_at, i), n, g, k, v);
      f32x4 s[2];
      q.scores(k, s);
      attend_thin<DH, QF>(st, s, v, score_factor(q.fac, __builtin_amdgcn_readlane(my_ke, i)),
                          __builtin_amdgcn_readlane(my_ve, i), kind, p.sight,
                          __builtin_amdgcn_readlane(my_tile, i) * 32, pos, g);
    };
    for (; todo; todo &= todo - 1) tile(Edge{}, __builtin_ctzll(todo));
    for (; rest; rest &= rest - 1) tile(Whole{}, __builtin_ctzll(rest));
  }
  float l = st.l + __shfl_xor(st.l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  if (__any(p.bad)) l = __builtin_nanf("");  // a tile that is not there: the rows become NaN
  if (n < live) {
    const float fe = out_factor(st.E);
#pragma unroll
    for (int x = 0; x < DH / 16; ++x)
      so[w][n * CH + ((4 * x + g) ^ (n & 7))] =
          make_float4(st.o[x][0] * fe, st.o[x][1] * fe, st.o[x][2] * fe, st.o[x][3] * fe);
    const float2 ml = out_sums(st.m, l);
    if (g == 0) sm[w][n] = ml.x, sl[w][n] = ml.y;
  }
  __syncthreads();
  // the waves' results of chunk c of row r
  auto join = [&](int r, int c, float& m, float& L, float4& o) {
    m = sm[0][r];
#pragma unroll
    for (int x = 1; x < NW; ++x) m = fmaxf(m, sm[x][r]);
    L = 0.f;
    o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int x = 0; x < NW; ++x) {
      const float f = __builtin_amdgcn_exp2f(sm[x][r] - m);
      const float4 v = so[x][r * CH + (c ^ (r & 7))];
      o.x += f * v.x, o.y += f * v.y, o.z += f * v.z, o.w += f * v.w;
      L += f * sl[x][r];
    }
  };
  if constexpr (!FUSED) {
    const long long prow = ((long long)p.u * a.pool.Hkv + p.hk) * R + first;
    for (int i = threadIdx.x; i < live * CH; i += 64 * NW) {
      const int r = i / CH, c = i % CH;
      if (count < a.nodes && (first + r) % a.nodes >= count) continue;  // an absent node
      float m, L;
      float4 o;
      join(r, c, m, L, o);
      *reinterpret_cast<float4*>(a.part_o + (prow + r) * DH + 4 * c) = o;
      if (c == 0) *reinterpret_cast<float2*>(a.part_ml + (prow + r) * 2) = make_float2(m, L);
    }
  } else {
    write_rows<DH, QF>(a, p, count, live, join);
  }
}

template <int DH, int QF>
void launch_form(const PagedAttn& a, hipStream_t s) {
  const int parts = a.fused ? a.batch : a.units;  // whole sequences, or units
  const int R = a.Hq / a.pool.Hkv * a.nodes, wgs = (parts * a.pool.Hkv + 7) / 8 * 8 * ((R + 15) / 16);
  if (a.fused) hipLaunchKernelGGL((paged_thin_kernel<DH, QF, 8, true>), dim3(wgs), dim3(512), 0, s, a);
  else hipLaunchKernelGGL((paged_thin_kernel<DH, QF, 4, false>), dim3(wgs), dim3(256), 0, s, a);
}

}  // namespace

hipError_t launch_paged_thin(const PagedAttn& a, hipStream_t s) {
  const bool split = a.q_lo.p || a.dtype == PT_F32;
  if (a.pool.dh == 128) {
    if (split) launch_form<128, Q_SPLIT>(a, s);
    else if (a.dtype == PT_F16) launch_form<128, Q_F16>(a, s);
    else launch_form<128, Q_BF16>(a, s);
  } else {
    if (split) launch_form<64, Q_SPLIT>(a, s);
    else if (a.dtype == PT_F16) launch_form<64, Q_F16>(a, s);
    else launch_form<64, Q_BF16>(a, s);
  }
  return hipGetLastError();
}

}  // namespace griffin

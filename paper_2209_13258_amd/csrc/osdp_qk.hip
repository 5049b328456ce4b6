// Norms of queries and keys for each head and their rotation by position, in one pass over the qkv operator's output, and the
// pass back.  HBM bound: 4 bytes an element forward, 6 backward, against some 10 and 20 operations in fp32.
//
// A head of D elements is held by a group of kG lanes (a power of two, 16 elements to a lane), so that its sum of squares takes
// log2 kG steps between neighbouring lanes.  A lane's 16 elements are two pieces of 16 bytes, chosen so that both elements of every
// pair that is turned lie in one lane: with pairs (i, i + rotary / 2) piece i and the piece rotary / 2 elements on, interleaved
// two neighbouring pieces.  Either way lane i turns its pairs by frequencies 8 i .. 8 i + 7, and these angles serve all heads of the
// token that the lane meets: cosines and sines are worked out once for kU heads, from the position in 64 bits, and no table is read.
#include "activation.h"

#include <algorithm>
#include <cstdio>

namespace osdp {
namespace {

struct HeadsIn {
  const uint16_t *p;
  int64_t ld, hs;
};
struct HeadsOut {
  uint16_t *p;
  int64_t ld, hs;
};
struct QkSide {
  HeadsIn x, dy;       // dy: backward
  HeadsOut y;          // forward: the turned heads; backward: dx
  const void *weight;
  void *dweight;       // backward, or nullptr
  int32_t heads, chunks;  // chunks: kU head groups each
};
struct QkParams {
  QkSide side[2];
  const int64_t *positions;
  const double *freqs;
  int64_t T, units;    // units: token tiles x chunks of both sides
  float eps;
  int32_t D, slots;    // slots: lanes of a group that hold elements
  int32_t rotary, interleaved, norm, weight_f32;
  int32_t heads_log2;  // head groups of a wave; the other lane groups hold the next tokens
  float *planes;       // backward: sums of workgroups, [gridDim.x][2][D]
};

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
  const bf16x2 v = {static_cast<__bf16>(lo), static_cast<__bf16>(hi)};
  return __builtin_bit_cast(uint32_t, v);
}

template <int kCtrl>
__device__ __forceinline__ float from_lane(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), kCtrl, 0xf, 0xf, true));
}

// The sum over a group of kG lanes, in all of them.
template <int kG>
__device__ __forceinline__ float group_sum(float x) {
  if constexpr (kG >= 2) x += from_lane<0xb1>(x);   // quad_perm 1 0 3 2
  if constexpr (kG >= 4) x += from_lane<0x4e>(x);   // quad_perm 2 3 0 1
  if constexpr (kG >= 8) x += from_lane<0x141>(x);  // row_half_mirror: the other quad of the eight
  if constexpr (kG >= 16) x += from_lane<0x140>(x); // row_mirror: the other eight of the sixteen
  if constexpr (kG >= 32) x += __shfl_xor(x, 16);
  return x;
}

// What a lane holds of every head, and the angles of its token.
template <int kG>
struct Lane {
  int i, first, second;  // its slot, where its two pieces begin (elements)
  bool has_first, has_second, turns_low, turns_high;  // turns: pairs 0..3 and 4..7 of its own
  __device__ __forceinline__ void begin(const QkParams &p, int lane) {
    i = lane & (kG - 1);
    const int pairs = p.rotary / 2;
    if (!p.interleaved && i < p.rotary / 16) {
      first = 8 * i;
      second = first + pairs;
    } else {
      first = p.interleaved ? 16 * i : p.rotary + 16 * (i - p.rotary / 16);
      second = first + 8;
    }
    has_first = i < p.slots && first < p.D;
    has_second = has_first && second < p.D;
    turns_low = 8 * i < pairs;
    turns_high = 8 * i + 4 < pairs;
  }
  __device__ __forceinline__ void weights(const QkParams &p, const void *w, float (&g)[16]) const {
#pragma unroll
    for (int e = 0; e < 16; ++e) g[e] = 1.0f;
    if (!w) return;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      if (!(half ? has_second : has_first)) continue;
      const int at = half ? second : first;
      if (p.weight_f32) {
        const float4 *src = reinterpret_cast<const float4 *>(static_cast<const float *>(w) + at);
        const float4 a = src[0], b = src[1];
        const float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) g[8 * half + e] = v[e];
      } else {
        const uint4 a = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(w) + at);
        const uint32_t v[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          g[8 * half + 2 * e] = bf16_low(v[e]);
          g[8 * half + 2 * e + 1] = bf16_high(v[e]);
        }
      }
    }
  }
  __device__ __forceinline__ void angles(const QkParams &p, int64_t position, float (&c)[8], float (&s)[8]) const {
    constexpr double kTurn = 0.15915494309189533577;  // 1 / (2 pi)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      c[e] = 1.0f;
      s[e] = 0.0f;
      if (e < 4 ? !turns_low : !turns_high) continue;
      const double turns = static_cast<double>(position) * p.freqs[8 * i + e] * kTurn;
      const float rest = static_cast<float>(turns - __builtin_rint(turns));
      c[e] = __builtin_amdgcn_cosf(rest);  // (of turns)
      s[e] = __builtin_amdgcn_sinf(rest);
    }
  }
  __device__ __forceinline__ void load(const HeadsIn &h, int64_t t, int head, bool valid, uint4 &a, uint4 &b) const {
    a = b = uint4{0u, 0u, 0u, 0u};
    if (!valid) return;
    const uint16_t *row = h.p + t * h.ld + head * h.hs;
    if (has_first) a = load_global16(row + first);
    if (has_second) b = load_global16(row + second);
  }
  __device__ __forceinline__ void store(const HeadsOut &h, int64_t t, int head, bool valid, const float (&v)[16]) const {
    if (!valid) return;
    uint16_t *row = h.p + t * h.ld + head * h.hs;
    if (has_first) store_global16(row + first, uint4{pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7])});
    if (has_second) store_global16(row + second, uint4{pack2(v[8], v[9]), pack2(v[10], v[11]), pack2(v[12], v[13]), pack2(v[14], v[15])});
  }
  // v turned by the angles, or (back) by their negatives.  Elements that are not turned are left alone, whatever their neighbours hold.
  template <bool kBack>
  __device__ __forceinline__ void turn(const QkParams &p, const float (&c)[8], const float (&s_)[8], float (&v)[16]) const {
    auto pair = [&](float &a, float &b, int e) {
      const float s = kBack ? -s_[e] : s_[e], x = a, y = b;
      if (e < 4 ? turns_low : turns_high) {
        a = x * c[e] - y * s;
        b = y * c[e] + x * s;
      }
    };
    if (p.interleaved) {
#pragma unroll
      for (int e = 0; e < 8; ++e) pair(v[2 * e], v[2 * e + 1], e);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) pair(v[e], v[8 + e], e);
    }
  }
};

__device__ __forceinline__ void widen(uint4 a, uint4 b, float (&v)[16]) {
  const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    v[2 * e] = bf16_low(w[e]);
    v[2 * e + 1] = bf16_high(w[e]);
  }
}

// v times 1 / sqrt(mean v^2 + eps), over the group; the factor.
template <int kG>
__device__ __forceinline__ float normalize(const QkParams &p, float (&v)[16]) {
  auto squares = [&] {
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < 16; ++e) s = __builtin_fmaf(v[e], v[e], s);
    return group_sum<kG>(s);
  };
  float s = squares(), scale = 1.0f;
  const float per = 1.0f / static_cast<float>(p.D);
  float eps = p.eps;
  if (__builtin_expect(s == __builtin_inff(), 0)) {  // (all lanes of the group or none: 2^70 of them still fit)
    scale = 0x1p-70f;
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] *= scale;
    s = squares();
    eps = 0.0f;
  }
  const float r = rsqrtf(__builtin_fmaf(s, per, eps));
#pragma unroll
  for (int e = 0; e < 16; ++e) v[e] *= r;
  return r * scale;
}

// Where a wave's unit lies: its token tile and its head groups of one side.
template <int kG, int kU>
struct Unit {
  int which, head0;
  int64_t t;
  __device__ __forceinline__ void find(const QkParams &p, int64_t unit, int lane) {
    const int chunks = p.side[0].chunks + p.side[1].chunks;
    const int64_t tile = unit / chunks;
    int chunk = static_cast<int>(unit - tile * chunks);
    which = chunk >= p.side[0].chunks;
    if (which) chunk -= p.side[0].chunks;
    const int group = lane / kG, heads = 1 << p.heads_log2;
    t = tile * ((64 / kG) >> p.heads_log2) + (group >> p.heads_log2);
    head0 = chunk * kU * heads + (group & (heads - 1));
  }
};

template <int kG, int kU>
__global__ __launch_bounds__(256) void qk_forward_kernel(QkParams p) {
  const int lane_id = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Lane<kG> lane;
  lane.begin(p, lane_id);
  for (int64_t u = static_cast<int64_t>(blockIdx.x) * 4 + wave; u < p.units; u += static_cast<int64_t>(gridDim.x) * 4) {
    Unit<kG, kU> unit;
    unit.find(p, u, lane_id);
    const QkSide &side = p.side[unit.which];
    const int64_t position = unit.t >= p.T ? -1 : p.positions ? p.positions[unit.t] : unit.t;
    const bool row = position >= 0;
    uint4 a[kU], b[kU];
    const int step = 1 << p.heads_log2;
#pragma unroll
    for (int i = 0; i < kU; ++i)
      lane.load(side.x, unit.t, unit.head0 + i * step, row && unit.head0 + i * step < side.heads, a[i], b[i]);
    float c[8], s[8], g[16];
    lane.angles(p, position, c, s);
    lane.weights(p, side.weight, g);
#pragma unroll
    for (int i = 0; i < kU; ++i) {
      float v[16];
      widen(a[i], b[i], v);
      if (p.norm) {
        normalize<kG>(p, v);
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] *= g[e];
      }
      lane.template turn<false>(p, c, s, v);
      lane.store(side.y, unit.t, unit.head0 + i * step, row && unit.head0 + i * step < side.heads, v);
    }
  }
}

// The pass back.  Workgroups [0, split) take units of the queries, the others of the keys, each every so many of them, and keep the
// sums for their weight in registers; the lane groups' sums are added up through LDS, in order, into the workgroup's plane.
template <int kG, int kU, bool kSums>
__global__ __launch_bounds__(256) void qk_backward_kernel(QkParams p, int split) {
  __shared__ float s_sum[kSums ? 256 * 16 : 1];
  const int lane_id = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int which = static_cast<int>(blockIdx.x) >= split;
  const QkSide &side = p.side[which];
  const int first = which ? split : 0, count = which ? gridDim.x - split : split;
  const int groups = 1 << p.heads_log2, tile_tokens = (64 / kG) >> p.heads_log2;
  Lane<kG> lane;
  lane.begin(p, lane_id);
  float g[16], sum[16] = {};
  lane.weights(p, side.weight, g);
  const int64_t tiles = (p.T + tile_tokens - 1) / tile_tokens, units = tiles * side.chunks;
  const float per = 1.0f / static_cast<float>(p.D);
  for (int64_t u = static_cast<int64_t>(blockIdx.x - first) * 4 + wave; u < units; u += static_cast<int64_t>(count) * 4) {
    const int64_t tile = u / side.chunks;
    const int group = lane_id / kG;
    const int64_t t = tile * tile_tokens + (group >> p.heads_log2);
    const int head0 = static_cast<int>(u - tile * side.chunks) * kU * groups + (group & (groups - 1));
    const int64_t position = t >= p.T ? -1 : p.positions ? p.positions[t] : t;
    const bool row = position >= 0;
    uint4 a[kU], b[kU], da[kU], db[kU];
#pragma unroll
    for (int i = 0; i < kU; ++i) {
      const bool valid = row && head0 + i * groups < side.heads;
      if (p.norm) lane.load(side.x, t, head0 + i * groups, valid, a[i], b[i]);
      lane.load(side.dy, t, head0 + i * groups, valid, da[i], db[i]);
    }
    float c[8], s[8];
    lane.angles(p, position, c, s);
#pragma unroll
    for (int i = 0; i < kU; ++i) {
      const bool valid = row && head0 + i * groups < side.heads;
      float d[16];
      widen(da[i], db[i], d);
      lane.template turn<true>(p, c, s, d);
      if (p.norm) {
        float x[16];
        widen(a[i], b[i], x);
        const float r = normalize<kG>(p, x);
        float dot = 0.0f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          if constexpr (kSums) sum[e] = __builtin_fmaf(d[e], x[e], sum[e]);  // (a head that is not there is all zeros)
          d[e] *= g[e];
          dot = __builtin_fmaf(d[e], x[e], dot);
        }
        dot = group_sum<kG>(dot) * per;
#pragma unroll
        for (int e = 0; e < 16; ++e) d[e] = r * __builtin_fmaf(-x[e], dot, d[e]);
      }
      lane.store(side.y, t, head0 + i * groups, valid, d);
    }
  }
  if constexpr (kSums) {
#pragma unroll
    for (int e = 0; e < 16; ++e) s_sum[e * 256 + threadIdx.x] = sum[e];
    __syncthreads();
    // element e of slot i: the sum over the workgroup's 256 / kG lane groups
    for (int at = threadIdx.x; at < 16 * kG; at += 256) {
      const int e = at / kG, i = at - e * kG;
      Lane<kG> of;
      of.begin(p, i);
      if (!(e < 8 ? of.has_first : of.has_second)) continue;
      float total = 0.0f;
      for (int grp = 0; grp < 256 / kG; ++grp) total += s_sum[e * 256 + grp * kG + i];
      p.planes[static_cast<int64_t>(blockIdx.x) * p.D + (e < 8 ? of.first + e : of.second + e - 8)] = total;
    }
  }
}

// dg of one side: the sum over its workgroups' planes, 16 elements to a workgroup of 1024, 64 planes side by side.
__global__ __launch_bounds__(1024) void qk_weight_kernel(QkParams p, int split, int planes) {
  __shared__ float s_sum[1024];
  const int which = blockIdx.y, first = which ? split : 0, end = which ? planes : split;
  const int j = threadIdx.x & 15, d = blockIdx.x * 16 + j;
  void *out = p.side[which].dweight;
  if (!out) return;
  float sum = 0.0f;
  if (d < p.D)
    for (int s = first + (threadIdx.x >> 4); s < end; s += 64) sum += p.planes[static_cast<int64_t>(s) * p.D + d];
  s_sum[threadIdx.x] = sum;
  for (int half = 512; half >= 16; half >>= 1) {
    __syncthreads();
    if (static_cast<int>(threadIdx.x) < half) s_sum[threadIdx.x] += s_sum[threadIdx.x + half];
  }
  if (threadIdx.x >= 16 || d >= p.D) return;
  if (p.weight_f32) static_cast<float *>(out)[d] = s_sum[threadIdx.x];
  else static_cast<__bf16 *>(out)[d] = static_cast<__bf16>(s_sum[threadIdx.x]);
}

constexpr int kMaxBackwardGroups = 1024;

int log2_up(int64_t n) {
  int l = 0;
  while ((int64_t{1} << l) < n) ++l;
  return l;
}

// Workgroups of the pass back, those of the queries first.
struct BackwardGrid {
  int queries, all;
};

constexpr int kBackwardUnroll = 2;

int heads_log2_of(int q_heads, int k_heads, int group) {
  return std::min(log2_up(64 / group), log2_up(std::max(q_heads, k_heads)));
}
int chunks_of(int heads, int heads_log2, int unroll) {
  const int per = unroll << heads_log2;
  return (heads + per - 1) / per;
}

BackwardGrid backward_grid(int64_t T, int q_heads, int k_heads, int D) {
  const int group = 1 << log2_up((D + 15) / 16), hl = heads_log2_of(q_heads, k_heads, group);
  const int tile = (64 / group) >> hl;
  const int64_t tiles = (T + tile - 1) / tile;
  const int64_t uq = (tiles * chunks_of(q_heads, hl, kBackwardUnroll) + 3) / 4, uk = (tiles * chunks_of(k_heads, hl, kBackwardUnroll) + 3) / 4;
  BackwardGrid g{};
  if (uq + uk <= kMaxBackwardGroups) {
    g.queries = static_cast<int>(uq);
    g.all = static_cast<int>(uq + uk);
  } else {
    g.queries = static_cast<int>(kMaxBackwardGroups * static_cast<double>(uq) / static_cast<double>(uq + uk) + 0.5);
    if (uq > 0) g.queries = std::max(g.queries, 1);
    if (uk > 0) g.queries = std::min(g.queries, kMaxBackwardGroups - 1);
    g.all = kMaxBackwardGroups;
  }
  return g;
}

osdp_status bad(osdp_status st, const char *fmt, long long a = 0, long long b = 0) {
  char buf[256];
  snprintf(buf, sizeof buf, fmt, a, b);
  return report_error(st, buf);
}

bool aligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Elements of a set of heads, as far as memory goes.
struct Extent {
  const osdp_heads *h;
  int64_t heads, T, D;
  __int128 begin() const { return reinterpret_cast<uintptr_t>(h->p); }
  __int128 end() const { return begin() + 2 * (static_cast<__int128>(T - 1) * h->ld + static_cast<__int128>(heads - 1) * h->head_stride + D); }
  bool empty() const { return T <= 0 || heads <= 0; }
};
bool same(const osdp_heads &a, const osdp_heads &b, const Extent &e) {
  return a.p == b.p && (e.T == 1 || a.ld == b.ld) && (e.heads == 1 || a.head_stride == b.head_stride);
}
// Whether two sets of heads share memory: by their extents, and, rows of one length, by the places of their heads in them.
bool share(const Extent &a, const Extent &b) {
  if (a.empty() || b.empty() || a.end() <= b.begin() || b.end() <= a.begin()) return false;
  const bool rows = (a.T == 1 && b.T == 1) || a.h->ld == b.h->ld;
  if (!rows) return true;
  const __int128 ld = a.T == 1 && b.T == 1 ? 0 : a.h->ld;
  __int128 d = (b.begin() - a.begin()) / 2;
  if (ld > 0) d %= ld;
  for (int wrap = -1; wrap <= 1; ++wrap) {
    const __int128 off = d + wrap * ld;  // where b's heads begin in a's rows
    for (int64_t i = 0; i < a.heads; ++i) {
      const __int128 at = static_cast<__int128>(i) * a.h->head_stride - off;  // a's head i, seen from b's first
      const int64_t hs = b.h->head_stride;
      if (hs <= 0 || b.heads == 1) {
        if (at < b.D && -at < a.D) return true;
        continue;
      }
      const __int128 j = at >= 0 ? at / hs : -1;
      for (__int128 k = j; k <= j + 1; ++k)
        if (k >= 0 && k < b.heads && at - k * hs < b.D && k * hs - at < a.D) return true;
    }
    if (ld == 0) break;
  }
  return false;
}

osdp_status check_heads(const osdp_heads *h, int64_t heads, const osdp_qk &q, const char *name, bool written) {
  if (heads == 0 || q.T == 0) return OSDP_OK;
  char buf[160];
  auto say = [&](osdp_status st, const char *what) {
    snprintf(buf, sizeof buf, "%s: %s", name, what);
    return report_error(st, buf);
  };
  if (!h || !h->p) return say(OSDP_ERR_INVALID_ARG, "NULL");
  if (h->ld < 0 || h->head_stride < 0) return say(OSDP_ERR_INVALID_ARG, "a stride is negative");
  if ((q.T > 1 && h->ld % 8) || (heads > 1 && h->head_stride % 8)) return say(OSDP_ERR_UNSUPPORTED, "a stride is not a multiple of 8");
  if (!aligned(h->p)) return say(OSDP_ERR_UNSUPPORTED, "not 16-byte aligned");
  if (written) {
    const __int128 D = q.D, row = static_cast<__int128>(heads - 1) * h->head_stride + D, column = static_cast<__int128>(q.T - 1) * h->ld + D;
    const bool heads_apart = heads == 1 || h->head_stride >= D, rows_apart = q.T == 1 || h->ld >= D;
    if (!heads_apart || !rows_apart || !(q.T == 1 || heads == 1 || h->ld >= row || h->head_stride >= column))
      return say(OSDP_ERR_INVALID_ARG, "its own heads overlap");
  }
  return OSDP_OK;
}

osdp_status check_qk(const osdp_qk *qk) {
  if (!qk) return bad(OSDP_ERR_INVALID_ARG, "qk is NULL");
  const osdp_qk &q = *qk;
  if (q.T < 0 || q.q_heads < 0 || q.k_heads < 0 || q.D <= 0) return bad(OSDP_ERR_INVALID_ARG, "T and heads must not be negative, D positive");
  if (q.rotary < 0 || q.rotary > q.D) return bad(OSDP_ERR_INVALID_ARG, "rotary (%lld) is not within D (%lld)", q.rotary, q.D);
  if (q.interleaved < 0 || q.interleaved > 1 || q.norm < 0 || q.norm > 1 || q.reserved != 0)
    return bad(OSDP_ERR_INVALID_ARG, "interleaved and norm are 0 or 1, reserved is 0");
  if (q.weight_type != OSDP_BF16 && q.weight_type != OSDP_F32) return bad(OSDP_ERR_INVALID_ARG, "unknown weight_type %lld", q.weight_type);
  if (q.norm && !(q.eps >= 1e-12 && q.eps <= 1e30)) return bad(OSDP_ERR_INVALID_ARG, "eps is not within 1e-12 and 1e30");
  if (!q.norm && (q.q_weight || q.k_weight)) return bad(OSDP_ERR_INVALID_ARG, "weights are given without a norm");
  if (q.rotary > 0 && !q.freqs) return bad(OSDP_ERR_INVALID_ARG, "freqs is NULL");
  if (q.D % 8 || q.D > 512) return bad(OSDP_ERR_UNSUPPORTED, "D (%lld) is not a multiple of 8 up to 512", q.D);
  if (q.rotary % (q.interleaved ? 8 : 16)) return bad(OSDP_ERR_UNSUPPORTED, "rotary (%lld) is not a multiple of %lld", q.rotary, q.interleaved ? 8 : 16);
  if (q.T >= (int64_t{1} << 31) || q.q_heads > 65535 || q.k_heads > 65535) return bad(OSDP_ERR_UNSUPPORTED, "too many tokens or heads");
  if (!aligned(q.q_weight) || !aligned(q.k_weight)) return bad(OSDP_ERR_UNSUPPORTED, "a weight is not 16-byte aligned");
  if ((reinterpret_cast<uintptr_t>(q.positions) | reinterpret_cast<uintptr_t>(q.freqs)) & 7u)
    return bad(OSDP_ERR_UNSUPPORTED, "positions or freqs is not 8-byte aligned");
  return OSDP_OK;
}

QkParams params_of(const osdp_qk &q, int group, int unroll) {
  QkParams p{};
  p.positions = q.positions; p.freqs = q.freqs;
  p.T = q.T; p.eps = static_cast<float>(q.eps);
  p.D = q.D; p.slots = (q.D + 15) / 16;
  p.rotary = q.rotary; p.interleaved = q.interleaved; p.norm = q.norm; p.weight_f32 = q.weight_type == OSDP_F32;
  p.heads_log2 = heads_log2_of(q.q_heads, q.k_heads, group);
  const int heads[2] = {q.q_heads, q.k_heads};
  const void *weight[2] = {q.q_weight, q.k_weight};
  for (int i = 0; i < 2; ++i) {
    p.side[i].heads = heads[i];
    p.side[i].chunks = chunks_of(heads[i], p.heads_log2, unroll);
    p.side[i].weight = weight[i];
  }
  return p;
}
HeadsIn in(const osdp_heads *h) { return h ? HeadsIn{static_cast<const uint16_t *>(h->p), h->ld, h->head_stride} : HeadsIn{nullptr, 0, 0}; }
HeadsOut out(const osdp_heads *h) { return h ? HeadsOut{static_cast<uint16_t *>(h->p), h->ld, h->head_stride} : HeadsOut{nullptr, 0, 0}; }

// Tokens times head groups from which a wave takes four head groups, with their angles worked out once, rather than one.
constexpr int64_t kManyUnits = 8192;

template <int kG>
void launch_forward(QkParams &p, const osdp_qk &q, hipStream_t stream) {
  const int tile = (64 / kG) >> p.heads_log2;
  const int64_t tiles = (q.T + tile - 1) / tile;
  const bool many = tiles * (p.side[0].chunks + p.side[1].chunks) >= kManyUnits;
  if (many)
    for (QkSide &s : p.side) s.chunks = chunks_of(s.heads, p.heads_log2, 4);
  p.units = tiles * (p.side[0].chunks + p.side[1].chunks);
  const unsigned grid = static_cast<unsigned>(std::min<int64_t>((p.units + 3) / 4, 1 << 22));
  if (many) hipLaunchKernelGGL((qk_forward_kernel<kG, 4>), dim3(grid), dim3(256), 0, stream, p);
  else hipLaunchKernelGGL((qk_forward_kernel<kG, 1>), dim3(grid), dim3(256), 0, stream, p);
}

template <int kG>
void launch_backward(const QkParams &p, BackwardGrid grid, hipStream_t stream) {
  if (p.planes) hipLaunchKernelGGL((qk_backward_kernel<kG, kBackwardUnroll, true>), dim3(grid.all), dim3(256), 0, stream, p, grid.queries);
  else hipLaunchKernelGGL((qk_backward_kernel<kG, kBackwardUnroll, false>), dim3(grid.all), dim3(256), 0, stream, p, grid.queries);
}

// f(integral_constant<kG>) for the lanes that hold a head.
template <class F>
void with_group(int D, F &&f) {
  switch (log2_up((D + 15) / 16)) {
    case 0: f(std::integral_constant<int, 1>{}); break;
    case 1: f(std::integral_constant<int, 2>{}); break;
    case 2: f(std::integral_constant<int, 4>{}); break;
    case 3: f(std::integral_constant<int, 8>{}); break;
    case 4: f(std::integral_constant<int, 16>{}); break;
    default: f(std::integral_constant<int, 32>{}); break;
  }
}

osdp_status hip_status(hipError_t e, const char *what) {
  if (e == hipSuccess) return OSDP_OK;
  char buf[160];
  snprintf(buf, sizeof buf, "%s: %s", what, hipGetErrorString(e));
  return report_error(OSDP_ERR_HIP, buf);
}
osdp_status right_device() {
  const hipError_t e = check_device();
  if (e == hipErrorInvalidDevice) return bad(OSDP_ERR_UNSUPPORTED, "the current device is not an MI355X");
  return hip_status(e, "querying the device");
}

}  // namespace
}  // namespace osdp

using namespace osdp;

osdp_status osdp_qk_norm_rope_fwd(const osdp_qk *qk, const osdp_heads *q, const osdp_heads *k, const osdp_heads *q_out,
                                  const osdp_heads *k_out, void *stream) {
  osdp_status st = check_qk(qk);
  if (st != OSDP_OK) return st;
  const osdp_qk &d = *qk;
  if ((st = check_heads(q, d.q_heads, d, "q", false)) != OSDP_OK || (st = check_heads(k, d.k_heads, d, "k", false)) != OSDP_OK ||
      (st = check_heads(q_out, d.q_heads, d, "q_out", true)) != OSDP_OK || (st = check_heads(k_out, d.k_heads, d, "k_out", true)) != OSDP_OK)
    return st;
  const Extent eq{q, d.q_heads, d.T, d.D}, ek{k, d.k_heads, d.T, d.D}, eqo{q_out, d.q_heads, d.T, d.D}, eko{k_out, d.k_heads, d.T, d.D};
  if ((!eq.empty() && !same(*q, *q_out, eq) && share(eq, eqo)) || (!ek.empty() && !same(*k, *k_out, ek) && share(ek, eko)) ||
      share(eqo, ek) || share(eko, eq) || share(eqo, eko))
    return bad(OSDP_ERR_INVALID_ARG, "an output overlaps an input or the other output");
  if ((st = right_device()) != OSDP_OK) return st;
  if (d.T == 0 || d.q_heads + d.k_heads == 0) return OSDP_OK;
  with_group(d.D, [&](auto group) {
    constexpr int kG = decltype(group)::value;
    QkParams p = params_of(d, kG, 1);
    p.side[0].x = in(q); p.side[0].y = out(q_out);
    p.side[1].x = in(k); p.side[1].y = out(k_out);
    launch_forward<kG>(p, d, static_cast<hipStream_t>(stream));
  });
  return hip_status(hipGetLastError(), "launching the norms of queries and keys");
}

osdp_status osdp_qk_norm_rope_bwd_workspace_bytes(const osdp_qk *qk, size_t *bytes) {
  if (!qk || !bytes) return bad(OSDP_ERR_INVALID_ARG, "NULL argument");
  if (qk->T < 0 || qk->q_heads < 0 || qk->k_heads < 0 || qk->D <= 0) return bad(OSDP_ERR_INVALID_ARG, "T and heads must not be negative, D positive");
  if (qk->D % 8 || qk->D > 512 || qk->T >= (int64_t{1} << 31) || qk->q_heads > 65535 || qk->k_heads > 65535)
    return bad(OSDP_ERR_UNSUPPORTED, "D must be a multiple of 8 up to 512, T below 2^31, heads at most 65535");
  *bytes = static_cast<size_t>(backward_grid(qk->T, qk->q_heads, qk->k_heads, qk->D).all) * qk->D * sizeof(float);
  return OSDP_OK;
}

osdp_status osdp_qk_norm_rope_bwd(const osdp_qk *qk, const osdp_heads *q, const osdp_heads *k, const osdp_heads *dq_out,
                                  const osdp_heads *dk_out, const osdp_heads *dq, const osdp_heads *dk, void *dq_weight,
                                  void *dk_weight, void *workspace, size_t workspace_bytes, void *stream) {
  osdp_status st = check_qk(qk);
  if (st != OSDP_OK) return st;
  const osdp_qk &d = *qk;
  const bool sums = dq_weight || dk_weight;
  if (sums && !d.norm) return bad(OSDP_ERR_INVALID_ARG, "weight gradients are asked for without a norm");
  if (!aligned(dq_weight) || !aligned(dk_weight)) return bad(OSDP_ERR_UNSUPPORTED, "a weight gradient is not 16-byte aligned");
  if (sums && dq_weight == dk_weight) return bad(OSDP_ERR_INVALID_ARG, "the two weight gradients are one");
  // (the inputs of the forward pass are read only for the norm)
  if ((d.norm && ((st = check_heads(q, d.q_heads, d, "q", false)) != OSDP_OK || (st = check_heads(k, d.k_heads, d, "k", false)) != OSDP_OK)) ||
      (st = check_heads(dq_out, d.q_heads, d, "dq_out", false)) != OSDP_OK || (st = check_heads(dk_out, d.k_heads, d, "dk_out", false)) != OSDP_OK ||
      (st = check_heads(dq, d.q_heads, d, "dq", true)) != OSDP_OK || (st = check_heads(dk, d.k_heads, d, "dk", true)) != OSDP_OK)
    return st;
  const int64_t T = d.T;
  const Extent ex[2] = {{q, d.norm ? d.q_heads : 0, T, d.D}, {k, d.norm ? d.k_heads : 0, T, d.D}};
  const Extent ey[2] = {{dq_out, d.q_heads, T, d.D}, {dk_out, d.k_heads, T, d.D}}, eo[2] = {{dq, d.q_heads, T, d.D}, {dk, d.k_heads, T, d.D}};
  bool clash = share(eo[0], eo[1]);
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2; ++j)
      for (const Extent *e : {&ex[j], &ey[j]})
        if (!e->empty() && !eo[i].empty() && !(i == j && same(*eo[i].h, *e->h, *e))) clash = clash || share(eo[i], *e);
  if (clash) return bad(OSDP_ERR_INVALID_ARG, "an output overlaps an input or the other output");
  const BackwardGrid grid = backward_grid(T, d.q_heads, d.k_heads, d.D);
  if (sums) {
    if (!workspace) return bad(OSDP_ERR_INVALID_ARG, "workspace is NULL");
    if (reinterpret_cast<uintptr_t>(workspace) & 255u) return bad(OSDP_ERR_UNSUPPORTED, "workspace is not 256-byte aligned");
    const size_t need = static_cast<size_t>(grid.all) * d.D * sizeof(float);
    if (workspace_bytes < need) return bad(OSDP_ERR_WORKSPACE, "workspace holds %lld bytes, %lld needed", workspace_bytes, need);
  }
  if ((st = right_device()) != OSDP_OK) return st;
  hipStream_t hs = static_cast<hipStream_t>(stream);
  QkParams last{};
  with_group(d.D, [&](auto group) {
    constexpr int kG = decltype(group)::value;
    QkParams p = params_of(d, kG, kBackwardUnroll);
    p.side[0].x = in(d.norm ? q : nullptr); p.side[0].dy = in(dq_out); p.side[0].y = out(dq); p.side[0].dweight = dq_weight;
    p.side[1].x = in(d.norm ? k : nullptr); p.side[1].dy = in(dk_out); p.side[1].y = out(dk); p.side[1].dweight = dk_weight;
    p.planes = sums ? static_cast<float *>(workspace) : nullptr;
    if (grid.all > 0) launch_backward<kG>(p, grid, hs);
    last = p;
  });
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && sums) {
    hipLaunchKernelGGL(qk_weight_kernel, dim3((d.D + 15) / 16, 2), dim3(1024), 0, hs, last, grid.queries, grid.all);
    e = hipGetLastError();
  }
  return hip_status(e, "launching the norms of queries and keys");
}

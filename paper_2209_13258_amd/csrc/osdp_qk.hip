// Norms of queries and keys for each head and their rotation by position, in one pass over the qkv operator's output, and the
// pass back.  HBM bound: 4 bytes an element forward, 6 backward, against some 10 and 20 operations in fp32.  8192 tokens, heads of
// 128: forward 32 + 32 heads 57 us (4.7 TB/s), backward 32 + 8 heads 53 us (4.75 TB/s) and 5 us for the weights' sums.
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
  int32_t heads, chunks, waves_log2;  // chunks: kU head groups each; waves of a workgroup that share a token tile (backward)
};
struct QkParams {
  QkSide side[2];
  const int64_t *positions;
  const double *freqs;
  int64_t T, tiles;    // tiles: of the tokens that a wave's lane groups hold
  float eps;
  int32_t D, slots;    // slots: lanes of a group that hold elements
  int32_t rotary, interleaved, norm, weight_f32;
  int32_t heads_log2;  // head groups of a wave; the other lane groups hold the next tokens
  int32_t waves_log2;  // waves of a workgroup that share a token tile (forward)
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

// How pairs lie, and whether every element is in one.  Elements that are not turned are kept from their neighbours, which may
// be infinite, by selections that heads turned as a whole do not need.
enum Pairs { kHalves = 0, kNeighbours = 1, kHalvesPartly = 2, kNeighboursPartly = 3 };
constexpr bool neighbours(int pairs) { return pairs & 1; }
constexpr bool partly(int pairs) { return pairs & 2; }

// A lane's elements 0..7 are its first piece, 8..15 its second; its pair e (of 8) is made of
constexpr int low_of(int pairs, int e) { return neighbours(pairs) ? 2 * e : e; }
constexpr int high_of(int pairs, int e) { return neighbours(pairs) ? 2 * e + 1 : 8 + e; }

// What a lane holds of every head.
template <int kG, int kPairs>
struct Lane {
  int i, first, second;          // its slot, where its two pieces begin (elements; where there is none: the head's first one)
  bool has_first, has_second, turns_low, turns_high;  // turns: its pairs 0..3 and 4..7
  __device__ __forceinline__ void begin(const QkParams &p, int lane) {
    i = lane & (kG - 1);
    const int pairs = p.rotary / 2;
    if (!neighbours(kPairs) && i < p.rotary / 16) {
      first = 8 * i;
      second = first + pairs;
    } else {
      first = neighbours(kPairs) ? 16 * i : p.rotary + 16 * (i - p.rotary / 16);
      second = first + 8;
    }
    has_first = i < p.slots && first < p.D;
    has_second = has_first && second < p.D;
    first = has_first ? first : 0;
    second = has_second ? second : 0;
    turns_low = has_first && 8 * i < pairs;
    turns_high = has_first && 8 * i + 4 < pairs;
  }
  __device__ __forceinline__ bool turns(int e) const { return neighbours(kPairs) && e >= 4 ? turns_high : turns_low; }
  __device__ __forceinline__ void weights(const QkParams &p, const void *w, float (&g)[16]) const {
#pragma unroll
    for (int e = 0; e < 16; ++e) g[e] = 1.0f;
    if (!w) return;
    const int at[2] = {first, second};
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      if (p.weight_f32) {
        const float4 *src = reinterpret_cast<const float4 *>(static_cast<const float *>(w) + at[half]);
        const float4 a = src[0], b = src[1];
        g[8 * half] = a.x; g[8 * half + 1] = a.y; g[8 * half + 2] = a.z; g[8 * half + 3] = a.w;
        g[8 * half + 4] = b.x; g[8 * half + 5] = b.y; g[8 * half + 6] = b.z; g[8 * half + 7] = b.w;
      } else {
        const uint4 a = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(w) + at[half]);
        g[8 * half] = bf16_low(a.x); g[8 * half + 1] = bf16_high(a.x); g[8 * half + 2] = bf16_low(a.y); g[8 * half + 3] = bf16_high(a.y);
        g[8 * half + 4] = bf16_low(a.z); g[8 * half + 5] = bf16_high(a.z); g[8 * half + 6] = bf16_low(a.w); g[8 * half + 7] = bf16_high(a.w);
      }
    }
  }
  // Cosines and sines of its pairs; 1 and 0 of those that do not turn.
  __device__ __forceinline__ void angles(const QkParams &p, int64_t position, float (&c)[8], float (&s)[8]) const {
    constexpr double kTurn = 0.15915494309189533577;  // 1 / (2 pi)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      c[e] = 1.0f;
      s[e] = 0.0f;
    }
    if (!turns_low) return;
    const double at = static_cast<double>(position) * kTurn;
    const double *freqs = p.freqs + 8 * i;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const bool there = e < 4 || !neighbours(kPairs) || turns_high;
      const double turned = at * freqs[there ? e : e - 4];
      const float rest = static_cast<float>(turned - __builtin_rint(turned));
      c[e] = there ? __builtin_amdgcn_cosf(rest) : 1.0f;  // (of turns)
      s[e] = there ? __builtin_amdgcn_sinf(rest) : 0.0f;
    }
  }
  __device__ __forceinline__ void store(uint16_t *head, bool valid, const float (&v)[16]) const {
    if (valid && has_first) store_global16(head + first, uint4{pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7])});
    if (valid && has_second) store_global16(head + second, uint4{pack2(v[8], v[9]), pack2(v[10], v[11]), pack2(v[12], v[13]), pack2(v[14], v[15])});
  }
  // The sum over the head of products of what the lanes hold (pieces that are not there hold the head's first ones).
  __device__ __forceinline__ float dot(const float (&a)[16], const float (&b)[16]) const {
    float lo = 0.0f, hi = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      lo = __builtin_fmaf(a[e], b[e], lo);
      hi = __builtin_fmaf(a[8 + e], b[8 + e], hi);
    }
    return group_sum<kG>((has_first ? lo : 0.0f) + (has_second ? hi : 0.0f));
  }
  // 1 / sqrt(mean v^2 + eps) over the head.  Where squares leave the range in which the rest is safe, v is scaled by 2^-70 first,
  // and so is *scale; eps goes with the squares, by 2^-140 (in two steps: that number is none of fp32's normal ones.  An eps that
  // ends below 2^-126 is nothing beside a mean of 2^-89 or more: the sum is above 2^60 and D at most 2^9).
  __device__ __forceinline__ float factor(const QkParams &p, float (&v)[16], float *scale) const {
    float s = dot(v, v), eps = p.eps;
    *scale = 1.0f;
    if (__builtin_expect(s > 0x1p60f, 0)) {  // (all lanes of the group or none)
      *scale = 0x1p-70f;
#pragma unroll
      for (int e = 0; e < 16; ++e) v[e] *= 0x1p-70f;
      s = dot(v, v);
      eps = eps * 0x1p-70f * 0x1p-70f;
    }
    return rsqrtf(__builtin_fmaf(s, 1.0f / static_cast<float>(p.D), eps));
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
__device__ __forceinline__ uint4 only_if(bool c, uint4 v) { return uint4{c ? v.x : 0u, c ? v.y : 0u, c ? v.z : 0u, c ? v.w : 0u}; }

// Forward.  With g the weight and r the head's factor a pair becomes r (a g_a c - b g_b s), r (b g_b c + a g_a s): the products
// of weights, cosines and sines are made once for a token's heads.  A wave takes kU head groups of a token tile; the waves of a
// workgroup those of one token tile, or of several where it has few.
template <int kG, int kU, int kPairs>
__global__ __launch_bounds__(256) void qk_forward_kernel(QkParams p) {
  const int lane_id = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Lane<kG, kPairs> lane;
  lane.begin(p, lane_id);
  const int group = lane_id / kG, step = 1 << p.heads_log2, tile_tokens = (64 / kG) >> p.heads_log2;
  const int chunk = (blockIdx.y << p.waves_log2) + (wave & ((1 << p.waves_log2) - 1));
  if (chunk >= p.side[0].chunks + p.side[1].chunks) return;
  const bool keys = chunk >= p.side[0].chunks;
  const HeadsIn x = keys ? p.side[1].x : p.side[0].x;
  const HeadsOut y = keys ? p.side[1].y : p.side[0].y;
  const int heads = keys ? p.side[1].heads : p.side[0].heads;
  const int head0 = (keys ? chunk - p.side[0].chunks : chunk) * kU * step + (group & (step - 1));
  const int tiles_at_once = 4 >> p.waves_log2;
  for (int64_t tile = static_cast<int64_t>(blockIdx.x) * tiles_at_once + (wave >> p.waves_log2); tile < p.tiles;
       tile += static_cast<int64_t>(gridDim.x) * tiles_at_once) {
    const int64_t t = tile * tile_tokens + (group >> p.heads_log2), t_in = t < p.T ? t : p.T - 1;
    const uint16_t *src = x.p + t_in * x.ld;
    uint4 a[kU], b[kU];
#pragma unroll
    for (int i = 0; i < kU; ++i) {  // (lanes without a head load one that is there)
      const int head = head0 + i * step;
      const uint16_t *at = src + (head < heads ? head : heads - 1) * x.hs;
      a[i] = load_global16(at + lane.first);
      b[i] = load_global16(at + lane.second);
    }
    const int64_t position = p.positions ? p.positions[t_in] : t;
    const bool row = t < p.T && position >= 0;
    float g[16], same[16], cross[16];  // what an element is multiplied by in its own place, and in its partner's
    lane.weights(p, keys ? p.side[1].weight : p.side[0].weight, g);
    {
      float c[8], s[8];
      lane.angles(p, position, c, s);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        constexpr int kP = kPairs;
        const int lo = low_of(kP, e), hi = high_of(kP, e);
        same[lo] = g[lo] * c[e];
        cross[lo] = g[lo] * s[e];
        same[hi] = g[hi] * c[e];
        cross[hi] = g[hi] * s[e];
      }
    }
    uint16_t *dst = y.p + t_in * y.ld;
#pragma unroll
    for (int i = 0; i < kU; ++i) {
      float v[16], o[16], r = 1.0f, scale;
      widen(a[i], b[i], v);
      if (p.norm) r = lane.factor(p, v, &scale);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int lo = low_of(kPairs, e), hi = high_of(kPairs, e);
        float to_lo = v[hi], to_hi = v[lo];
        if constexpr (partly(kPairs)) {
          to_lo = lane.turns(e) ? to_lo : 0.0f;
          to_hi = lane.turns(e) ? to_hi : 0.0f;
        }
        o[lo] = r * __builtin_fmaf(v[lo], same[lo], -(to_lo * cross[hi]));
        o[hi] = r * __builtin_fmaf(v[hi], same[hi], to_hi * cross[lo]);
      }
      const int head = head0 + i * step;
      lane.store(dst + head * y.hs, row && head < heads, o);
    }
  }
}

// The pass back.  Workgroups [0, split) take token tiles of the queries, the others of the keys, each every so many of them, and keep
// the sums for their weight in registers; the lane groups' sums are added up through LDS, in order, into the workgroup's plane.
// With d the gradients turned back, x the head and r its factor:  u = d r,  sum += u x,  t = u g,  dx = t - x r^2 mean(t x).
template <int kG, int kU, int kPairs, bool kSums>
__global__ __launch_bounds__(256) void qk_backward_kernel(QkParams p, int split) {
  __shared__ float s_sum[kSums ? 256 * 16 : 1];
  const int lane_id = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool keys = static_cast<int>(blockIdx.x) >= split;
  const HeadsIn x = keys ? p.side[1].x : p.side[0].x, dy = keys ? p.side[1].dy : p.side[0].dy;
  const HeadsOut y = keys ? p.side[1].y : p.side[0].y;
  const int heads = keys ? p.side[1].heads : p.side[0].heads, chunks = keys ? p.side[1].chunks : p.side[0].chunks;
  const int waves_log2 = keys ? p.side[1].waves_log2 : p.side[0].waves_log2;
  const int first = keys ? split : 0, count = keys ? gridDim.x - split : split;
  const int group = lane_id / kG, step = 1 << p.heads_log2, tile_tokens = (64 / kG) >> p.heads_log2;
  Lane<kG, kPairs> lane;
  lane.begin(p, lane_id);
  float g[16], sum[16] = {};
  lane.weights(p, keys ? p.side[1].weight : p.side[0].weight, g);
  const float per = 1.0f / static_cast<float>(p.D);
  const int tiles_at_once = 4 >> waves_log2;
  for (int64_t tile = static_cast<int64_t>(blockIdx.x - first) * tiles_at_once + (wave >> waves_log2); tile < p.tiles;
       tile += static_cast<int64_t>(count) * tiles_at_once) {
    const int64_t t = tile * tile_tokens + (group >> p.heads_log2), t_in = t < p.T ? t : p.T - 1;
    const int64_t position = p.positions ? p.positions[t_in] : t;
    const bool row = t < p.T && position >= 0;
    float c[8], s[8];
    lane.angles(p, position, c, s);
    const uint16_t *src_x = x.p + t_in * x.ld, *src_dy = dy.p + t_in * dy.ld;
    uint16_t *dst = y.p + t_in * y.ld;
    for (int chunk = wave & ((1 << waves_log2) - 1); chunk < chunks; chunk += 1 << waves_log2) {
      const int head0 = chunk * kU * step + (group & (step - 1));
      uint4 a[kU], b[kU], da[kU], db[kU];
#pragma unroll
      for (int i = 0; i < kU; ++i) {
        const int head = head0 + i * step, in = head < heads ? head : heads - 1;
        a[i] = b[i] = uint4{0u, 0u, 0u, 0u};
        if (p.norm) {
          a[i] = load_global16(src_x + in * x.hs + lane.first);
          b[i] = load_global16(src_x + in * x.hs + lane.second);
        }
        da[i] = load_global16(src_dy + in * dy.hs + lane.first);
        db[i] = load_global16(src_dy + in * dy.hs + lane.second);
      }
#pragma unroll
      for (int i = 0; i < kU; ++i) {
        const int head = head0 + i * step;
        const bool valid = row && head < heads;
        float w[16], d[16];
        widen(kSums ? only_if(valid, da[i]) : da[i], kSums ? only_if(valid, db[i]) : db[i], w);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int lo = low_of(kPairs, e), hi = high_of(kPairs, e);
          float to_lo = w[hi], to_hi = w[lo];
          if constexpr (partly(kPairs)) {
            to_lo = lane.turns(e) ? to_lo : 0.0f;
            to_hi = lane.turns(e) ? to_hi : 0.0f;
          }
          d[lo] = __builtin_fmaf(w[lo], c[e], to_lo * s[e]);
          d[hi] = __builtin_fmaf(w[hi], c[e], -(to_hi * s[e]));
        }
        if (p.norm) {
          float v[16], scale;
          widen(kSums ? only_if(valid, a[i]) : a[i], kSums ? only_if(valid, b[i]) : b[i], v);
          const float r = lane.factor(p, v, &scale);
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            d[e] *= r;
            if constexpr (kSums) sum[e] = __builtin_fmaf(d[e], v[e], sum[e]);
            d[e] *= g[e];
          }
          const float k = lane.dot(d, v) * per * (r * r);
#pragma unroll
          for (int e = 0; e < 16; ++e) d[e] = __builtin_fmaf(-v[e], k, d[e]);
          if (__builtin_expect(scale != 1.0f, 0))
#pragma unroll
            for (int e = 0; e < 16; ++e) d[e] *= scale;
        }
        lane.store(dst + head * y.hs, valid, d);
      }
    }
  }
  if constexpr (kSums) {
#pragma unroll
    for (int e = 0; e < 16; ++e) s_sum[e * 256 + threadIdx.x] = sum[e];
    __syncthreads();
    // element e of slot i: the sum over the workgroup's 256 / kG lane groups
    for (int at = threadIdx.x; at < 16 * kG; at += 256) {
      const int e = at / kG, i = at - e * kG;
      Lane<kG, kPairs> of;
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

// Workgroups of the pass back: three to a CU, which is what its registers let run, so that all of them run from the start.  us for 8192
// tokens, 32 + 8 heads of 128, with the sums' launch: 768 58, 1024 71; one head group at a time 79; held to 128 registers, which
// spills, 1024 60.
constexpr int kMaxBackwardGroups = 768;

int log2_up(int64_t n) {
  int l = 0;
  while ((int64_t{1} << l) < n) ++l;
  return l;
}

int waves_log2_of(int chunks) { return std::min(2, log2_up(std::max(1, chunks))); }

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
  const int cq = chunks_of(q_heads, hl, kBackwardUnroll), ck = chunks_of(k_heads, hl, kBackwardUnroll);
  // Workgroups that the token tiles can keep busy (of a side with no heads none).  Where both sides have more than run at once, they
  // share those by their work, head groups beyond a workgroup's four waves included: a workgroup walks these itself.
  const int64_t at_once[2] = {4 >> waves_log2_of(cq), 4 >> waves_log2_of(ck)};
  const int64_t mq = cq ? (tiles + at_once[0] - 1) / at_once[0] : 0, mk = ck ? (tiles + at_once[1] - 1) / at_once[1] : 0;
  BackwardGrid g{};
  if (mq + mk <= kMaxBackwardGroups) {
    g.queries = static_cast<int>(mq);
    g.all = static_cast<int>(mq + mk);
    return g;
  }
  const int64_t wq = mq * ((cq + 3) / 4), wk = mk * ((ck + 3) / 4);
  int64_t queries = static_cast<int64_t>(kMaxBackwardGroups * static_cast<double>(wq) / static_cast<double>(wq + wk) + 0.5);
  if (wq > 0) queries = std::max<int64_t>(queries, 1);
  if (wk > 0) queries = std::min<int64_t>(queries, kMaxBackwardGroups - 1);
  const int64_t keys = std::min(mk, kMaxBackwardGroups - std::min(queries, mq));
  g.queries = static_cast<int>(std::min(mq, kMaxBackwardGroups - keys));
  g.all = g.queries + static_cast<int>(keys);
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
// Whether two sets of heads share memory.  Head i of token t of the one and head j of token u of the other do where
// |i hs_a - j hs_b - n ld - d| < D, with n = u - t and d the distance of the two pointers: exact for rows of one length, in any order of
// heads and tokens.  Rows of two lengths are taken to share what their extents do, as are more than 2^20 pairs of heads of two strides.
// (32-bit lengths and extents below 2^60: nothing here leaves 64 bits.)
bool share(const Extent &a, const Extent &b) {
  if (a.empty() || b.empty() || a.end() <= b.begin() || b.end() <= a.begin()) return false;
  const int64_t D = a.D, last = a.T - 1, ld = last > 0 ? a.h->ld : 0;
  if (last > 0 && (a.h->ld != b.h->ld || ld == 0)) return true;
  const int64_t d = static_cast<int64_t>((b.begin() - a.begin()) / 2);
  const int64_t hs_a = a.heads > 1 ? a.h->head_stride : 0, hs_b = b.heads > 1 ? b.h->head_stride : 0;
  if (last > 0) {  // parts of one wide row, side by side
    const int64_t row_a = (a.heads - 1) * hs_a + D, row_b = (b.heads - 1) * hs_b + D, place = (d % ld + ld) % ld;
    if (place >= row_a && place + row_b <= ld) return false;
  }
  auto meet = [&](int64_t off) {  // heads this far apart in tokens of one number
    int64_t n = 0;
    if (last > 0) {  // the largest n with off - n ld > -D, as far as there are tokens
      const int64_t x = off + D - 1;
      n = x >= 0 ? x / ld : -((ld - 1 - x) / ld);
      n = std::max(-last, std::min(last, n));
    }
    const int64_t apart = off - n * ld;
    return apart < D && -apart < D;
  };
  if (hs_a == hs_b || a.heads == 1 || b.heads == 1) {  // the difference of the heads' numbers is what counts
    for (int64_t m = 0; m < a.heads; ++m)
      if (meet(m * hs_a - d)) return true;
    for (int64_t m = 1; m < b.heads; ++m)
      if (meet(-m * hs_b - d)) return true;
    return false;
  }
  if (a.heads * b.heads > (int64_t{1} << 20)) return true;
  for (int64_t i = 0; i < a.heads; ++i)
    for (int64_t j = 0; j < b.heads; ++j)
      if (meet(i * hs_a - j * hs_b - d)) return true;
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
  if (static_cast<__int128>(q.T - 1) * h->ld + static_cast<__int128>(heads - 1) * h->head_stride >= (int64_t{1} << 60))
    return say(OSDP_ERR_INVALID_ARG, "its strides leave the address space");
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
    p.side[i].waves_log2 = waves_log2_of(p.side[i].chunks);
    p.side[i].weight = weight[i];
  }
  const int tile = (64 / group) >> p.heads_log2;
  p.tiles = (q.T + tile - 1) / tile;
  return p;
}
HeadsIn in(const osdp_heads *h) { return h ? HeadsIn{static_cast<const uint16_t *>(h->p), h->ld, h->head_stride} : HeadsIn{nullptr, 0, 0}; }
HeadsOut out(const osdp_heads *h) { return h ? HeadsOut{static_cast<uint16_t *>(h->p), h->ld, h->head_stride} : HeadsOut{nullptr, 0, 0}; }

// Tokens times head groups from which a wave takes four head groups, with their angles worked out once, rather than one.  us with four /
// with one: 8192 tokens, 32 + 32 heads of 128 46.1 / 48.5, 32 + 8 31.3 / 32.5, 64 + 8 of 256 112 / 118; 1024 tokens, 32 + 32 of 128 8.6 / 8.6
// (8192 units), 256 tokens 4.7 / 4.2.  Few heads leave some of the four without one, and then four lose: 8192 tokens, 32 + 8 heads of
// 64 20.7 / 17.8, 8 + 8 of 128 19.5 / 13.6.
constexpr int64_t kManyUnits = 8192;

template <int kG, int kPairs>
void launch_forward(QkParams &p, hipStream_t stream) {
  const bool many = p.tiles * (p.side[0].chunks + p.side[1].chunks) >= kManyUnits;
  if (many)
    for (QkSide &s : p.side) s.chunks = chunks_of(s.heads, p.heads_log2, 4);
  const int chunks = p.side[0].chunks + p.side[1].chunks;
  p.waves_log2 = waves_log2_of(chunks);
  const int at_once = 4 >> p.waves_log2, rows = (chunks + (1 << p.waves_log2) - 1) >> p.waves_log2;
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>((p.tiles + at_once - 1) / at_once, (1 << 22) / std::min(rows, 1 << 12))), rows);
  if (many) hipLaunchKernelGGL((qk_forward_kernel<kG, 4, kPairs>), grid, dim3(256), 0, stream, p);
  else hipLaunchKernelGGL((qk_forward_kernel<kG, 1, kPairs>), grid, dim3(256), 0, stream, p);
}

template <int kG, int kPairs>
void launch_backward(const QkParams &p, BackwardGrid grid, hipStream_t stream) {
  constexpr int kU = kBackwardUnroll;
  if (p.planes) hipLaunchKernelGGL((qk_backward_kernel<kG, kU, kPairs, true>), dim3(grid.all), dim3(256), 0, stream, p, grid.queries);
  else hipLaunchKernelGGL((qk_backward_kernel<kG, kU, kPairs, false>), dim3(grid.all), dim3(256), 0, stream, p, grid.queries);
}

// f(integral_constant<kG>, integral_constant<kPairs>) for the lanes that hold a head and the pairs that are turned.
template <int kPairs, class F>
void with_group(int D, F &&f) {
  std::integral_constant<int, kPairs> pairs;
  switch (log2_up((D + 15) / 16)) {
    case 0: f(std::integral_constant<int, 1>{}, pairs); break;
    case 1: f(std::integral_constant<int, 2>{}, pairs); break;
    case 2: f(std::integral_constant<int, 4>{}, pairs); break;
    case 3: f(std::integral_constant<int, 8>{}, pairs); break;
    case 4: f(std::integral_constant<int, 16>{}, pairs); break;
    default: f(std::integral_constant<int, 32>{}, pairs); break;
  }
}
template <class F>
void with_kernel(const osdp_qk &q, F &&f) {
  const bool part = q.rotary < q.D;
  if (q.interleaved) part ? with_group<kNeighboursPartly>(q.D, f) : with_group<kNeighbours>(q.D, f);
  else part ? with_group<kHalvesPartly>(q.D, f) : with_group<kHalves>(q.D, f);
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
  with_kernel(d, [&](auto group, auto pairs) {
    constexpr int kG = decltype(group)::value;
    QkParams p = params_of(d, kG, 1);
    p.side[0].x = in(q); p.side[0].y = out(q_out);
    p.side[1].x = in(k); p.side[1].y = out(k_out);
    launch_forward<kG, decltype(pairs)::value>(p, static_cast<hipStream_t>(stream));
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
  if (dq_weight && dk_weight) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(dq_weight), b = reinterpret_cast<uintptr_t>(dk_weight);
    if ((a < b ? b - a : a - b) < static_cast<uintptr_t>(d.D) * (d.weight_type == OSDP_F32 ? 4 : 2))
      return bad(OSDP_ERR_INVALID_ARG, "the two weight gradients share memory");
  }
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
  with_kernel(d, [&](auto group, auto pairs) {
    constexpr int kG = decltype(group)::value;
    QkParams p = params_of(d, kG, kBackwardUnroll);
    p.side[0].x = in(d.norm ? q : nullptr); p.side[0].dy = in(dq_out); p.side[0].y = out(dq); p.side[0].dweight = dq_weight;
    p.side[1].x = in(d.norm ? k : nullptr); p.side[1].dy = in(dk_out); p.side[1].y = out(dk); p.side[1].dweight = dk_weight;
    p.planes = sums ? static_cast<float *>(workspace) : nullptr;
    if (grid.all > 0) launch_backward<kG, decltype(pairs)::value>(p, grid, hs);
    last = p;
  });
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && sums) {
    hipLaunchKernelGGL(qk_weight_kernel, dim3((d.D + 15) / 16, 2), dim3(1024), 0, hs, last, grid.queries, grid.all);
    e = hipGetLastError();
  }
  return hip_status(e, "launching the norms of queries and keys");
}

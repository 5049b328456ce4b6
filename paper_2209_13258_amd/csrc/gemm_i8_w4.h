// Tiles of the 8-bit product for many tokens: four waves, accumulators in AGPRs, one workgroup walking through its tiles, as in
// gemm_w4.h and gemm_w4p.h, whose operand layout and loads these kernels share.  To those a row of 8-bit integers is a row of
// half as many 16-bit elements: a K block of 64 of them is 128 integers, and the 16 bytes a lane holds for a matrix step are
// 16 consecutive integers of v_mfma_i32_16x16x64_i8 instead of 8 bf16 of v_mfma_f32_16x16x32_bf16.  The two instructions take
// the same operands' bytes in the same time, so the balance of reads, loads and matrix steps that those kernels were built for holds here too,
// at twice the products.
//
// What bounds them: 4096 tokens 8192 -> 32768 on walking tiles of 256 x 256 take 850 us (2.6e15 operations a second) with random
// integers and 764 with zeros, so the card's power, not the schedule; 33 tokens of the same weight on tiles of 64 x 64 take 48 us (5.6 TB/s),
// the weight's bytes; 500 tokens 2560 -> 10240, 320 tiles of 128 x 128 on 256 compute units, 21 us for the 13 that their
// operations cost a full card: the second round of tiles.
#pragma once
#include <atomic>
#include "gemm_i8.h"
#include "gemm_w4p.h"

namespace osdp {
namespace {

__device__ __forceinline__ void i8_mma_agpr(i32x4 &c, bf16x8 a_rows, bf16x8 b_cols) {
  asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+a"(c) : "v"(b_cols), "v"(a_rows));
}
__device__ __forceinline__ void i8_acc_clear(i32x4 &c, bf16x8 zero) {
  asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %1, 0" : "+a"(c) : "v"(zero));
}
__device__ __forceinline__ i32x4 i8_acc_read(const i32x4 &c) {
  int x0, x1, x2, x3;
  asm volatile("v_accvgpr_read_b32 %0, %4\n\tv_accvgpr_read_b32 %1, %5\n\tv_accvgpr_read_b32 %2, %6\n\tv_accvgpr_read_b32 %3, %7"
               : "=v"(x0), "=v"(x1), "=v"(x2), "=v"(x3) : "a"(c[0]), "a"(c[1]), "a"(c[2]), "a"(c[3]));
  return i32x4{x0, x1, x2, x3};
}

// Four sums as Y: both scales, then two bf16 to a register.
__device__ __forceinline__ uint2 i8_scaled(i32x4 c, float st, f32x4 so) {
  return uint2{pack_bf16x2(static_cast<float>(c[0]) * st * so[0], static_cast<float>(c[1]) * st * so[1]),
               pack_bf16x2(static_cast<float>(c[2]) * st * so[2], static_cast<float>(c[3]) * st * so[3])};
}

// What a launch needs.  Lengths along the reduction are counted in pairs of integers (16 bits), as the shared operand code does.
struct I8Tiles {
  int32_t T, O, K;
  const uint16_t *xq;
  int64_t ldx, ldw;            // of Xq and Wq, in pairs
  ShardTable shards;
  int32_t rows_each;           // output channels to a shard
  int32_t per_shard;           // columns of tiles to a shard
  uint16_t *y;
  int64_t ldy;
  const float *x_scale, *w_scale;
  int32_t tiles_m, tiles_n;
  int32_t parts, part_blocks;  // workgroups that share a tile's reduction, K blocks to each (the last may have fewer)
  uint64_t *sums;              // parts > 1: MB * NB * 512 for each workgroup, in the order its lanes hold them
  uint32_t *arrived;           // parts > 1: a counter for each tile, 0 when the launch begins
};

// Both operands of a tile, K block by K block.  Columns of tiles do not reach over the end of a shard, and begin on multiples of 8 so
// that results can be stored 16 bytes at a time: where a shard's first channel is no such multiple, its first tile begins with
// up to 7 channels of the shard before, which it reads as zeros (their offsets are negative, so out of range) and does not store.
template <class OpA, class OpB, int BM, int BN>
struct I8Source {
  OperandSource<OpA, true, BM, 64> a;
  OperandSource<OpB, true, BN, 64> b;
  int32_t block, nb;

  static __device__ __forceinline__ void columns(const I8Tiles &p, int tn, int *n0, int *n_begin, int *n_end, int *shard) {
    const int s = __builtin_amdgcn_readfirstlane(tn / p.per_shard), first = s * p.rows_each;
    *shard = s;
    const int n = (first & ~7) + (tn - s * p.per_shard) * BN;
    // (what the loads' buffers are made of has to be in scalar registers, as far as the compiler can see)
    *n0 = __builtin_amdgcn_readfirstlane(n);
    *n_begin = __builtin_amdgcn_readfirstlane(max(n, first));
    *n_end = __builtin_amdgcn_readfirstlane(min(n + BN, first + p.rows_each));
  }
  // Block 0 of the tile of rows m0 .. and tile column tn, reducing over k0 .. k0 + K.
  __device__ __forceinline__ void begin(const I8Tiles &p, int m0, int tn, int64_t k0, int K, int wave, int lane) {
    int n0, n_begin, n_end, s;
    columns(p, tn, &n0, &n_begin, &n_end, &s);
    const uint16_t *w = static_cast<const uint16_t *>(p.shards.p[s]) + static_cast<int64_t>(n_begin - s * p.rows_each) * p.ldw;
    a.begin(p.xq + static_cast<int64_t>(m0) * p.ldx + k0, p.ldx, p.T - m0, wave, lane);
    b.begin(w + k0, p.ldw, __builtin_amdgcn_readfirstlane(max(n_end - n_begin, 0)), wave, lane);
    b.lane -= static_cast<uint32_t>(n_begin - n0) * b.ld2;
    nb = (K + 63) / 64;
    block = -1;
    cut(K, wave, lane);
  }
  // What a block that is not full holds, and what follows the last one: less, and nothing.
  __device__ __forceinline__ void cut(int K, int wave, int lane) {
    const int left = K - ++block * 64;
    if (__builtin_expect(left < 64, 0)) {
      a.cut(left > 0 ? left : 0, wave, lane);
      b.cut(left > 0 ? left : 0, wave, lane);
    }
  }
  __device__ __forceinline__ void next(int K, int wave, int lane) {
    a.next();
    b.next();
    cut(K, wave, lane);
  }
};

// The scales of a lane's rows and columns of a wave's share of a tile.  They are asked for when the tile begins: at its end, where
// nothing else is under way, they would cost trips to memory (16384 tokens 2560 -> 2560: 133.9 us, so 131.9).
template <int MB, int NB>
struct I8Scales {
  float st[MB];
  f32x4 so[NB];
  __device__ __forceinline__ void load(const I8Tiles &p, int m_base, int n_base, int l16, int q) {
#pragma unroll
    for (int b = 0; b < MB; ++b) st[b] = p.x_scale[min(m_base + 16 * b + l16, p.T - 1)];
#pragma unroll
    for (int b = 0; b < NB; ++b) so[b] = *reinterpret_cast<const f32x4 *>(p.w_scale + min(n_base + 16 * b + 4 * q, p.O - 4));
  }
};

// One wave's share of a tile, 16 * MB x 16 * NB from row m_base and column n_base on: blocks 2 i and 2 i + 1 change lanes, so that
// a lane stores 8 columns.
template <int MB, int NB, class Read>
__device__ __forceinline__ void i8_store_tile(const I8Tiles &p, const I8Scales<MB, NB> &scales, Read &&read, int m_base, int n_base,
                                              int n_begin, int n_end, int l16, int q) {
  static_assert(NB % 2 == 0, "blocks are stored in pairs");
  const int m = m_base + l16, col = 16 * (q & 1) + 8 * (q >> 1);
  uint16_t *dst = p.y + static_cast<int64_t>(m) * p.ldy + n_base + col;
  static_for<MB>([&](auto bm_) {
    constexpr int bm = decltype(bm_)::value;
    const bool row = m + 16 * bm < p.T;
    const float st = scales.st[bm];
    static_for<NB / 2>([&](auto i_) {
      constexpr int i = decltype(i_)::value;
      const uint2 c = i8_scaled(read(Int<bm>{}, Int<2 * i>{}), st, scales.so[2 * i]);
      const uint2 d = i8_scaled(read(Int<bm>{}, Int<2 * i + 1>{}), st, scales.so[2 * i + 1]);
      const auto lo = __builtin_amdgcn_permlane16_swap(c.x, d.x, false, false);
      const auto hi = __builtin_amdgcn_permlane16_swap(c.y, d.y, false, false);
      const int n = n_base + 32 * i + col;
      if (row && n >= n_begin && n + 8 <= n_end) {
        __builtin_nontemporal_store(osdp_u32x4{lo[0], hi[0], lo[1], hi[1]}, (__attribute__((address_space(1))) osdp_u32x4 *)(dst + 32 * i));
      } else if (row && n + 8 > n_begin && n < n_end) {  // (the ends of a shard that are no multiples of 8)
        const uint32_t w[4] = {lo[0], hi[0], lo[1], hi[1]};
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (n + e >= n_begin && n + e < n_end) dst[32 * i + e] = static_cast<uint16_t>(w[e >> 1] >> (16 * (e & 1)));
      }
      __builtin_amdgcn_sched_barrier(0);
    });
    dst += static_cast<int64_t>(16) * p.ldy;
  });
}

// kSlots: K blocks of LDS.  Two: any number of tiles to a workgroup.  More: launches that do not fill the card, with one tile, or a
// part of its reduction, to a workgroup and loads further ahead.  The parts of a tile meet in memory: each writes its sums, and
// the last one to arrive (a counter says which; nobody waits) adds the others' to its own and stores the tile.  They are
// consecutive workgroups of one XCD, whose L2 then holds all of it.
//
// kTurn (with more than two slots, where the weight's bytes are the bound): a workgroup begins at another block of the reduction than those of
// the next columns and takes the blocks ahead of it at the end (see kI8Turn).  us: 33 tokens 8192 -> 32768 59.1, with turns 52.9; 16384 -> 16384
// 63.2 and 56.1, 24576 -> 8192 48.6 and 49.4; 100 tokens 8192 -> 32768 65.3 and 54.4.  Not so rows that lie apart otherwise, 33 tokens 6144 -> 24576
// 36.4 and 37.2, or several rows of tiles, of which those of a column are to read the same weights at a time: 160 tokens 4096 -> 4096 14.3 and
// 15.5, 1000 26.2 and 27.6.
template <int MB, int NB, int kSlots, bool kTurn>
__device__ __forceinline__ void i8_w4_tiles(const I8Tiles &p) {
  constexpr int WM = 16 * MB, WN = 16 * NB, BM = 2 * WM, BN = 2 * WN;
  using OpA = W4Operand<true, MB>;
  using OpB = W4Operand<true, NB>;
  constexpr int kAhead = kSlots == 2 ? 2 : kSlots - 1;   // (see gemm_w4_tile)
  constexpr int kSlotElems = OpA::kElems + OpB::kElems;
  constexpr int L = OpA::kLoads + OpB::kLoads;
  static_assert(w4_all_placed(MB, NB, L), "a K step must hold the next one's fragment reads and a block's loads");
  extern __shared__ __attribute__((aligned(1024))) uint16_t smem[];
  const int tid = threadIdx.x;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = (wave >> 1) * WM, wn = (wave & 1) * WN;
  const int l16 = lane & 15, q4 = lane >> 4;
  const int tiles_m = p.tiles_m, tiles_n = p.tiles_n, tiles = tiles_m * tiles_n, G = gridDim.x;
  int first = logical_block(), part = 0;
  int64_t k0 = 0;
  int K = p.K;
  if constexpr (kSlots > 2) {
    if (p.parts > 1) {
      const int id = first;
      first = __builtin_amdgcn_readfirstlane(id / p.parts);
      part = id - first * p.parts;
      k0 = static_cast<int64_t>(part) * p.part_blocks * 64;
      K = min(p.K - static_cast<int>(k0), p.part_blocks * 64);
    }
  }
  const int nb = (K + 63) / 64;
  const int my_tiles = kSlots == 2 ? __builtin_amdgcn_readfirstlane((tiles - first + G - 1) / G) : 1;

  static_assert(!kTurn || kSlots > 2);
  int lt = first, turn = 0;  // (blocks that are left for the end)
  if constexpr (kTurn) {
    int tm, tn;
    tile_of_pid(first, tiles_m, tiles_n, &tm, &tn);
    turn = __builtin_amdgcn_readfirstlane(tn % nb);
  }
  I8Source<OpA, OpB, BM, BN> src;
  auto load_tile = [&](int tile, int from, int length) {
    int tm, tn;
    tile_of_pid(tile, tiles_m, tiles_n, &tm, &tn);
    src.begin(p, tm * BM, tn, k0 + from, length, wave, lane);
  };
  int length = K - turn * 64;  // of the reduction that the source is at
  auto block_issued = [&]() {
    if (kSlots == 2 && src.block + 1 == nb && lt + G < tiles) {
      lt += G;
      load_tile(lt, 0, K);
    } else if (kTurn && turn > 0 && src.block + 1 == src.nb) {
      length = turn * 64;
      turn = 0;
      load_tile(lt, 0, length);
    } else {
      src.next(length, wave, lane);
    }
  };
  const uint32_t lds_base = lds_address(smem);
  const uint32_t dstA = lds_base + OpA::first_chunk(wave) * 1024;
  const uint32_t dstB = lds_base + OpA::kElems * 2 + OpB::first_chunk(wave) * 1024;
  auto issue = [&](int slot, auto idx) {
    constexpr int i = decltype(idx)::value;
    if constexpr (i < OpA::kLoads) src.a.template load<i>(dstA + slot * (kSlotElems * 2));
    else src.b.template load<i - OpA::kLoads>(dstB + slot * (kSlotElems * 2));
  };

  int ct = first, cb = 0, m0c = 0, n0c = 0, n_beginc = 0, n_endc = 0;
  I8Scales<MB, NB> scales;
  i32x4 acc[MB][NB];
#pragma unroll
  for (int bm = 0; bm < MB; ++bm)
#pragma unroll
    for (int bn = 0; bn < NB; ++bn)
      asm volatile("" : "=a"(acc[bm][bn]));  // (a value to the compiler, no instruction: begin_tile sets the registers)
  bf16x8 zero;
#pragma unroll
  for (int i = 0; i < 8; ++i) zero[i] = static_cast<__bf16>(0.0f);
  asm volatile("s_nop 1" : "+v"(zero));  // (written once, here: see gemm_w4p_tiles)
  auto begin_tile = [&](int tile) {
    int tm, tn, shard;
    tile_of_pid(tile, tiles_m, tiles_n, &tm, &tn);
    m0c = tm * BM;
    src.columns(p, tn, &n0c, &n_beginc, &n_endc, &shard);
    scales.load(p, m0c + wm, n0c + wn, l16, q4);
    static_for<MB * NB>([&](auto idx) {
      constexpr int i = decltype(idx)::value, bn = i / MB, bm = i % MB;  // the order of the K loop's steps
      i8_acc_clear(acc[bm][bn], zero);
    });
  };

  load_tile(lt, turn * 64, length);
  static_for<kAhead>([&](auto b) {
    static_for<L>([&](auto i) { issue(decltype(b)::value, i); });
    block_issued();
  });
  begin_tile(ct);
  wait_vmcnt<(kAhead - 1) * L>();
  __builtin_amdgcn_s_barrier();
  bf16x8 fa[2][MB], fb[2][NB];
  auto first_fragments = [&](int slot) {
    const uint16_t *sA = smem + slot * kSlotElems, *sB = sA + OpA::kElems;
#pragma unroll
    for (int b = 0; b < MB; ++b) fa[0][b] = OpA::frag(sA, wm + b * 16, 0, lane);
#pragma unroll
    for (int b = 0; b < NB; ++b) fb[0][b] = OpB::frag(sB, wn + b * 16, 0, lane);
  };
  first_fragments(0);

  auto kstep = [&](auto par, auto load_, const uint16_t *rs, int rk, int ls) {
    constexpr int P = decltype(par)::value, Q = P ^ 1;
    constexpr bool kLoad = decltype(load_)::value != 0;
    const uint16_t *nA = rs, *nB = rs + OpA::kElems;
    static_for<MB * NB>([&](auto idx) {
      constexpr int i = decltype(idx)::value, bn = i / MB, bm = i % MB;
      i8_mma_agpr(acc[bm][bn], fa[P][bm], fb[P][bn]);
      if constexpr (w4_read_behind(i, MB, NB) >= 0) {
        constexpr int r = w4_read_behind(i, MB, NB);
        if constexpr (r == 0) fb[Q][0] = OpB::frag(nB, wn, rk, lane);
        else if constexpr (r <= MB) fa[Q][r - 1] = OpA::frag(nA, wm + (r - 1) * 16, rk, lane);
        else fb[Q][r - MB] = OpB::frag(nB, wn + (r - MB) * 16, rk, lane);
      }
      if constexpr (kLoad && w4_load_behind(i, MB * NB, L) >= 0) {
        issue(ls, Int<w4_load_behind(i, MB * NB, L)>{});
        if constexpr (w4_load_behind(i, MB * NB, L) == L - 1) block_issued();
      }
      __builtin_amdgcn_sched_barrier(0);
    });
  };

  int cur = 0, fill = kSlots == 2 ? 0 : kAhead;
  auto after = [](int slot) { return slot + 1 == kSlots ? 0 : slot + 1; };
  const int total = my_tiles * nb;
  for (int g = 0; g < total; ++g) {
    const uint16_t *sc = smem + cur * kSlotElems, *sn = smem + after(cur) * kSlotElems;
    kstep(Int<0>{}, Int<0>{}, sc, 1, 0);
    wait_vmcnt<(kAhead - 2) * L>();
    if constexpr (kSlots == 2) __builtin_amdgcn_s_waitcnt((15) | (7 << 4) | (0 << 8) | (3 << 14));  // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    kstep(Int<1>{}, Int<1>{}, sn, 0, fill);
    cur = after(cur);
    fill = after(fill);
    if (++cb == nb) {
      cb = 0;
      asm volatile("s_nop 15");
      asm volatile("s_nop 15");
      int l16e = l16, q4e = q4;
      asm volatile("" : "+v"(l16e), "+v"(q4e));  // (the epilogue's addresses are worked out here, not ahead of the loop)
      if constexpr (kSlots > 2) {
        if (p.parts > 1) break;
      }
      i8_store_tile<MB, NB>(p, scales, [&](auto bm, auto bn) { return i8_acc_read(acc[decltype(bm)::value][decltype(bn)::value]); },
                            m0c + wm, n0c + wn, n_beginc, n_endc, l16e, q4e);
      if constexpr (kSlots == 2) {
        ct += G;
        if (ct < tiles) begin_tile(ct);
        first_fragments(cur);  // (read again, so that none of them has to outlive the epilogue)
      }
    }
  }
  wait_vmcnt<0>();  // surplus loads must have landed before the workgroup gives its LDS back
  if constexpr (kSlots > 2) {
    if (p.parts <= 1) return;
    i32x4 sum[MB][NB];
    uint64_t *own = p.sums + static_cast<int64_t>(first) * p.parts * (MB * NB * 512) + tid;
    static_for<MB * NB>([&](auto idx) {
      constexpr int i = decltype(idx)::value, bn = i / MB, bm = i % MB;
      sum[bm][bn] = i8_acc_read(acc[bm][bn]);
      uint64_t *at = own + (static_cast<int64_t>(part) * (MB * NB) + i) * 512;
      const uint64_t lo = static_cast<uint32_t>(sum[bm][bn][0]) | static_cast<uint64_t>(static_cast<uint32_t>(sum[bm][bn][1])) << 32;
      const uint64_t hi = static_cast<uint32_t>(sum[bm][bn][2]) | static_cast<uint64_t>(static_cast<uint32_t>(sum[bm][bn][3])) << 32;
      __hip_atomic_store(at, lo, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __hip_atomic_store(at + 256, hi, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    });
    __shared__ uint32_t before;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) before = __hip_atomic_fetch_add(p.arrived + first, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (before + 1 != static_cast<uint32_t>(p.parts)) return;
    if (tid == 0) __hip_atomic_store(p.arrived + first, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // (for the launch over the next slice)
    for (int s = 0; s < p.parts; ++s) {
      if (s == part) continue;
      const uint64_t *other = own + static_cast<int64_t>(s) * (MB * NB * 512);
      static_for<MB * NB>([&](auto idx) {
        constexpr int i = decltype(idx)::value, bn = i / MB, bm = i % MB;
        const uint64_t lo = __hip_atomic_load(other + i * 512, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const uint64_t hi = __hip_atomic_load(other + i * 512 + 256, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        sum[bm][bn] += i32x4{static_cast<int>(lo), static_cast<int>(lo >> 32), static_cast<int>(hi), static_cast<int>(hi >> 32)};
      });
    }
    i8_store_tile<MB, NB>(p, scales, [&](auto bm, auto bn) { return sum[decltype(bm)::value][decltype(bn)::value]; },
                          m0c + wm, n0c + wn, n_beginc, n_endc, l16, q4);
  }
}

template <int MB, int NB, int kSlots, bool kTurn>
__global__ __launch_bounds__(256, kSlots * (32 * (MB + NB) * 128) <= 80 * 1024 ? 2 : 1)
void i8_w4_kernel(I8Tiles p) {
  i8_w4_tiles<MB, NB, kSlots, kTurn>(p);
}

constexpr int kI8Cus = 256;

// Columns of tiles of BN channels that cover all shards.
inline int64_t i8_shard_tiles(int64_t rows_each, int BN) { return ((rows_each % 8 ? rows_each + 7 : rows_each) + BN - 1) / BN; }

template <int MB, int NB, int kSlots, bool kTurn = false>
hipError_t launch_i8_tiles(const I8Problem &p, int parts, hipStream_t stream) {
  constexpr int BM = 32 * MB, BN = 32 * NB, kLds = kSlots * (BM + BN) * 128;
  if constexpr (kSlots > 2 && !kTurn)
    if (p.I % kI8Turn == 0 && p.T <= 2 * BM) return launch_i8_tiles<MB, NB, kSlots, true>(p, parts, stream);
  constexpr int kPerCu = kLds <= 80 * 1024 ? 2 : 1;
  static std::atomic<uint64_t> ready{0};  // devices that know the kernel's LDS size
  I8Tiles t{};
  t.T = p.T; t.O = p.O; t.K = p.I / 2;
  t.xq = reinterpret_cast<const uint16_t *>(p.xq); t.ldx = p.ldq / 2; t.ldw = p.I / 2;
  t.shards = p.shards; t.rows_each = p.rows_each;
  t.y = p.y; t.ldy = p.ldy; t.x_scale = p.x_scale; t.w_scale = p.w_scale;
  t.per_shard = static_cast<int32_t>(i8_shard_tiles(p.rows_each, BN));
  const int64_t tiles_n = static_cast<int64_t>(p.O / p.rows_each) * t.per_shard;
  const int64_t tiles_m = (p.T + BM - 1) / BM, tiles = tiles_m * tiles_n;
  if (tiles >= (1ll << 31)) return hipErrorInvalidValue;
  t.tiles_m = static_cast<int32_t>(tiles_m); t.tiles_n = static_cast<int32_t>(tiles_n);
  const int blocks = (t.K + 63) / 64;
  t.part_blocks = (blocks + parts - 1) / parts;
  t.parts = (blocks + t.part_blocks - 1) / t.part_blocks;
  t.sums = static_cast<uint64_t *>(p.sums);
  t.arrived = p.arrived;
  int64_t grid = std::min<int64_t>(tiles, kI8Cus * kPerCu);
  if (kSlots > 2) grid = tiles * t.parts;
  if (grid > (1 << 24) || (t.parts > 1 && (kSlots == 2 || !t.sums || tiles > kI8MostTiles || grid * (MB * NB * 4096) > static_cast<int64_t>(kI8SumBytes))))
    return hipErrorInvalidValue;
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 0 || dev >= 64) return hipErrorInvalidDevice;
  if (!(ready.load(std::memory_order_relaxed) >> dev & 1)) {  // (a benign race sets the same attribute twice)
    e = hipFuncSetAttribute(reinterpret_cast<const void *>(i8_w4_kernel<MB, NB, kSlots, kTurn>), hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
    if (e != hipSuccess) return e;
    ready.fetch_or(1ull << dev);
  }
  hipLaunchKernelGGL((i8_w4_kernel<MB, NB, kSlots, kTurn>), dim3(static_cast<unsigned>(grid)), dim3(256), kLds, stream, t);
  return hipGetLastError();
}

}  // namespace
}  // namespace osdp

// Products of the training calls on the 5th-generation tensor cores (tcgen05.mma, accumulators in tensor memory).
//
// A pair of CTAs (cta_group::2) owns a 256 x 256 tile of C = A B^T: each holds 128 rows of A and half of B's 256 rows of a
// 64-deep K block in one of six 32 KB stages, and 128 x 256 accumulators, twice.  Both operands may lie K-major or MN-major in
// memory (the tensor core takes either from the 128-byte-swizzled boxes that the tensor-map copies leave), so none of the six
// products of a training step needs a transposed copy.  kGateUp: the even CTA's half of B is W_g, the odd one's W_up, of
// the same 128 neurons, so that z and u of a neuron are in the same lane of tensor memory, 128 columns apart.
//
//   warp 0      one thread issues the copies of its CTA; their bytes complete on the even CTA's barrier
//   warp 1      even CTA: one thread issues the MMAs of both
//   warps 4-11  epilogue: lane quadrant = warp mod 4, the two warps of a quadrant share the columns
//
// PROMOTE: the tensor cores truncate when they add onto an accumulator (a sum over K = 2688 comes out low by 1e-6 of its
// typical size).  Where a sum leaves as fp32, short runs of K get an accumulator of their own and the epilogue warps add
// them up in registers, rounding to nearest: fp32 storage, whose operands are three bf16 terms each and whose products are the
// six of the terms' products above 2^-27 (smallest first), 256 deep a run; and dh, whose dz is summed over the tokens in
// fp32, 1024 deep a run.
//
// Tiles are dealt to the pairs round robin.  What is left for a last, partly idle round is cut along K instead so that all pairs get
// the same share of it: each leaves its piece of a tile as fp32 in a workspace, and whoever finishes last, warp by warp, adds up
// the pieces in their order in K.  Nobody waits for anybody, and which warp adds does not change what it adds.
// Every wait is bounded by a cycle budget; on expiry the status word is set, all roles wind down and tensor memory is given back.
#include <cuda.h>

#include "fused_kernel.cuh"
#include "tcgen05.cuh"
#include "train_kernels.cuh"

namespace sffn {
namespace {

using namespace tc;

constexpr int kRows = 256, kCols = 256;      // of a pair's tile
constexpr int kDeep = 64;                    // bf16 elements of one 128-byte swizzle row
constexpr int kHalfBytes = 128 * kDeep * 2;  // one operand's share of a stage
constexpr int kStageBytes = 2 * kHalfBytes;
constexpr int kStages = 6;
constexpr int kThreads = 384;
constexpr int kEpilogueWarps = 8;
constexpr int kSmemBytes = kStages * kStageBytes + 1024 + 256;
constexpr int kLimbBlocks = 4;               // fp32: K blocks of a run, which is six times as long
constexpr int kLimbUnit = 6 * kLimbBlocks;
constexpr int kRunBlocks = 16;               // dh: K blocks of a run

struct UmmaParams {
  TrainEpilogue epi;
  int epilogue, f32;
  int m_tiles, n_tiles, tiles;        // tiles = m_tiles * n_tiles * batch
  int blocks;                         // K blocks of a part (fp32: rounded up to runs)
  int units, unit_blocks, run_units;  // a tile's K in units (what is not cut), K blocks of a unit, units of a run
  int whole;                          // tiles dealt whole; the others are cut along K
  int batch, tile_cols;
  int a_mn, b_mn;
  float* partial;
  uint32_t* counters;
  int32_t* status;
  long long budget;
};

struct Maps {
  CUtensorMap a[3], b[3];
};

// One piece of work of a pair of CTAs: units [u0, u1) of a tile.
struct Item {
  int tile, u0, u1;
};
// A pair's items in order: its share of the tiles that are cut, then whole tiles.
struct Walk {
  int pairs, pair, cut, units, lo, hi, next;  // lo, hi: its units of all cut tiles in a row
  __device__ __forceinline__ Walk(const UmmaParams& p, int pairs_, int pair_) {
    pairs = pairs_; pair = pair_; units = p.units;
    cut = p.tiles - p.whole;
    lo = share(pair);
    hi = share(pair + 1);
    next = pair;
  }
  __device__ __forceinline__ int share(int q) const { return (int)((long long)cut * units * q / pairs); }
  __device__ __forceinline__ bool step(const UmmaParams& p, Item& it) {
    if (lo < hi) {
      const int t = lo / units;
      it.tile = p.whole + t;
      it.u0 = lo - t * units;
      it.u1 = min(units, hi - t * units);
      lo = t * units + it.u1;
      return true;
    }
    if (next >= p.whole) return false;
    it.tile = next;
    it.u0 = 0;
    it.u1 = units;
    next += pairs;
    return true;
  }
};

// Where a tile lies: groups of eight tile rows, column by column, so that what runs at one time shares rows and columns in L2.
struct Place {
  int batch, m, n;
};
__device__ __forceinline__ Place place_of(const UmmaParams& p, int tile) {
  constexpr int kGroup = 8;
  const int per = p.m_tiles * p.n_tiles;
  Place at;
  at.batch = tile / per;
  tile -= at.batch * per;
  const int group = tile / (kGroup * p.n_tiles), first = group * kGroup, rows = min(kGroup, p.m_tiles - first);
  tile -= first * p.n_tiles;
  at.m = first + tile % rows;
  at.n = tile / rows;
  return at;
}

// K block j of unit u: which part, which block of it, which terms.
__device__ __forceinline__ void block_of(const UmmaParams& p, int u, int j, int& part, int& kb, int& la, int& lb) {
  if (p.unit_blocks == 1) {
    part = u >= p.blocks ? 1 : 0;
    kb = u - part * p.blocks;
    la = lb = 0;
  } else {
    const int first = u * kLimbBlocks;
    part = first >= p.blocks ? 1 : 0;
    kb = first - part * p.blocks + j % kLimbBlocks;
    const int product = j / kLimbBlocks;  // (0,2) (2,0) (1,1) (0,1) (1,0) (0,0)
    la = product == 1 ? 2 : product == 2 || product == 4 ? 1 : 0;
    lb = product == 0 ? 2 : product == 2 || product == 3 ? 1 : 0;
  }
}

// ---- sixteen columns of a row --------------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ void st8(void* p, const uint32_t* w, bool wide) {  // 32 bytes
  if (wide) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]),
                 "r"(w[6]), "r"(w[7])
                 : "memory");
  } else {
    reinterpret_cast<uint4*>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
    reinterpret_cast<uint4*>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
  }
}
__device__ __forceinline__ void ld8(const void* p, uint32_t* w, bool wide) {
  if (wide) {
    asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                 : "l"(p)
                 : "memory");
  } else {
    const uint4 a = reinterpret_cast<const uint4*>(p)[0], b = reinterpret_cast<const uint4*>(p)[1];
    w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
    w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
  }
}

// Stores the first n of sixteen values from element `at` on; `wide`: 32-byte accesses are aligned.
template <bool F32>
__device__ __forceinline__ void store16(void* base, int64_t at, const float* v, int n, bool wide) {
  if constexpr (F32) {
    float* p = static_cast<float*>(base) + at;
    if (n == 16) {
      st8(p, reinterpret_cast<const uint32_t*>(v), wide);
      st8(p + 8, reinterpret_cast<const uint32_t*>(v) + 8, wide);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (i < n) p[i] = v[i];
    }
  } else {
    __nv_bfloat16* p = static_cast<__nv_bfloat16*>(base) + at;
    if (n == 16) {
      uint32_t w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
      st8(p, w, wide);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (i < n) p[i] = __float2bfloat16(v[i]);
    }
  }
}
// The three bf16 terms of sixteen values.
__device__ __forceinline__ void store16_limbs(void* base, int64_t at, int64_t limb, float* v, int n, bool wide) {
#pragma unroll
  for (int l = 0; l < 3; ++l) {
    store16<false>(static_cast<__nv_bfloat16*>(base) + l * limb, at, v, n, wide);
    if (l < 2) {
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] -= __bfloat162float(__float2bfloat16(v[i]));
    }
  }
}
template <bool F32>
struct Raw16 {
  uint32_t w[F32 ? 16 : 8];
  __device__ __forceinline__ void load(const void* base, int64_t at, int n, bool wide) {
    constexpr int kWords = F32 ? 16 : 8;
    if (n == 16) {
      const char* p = static_cast<const char*>(base) + at * (F32 ? 4 : 2);
      ld8(p, w, wide);
      if constexpr (F32) ld8(p + 32, w + 8, wide);
    } else {
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[i] = 0;
      if constexpr (F32) {
        const uint32_t* p = static_cast<const uint32_t*>(base) + at;
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (i < n) w[i] = p[i];
      } else {
        const uint16_t* p = static_cast<const uint16_t*>(base) + at;
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (i < n) w[i / 2] |= (uint32_t)p[i] << (16 * (i & 1));
      }
    }
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (F32) return __uint_as_float(w[i]);
    else return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
  }
};

// Activations of sixteen values, the choice made once: inside the loops it would be made, and its code be there, sixteen times.
template <bool FAST>
__device__ __forceinline__ void act16(int act, const float* t, float* v) {
  if (act == kActNone) {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = t[i];
  } else if (act == kActRelu) {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = train_act<FAST>(kActRelu, t[i]);
  } else if (act == kActSqRelu) {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = train_act<FAST>(kActSqRelu, t[i]);
  } else if (act == kActRsPlus) {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = train_act<FAST>(kActRsPlus, t[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = train_act<FAST>(kActSilu, t[i]);
  }
}
template <bool FAST, int ACT, typename Raw>
__device__ __forceinline__ void slope16_of(const Raw& t, float* v, float* d) {
#pragma unroll
  for (int i = 0; i < 16; ++i) train_act_slope<FAST>(ACT, t.get(i), v[i], d[i]);
}
template <bool FAST, typename Raw>
__device__ __forceinline__ void slope16(int act, const Raw& t, float* v, float* d) {
  if (act == kActNone) slope16_of<FAST, kActNone>(t, v, d);
  else if (act == kActRelu) slope16_of<FAST, kActRelu>(t, v, d);
  else if (act == kActSqRelu) slope16_of<FAST, kActSqRelu>(t, v, d);
  else if (act == kActRsPlus) slope16_of<FAST, kActRsPlus>(t, v, d);
  else slope16_of<FAST, kActSilu>(t, v, d);
}

// Sums of sixteen columns over the lanes of a warp: lanes 2 i and 2 i + 1 get column i's (in halves of what is left, five
// exchanges deep, sixteen shuffles).
__device__ __forceinline__ float column_sum(float* v, int lane) {
#pragma unroll
  for (int width = 8; width >= 1; width >>= 1) {
    const bool upper = lane & (2 * width);
#pragma unroll
    for (int i = 0; i < width; ++i) {
      const float send = upper ? v[i] : v[i + width], keep = upper ? v[i + width] : v[i];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, send, 2 * width);
    }
  }
  return v[0] + __shfl_xor_sync(0xffffffffu, v[0], 1);
}

template <int EPI, bool F32, bool PROMOTE>
__global__ void __launch_bounds__(kThreads, 1) train_umma_kernel(const __grid_constant__ UmmaParams p, const __grid_constant__ Maps maps) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ int abort_word;
  __shared__ uint32_t tmem_slot;
  __shared__ __align__(8) uint64_t bars[2 * kStages + 4];
  volatile int* const abort_flag = &abort_word;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t full = smem_u32(bars), empty = full + 8 * kStages, acc_full = empty + 8 * kStages, acc_empty = acc_full + 16;
  const int rank = (int)cluster_rank(), pair = (int)blockIdx.x >> 1, pairs = (int)gridDim.x >> 1;

  if (tid == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(full + 8 * s, 1);
      mbar_init(empty + 8 * s, 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(acc_full + 8 * b, 1);
      mbar_init(acc_empty + 8 * b, 2 * kEpilogueWarps);
    }
    abort_word = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 2) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  fence_before();
  cluster_sync();
  fence_after();
  const uint32_t tmem = tmem_slot;
  pdl_launch_dependents();
  pdl_wait();

  if (warp < 4) {
    if constexpr (PROMOTE) asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    Walk walk(p, pairs, pair);
    Item it;
    if (warp == 0 && lane == 0) {
      int s = 0, phase = 0;
      bool ok = true;
      while (ok && walk.step(p, it)) {
        const Place at = place_of(p, it.tile);
        const int m0 = at.m * kRows + rank * 128;
        const int n0 = at.n * p.tile_cols + (EPI == kEpiGateUp ? 0 : rank * 128);
        for (int u = it.u0; ok && u < it.u1; ++u)
          for (int j = 0; j < p.unit_blocks; ++j) {
            ok = mbar_wait(empty + 8 * s, phase ^ 1, abort_flag, p.status, p.budget);
            if (!ok) break;
            int part, kb, la, lb;
            block_of(p, u, j, part, kb, la, lb);
            const int which = p.batch > 1 ? at.batch : part;
            const CUtensorMap* ma = &maps.a[EPI == kEpiGateUp ? 0 : which];
            const CUtensorMap* mb = &maps.b[EPI == kEpiGateUp ? rank : which];
            const uint32_t bar = map_rank(full + 8 * s, 0), da = ring + s * kStageBytes, db = da + kHalfBytes;
            if (rank == 0) mbar_expect_tx(full + 8 * s, 2 * kStageBytes);
            const int k0 = kb * kDeep;
            if (p.a_mn) {
              tma_tile_3d(da, ma, m0, k0, la, bar);
              tma_tile_3d(da + kHalfBytes / 2, ma, m0 + 64, k0, la, bar);
            } else {
              tma_tile_3d(da, ma, k0, m0, la, bar);
            }
            if (p.b_mn) {
              tma_tile_3d(db, mb, n0, k0, lb, bar);
              tma_tile_3d(db + kHalfBytes / 2, mb, n0 + 64, k0, lb, bar);
            } else {
              tma_tile_3d(db, mb, k0, n0, lb, bar);
            }
            if (++s == kStages) { s = 0; phase ^= 1; }
          }
      }
    } else if (warp == 1 && lane == 0 && rank == 0) {
      const uint32_t idesc = idesc_bf16(kRows, kCols, p.a_mn, p.b_mn);
      const uint64_t a0 = p.a_mn ? desc_mn_major(ring, kHalfBytes / 2) : desc_k_major(ring);
      const uint64_t b0 = p.b_mn ? desc_mn_major(ring + kHalfBytes, kHalfBytes / 2) : desc_k_major(ring + kHalfBytes);
      const uint32_t a_step = p.a_mn ? 2048 >> 4 : 32 >> 4, b_step = p.b_mn ? 2048 >> 4 : 32 >> 4;  // sixteen k
      int s = 0, phase = 0, b = 0, b_phase = 0;
      bool ok = true;
      while (ok && walk.step(p, it)) {
        for (int u = it.u0; ok && u < it.u1;) {
          const int end = PROMOTE ? min(it.u1, u + p.run_units) : it.u1;
          ok = mbar_wait(acc_empty + 8 * b, b_phase ^ 1, abort_flag, p.status, p.budget);
          if (!ok) break;
          fence_after();
          const uint32_t acc = tmem + b * kCols;
          uint32_t more = 0;
          for (int n = (end - u) * p.unit_blocks; n > 0; --n) {
            ok = mbar_wait(full + 8 * s, phase, abort_flag, p.status, p.budget);
            if (!ok) break;
            fence_after();
            const uint32_t off = (uint32_t)(s * kStageBytes) >> 4;
#pragma unroll
            for (int k = 0; k < kDeep / 16; ++k) {
              umma_pair(acc, a0 + off + k * a_step, b0 + off + k * b_step, idesc, more);
              more = 1;
            }
            commit_pair(empty + 8 * s);
            if (++s == kStages) { s = 0; phase ^= 1; }
          }
          if (!ok) break;
          commit_pair(acc_full + 8 * b);
          b ^= 1;
          if (b == 0) b_phase ^= 1;
          u = end;
        }
      }
    }
  } else {
    if constexpr (PROMOTE) asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    const TrainEpilogue& e = p.epi;
    const int quad = warp & 3, half = (warp - 4) >> 2;
    const uint32_t lanes = (uint32_t)(32 * quad) << 16;
    constexpr int kChunks = 8;                                   // of sixteen columns, of a warp
    constexpr int kOut = EPI == kEpiGateUp ? kChunks / 2 : kChunks;  // of sixteen output columns
    // column (in the accumulator) of a chunk: kGateUp: a warp has z and u of 64 neurons, z's chunks first
    auto column = [&](int c) { return EPI == kEpiGateUp ? (c < 4 ? 0 : 128) + 64 * half + 16 * (c & 3) : 128 * half + 16 * c; };
    const uint32_t empty0 = map_rank(acc_empty, 0);
    const uintptr_t wide_out = EPI == kEpiStore ? (uintptr_t)(e.ld_out * (F32 ? 4 : 2)) : (uintptr_t)(e.ld_zu * (F32 ? 4 : 2)) | reinterpret_cast<uintptr_t>(e.z) | reinterpret_cast<uintptr_t>(e.u);
    const bool wide_user = (wide_out & 31) == 0;
    const bool wide_own = EPI != kEpiStore && (e.ld_h & 15) == 0;
    int b = 0, b_phase = 0;
    bool ok = true;
    Walk walk(p, pairs, pair);
    Item it;
    while (ok && walk.step(p, it)) {
      const Place at = place_of(p, it.tile);
      const int m = at.m * kRows + rank * 128 + 32 * quad + lane;
      const int n0 = at.n * p.tile_cols + (EPI == kEpiGateUp ? 64 : 128) * half;  // first output column of this warp
      const bool row = m < e.M;
      // This item's sums, in tensor memory: as the MMAs left them, or added up over the runs and put back where the last run was.
      uint32_t tacc = 0;
      if constexpr (PROMOTE) {
        float acc[16 * kChunks];
        for (int u = it.u0; u < it.u1;) {
          const int end = min(it.u1, u + p.run_units);
          ok = __all_sync(0xffffffffu, mbar_wait(acc_full + 8 * b, b_phase, abort_flag, p.status, p.budget));
          if (!ok) break;
          fence_after();
          tacc = tmem + lanes + b * kCols;
          const bool first = u == it.u0;
#pragma unroll
          for (int c = 0; c < kChunks; ++c) {
            float v[16];
            tmem_ld16(tacc + column(c), v);
            tmem_arrived(v);
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[16 * c + i] = first ? v[i] : acc[16 * c + i] + v[i];
          }
          u = end;
          if (u < it.u1) {
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(empty0 + 8 * b);
            b ^= 1;
            if (b == 0) b_phase ^= 1;
          }
        }
        if (!ok) break;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) tmem_st16(tacc + column(c), acc + 16 * c);
        tmem_stored();
      } else {
        ok = __all_sync(0xffffffffu, mbar_wait(acc_full + 8 * b, b_phase, abort_flag, p.status, p.budget));
        if (!ok) break;
        fence_after();
        tacc = tmem + lanes + b * kCols;
      }
      auto own = [&](int c, float* v) {
        tmem_ld16(tacc + column(c), v);
        tmem_arrived(v);
      };
      // A tile that several pairs share: this warp's part of it is 16 KB of every piece.
      int pieces = 1, mine = 0, first_pair = 0;
      bool finish = true;
      const size_t region = ((size_t)rank * kEpilogueWarps + (warp - 4)) * (16 * kChunks * 32);  // floats
      if (it.u0 > 0 || it.u1 < p.units) {
        const long long all = (long long)(p.tiles - p.whole) * p.units, lo = (long long)(it.tile - p.whole) * p.units, hi = lo + p.units;
        first_pair = (int)(lo * pairs / all);  // the first whose share reaches beyond lo, the last whose share begins before hi
        while (walk.share(first_pair + 1) <= lo) ++first_pair;
        while (first_pair > 0 && walk.share(first_pair) > lo) --first_pair;
        int last = first_pair;
        while (walk.share(last + 1) < hi) ++last;
        pieces = last - first_pair + 1;
        mine = pair - first_pair;
        // a pair's first piece and its second (the one that begins its tile) have places of their own
        float4* out = reinterpret_cast<float4*>(p.partial + (size_t)(2 * pair + (it.u0 == 0 && walk.share(pair) < lo ? 1 : 0)) * (kTrainPieceBytes / 4) + region);
#pragma unroll 2
        for (int c = 0; c < kChunks; ++c) {
          float v[16];
          own(c, v);
#pragma unroll
          for (int q = 0; q < 4; ++q) __stcg(out + (4 * c + q) * 32 + lane, make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]));
        }
        __threadfence();
        __syncwarp();
        uint32_t before = 0;
        uint32_t* counter = p.counters + (it.tile - p.whole) * 16 + rank * kEpilogueWarps + (warp - 4);
        if (lane == 0) before = atomicAdd(counter, 1u);
        before = __shfl_sync(0xffffffffu, before, 0);
        finish = before == (uint32_t)(pieces - 1);
        if (finish) {
          __threadfence();
          if (lane == 0) *counter = 0;
        }
      }
      auto sums = [&](int c, float* v) {
        if (pieces == 1) {
          own(c, v);
          return;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = 0.f;
        const long long lo = (long long)(it.tile - p.whole) * p.units;
#pragma unroll 1
        for (int q = 0; q < pieces; ++q) {
          const int from = first_pair + q;
          const float4* in = reinterpret_cast<const float4*>(p.partial + (size_t)(2 * from + (q > 0 || walk.share(from) == lo ? 0 : 1)) * (kTrainPieceBytes / 4) + region);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float4 f = __ldcg(in + (4 * c + k) * 32 + lane);
            v[4 * k] += f.x; v[4 * k + 1] += f.y; v[4 * k + 2] += f.z; v[4 * k + 3] += f.w;
          }
        }
      };
      if (finish) {
        if constexpr (EPI == kEpiStore) {
          void* out = e.out[at.batch];
          const bool wide = wide_user && (reinterpret_cast<uintptr_t>(out) & 31) == 0;
#pragma unroll 2
          for (int c = 0; c < kOut; ++c) {
            const int n = n0 + 16 * c;
            float v[16];
            sums(c, v);
            if (row && n < e.N) store16<F32>(out, m * e.ld_out + n, v, min(16, e.N - n), wide);
          }
        } else if constexpr (EPI == kEpiGateUp) {
#pragma unroll 1
          for (int c = 0; c < kOut; ++c) {
            const int n = n0 + 16 * c;
            float z[16], u[16];
            sums(c, z);
            sums(c + 4, u);
            const int left = min(16, e.N - n);
            if (e.bias) {
              const float bias = lane < left ? e.bias[n + lane] : 0.f;
#pragma unroll
              for (int i = 0; i < 16; ++i) z[i] += __shfl_sync(0xffffffffu, bias, i);
            }
            if (row && left > 0) {
              if (e.z) {
                store16<F32>(e.z, m * e.ld_zu + n, z, left, wide_user);
                store16<F32>(e.u, m * e.ld_zu + n, u, left, wide_user);
              }
              act16<!F32>(e.act, z, z);
              act16<!F32>(e.act_up, u, u);
#pragma unroll
              for (int i = 0; i < 16; ++i) z[i] *= u[i];
              const int room = (int)min((int64_t)16, e.ld_h - n);
              if constexpr (F32) store16_limbs(e.h, m * e.ld_h + n, e.limb, z, room, wide_own);
              else store16<false>(e.h, m * e.ld_h + n, z, room, wide_own);
            }
          }
        } else {
          Raw16<F32> rz, ru;
          auto fetch = [&](int c) {
            const int n = n0 + 16 * c, left = row ? min(16, e.N - n) : 0;
            rz.load(e.z, m * e.ld_zu + n, left, wide_user);
            ru.load(e.u, m * e.ld_zu + n, left, wide_user);
          };
          auto store = [&](void* to, int64_t at_h, float* v, int room) {
            if (!to || room <= 0) return;
            if constexpr (F32) store16_limbs(to, at_h, e.limb, v, room, wide_own);
            else store16<false>(to, at_h, v, room, wide_own);
          };
          fetch(0);
#pragma unroll 1
          for (int c = 0; c < kOut; ++c) {
            const int n = n0 + 16 * c, room = row ? (int)min((int64_t)16, e.ld_h - n) : 0;
            const int64_t at_h = m * e.ld_h + n;
            float dh[16], a[16], da[16], bv[16], db[16];
            slope16<!F32>(e.act, rz, a, da);
            slope16<!F32>(e.act_up, ru, bv, db);
            if (c + 1 < kOut) fetch(c + 1);
            sums(c, dh);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              db[i] *= dh[i] * a[i];   // du
              da[i] *= dh[i] * bv[i];  // dz
              a[i] *= bv[i];           // h
            }
            store(e.h, at_h, a, room);
            store(e.du, at_h, db, room);
            float sum = 0.f;
            if (e.db) {
#pragma unroll
              for (int i = 0; i < 16; ++i) dh[i] = da[i];
              sum = column_sum(dh, lane);
            }
            store(e.dz, at_h, da, room);
            if (e.db) {
              const int line = at.m * (kRows / 32) + rank * 4 + quad, n_of = n + (lane >> 1);
              if (!(lane & 1) && n_of < e.N && line * 32 < e.M) e.db[line * e.ld_h + n_of] = sum;
            }
          }
        }
      }
      fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(empty0 + 8 * b);
      b ^= 1;
      if (b == 0) b_phase ^= 1;
    }
  }

  // Everybody meets, then the allocating warps free tensor memory.  (After a wait that ran out, copies and MMAs may still be in
  // flight: they end within microseconds, and shared memory and tensor memory are only given back after that.)
  if (*abort_flag)
    for (int i = 0; i < 50; ++i) __nanosleep(1000);
  fence_before();
  cluster_sync();
  if (warp == 2) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn() {
  static EncodeTiledFn fn = [] {
    cudaDriverEntryPointQueryResult q;
    void* ptr = nullptr;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) ptr = nullptr;
    return reinterpret_cast<EncodeTiledFn>(ptr);
  }();
  return fn;
}

// `terms` bf16 matrices [rows, width], rows `ld` elements apart, in boxes of 64 elements x `box` rows, 128-byte swizzle.
bool make_map(CUtensorMap* m, const void* base, int64_t width, int64_t rows, int64_t ld, int terms, int64_t limb, int box) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)width, (cuuint64_t)rows, (cuuint64_t)terms};
  const cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)(terms > 1 ? limb : ld * rows) * 2};
  const cuuint32_t boxes[3] = {(cuuint32_t)kDeep, (cuuint32_t)box, 1};
  const cuuint32_t steps[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The terms of fp32 values: eight a thread.
__global__ void __launch_bounds__(256) train_split_kernel(const float* in, int64_t ld_in, int rows, int cols, __nv_bfloat16* out, int64_t ld_out, int64_t limb) {
  pdl_launch_dependents();
  pdl_wait();
  const int per = (cols + 7) / 8;
  const int64_t total = (int64_t)rows * per;
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < total; i += gridDim.x * 256ll) {
    const int64_t r = i / per;
    const int c = (int)(i - r * per) * 8;
    const float* p = in + r * ld_in + c;
    float v[8];
    const int n = min(8, cols - c);
#pragma unroll
    for (int q = 0; q < 2; ++q) {  // columns are a multiple of four
      const float4 f = 4 * q < n ? *reinterpret_cast<const float4*>(p + 4 * q) : make_float4(0, 0, 0, 0);
      v[4 * q] = f.x; v[4 * q + 1] = f.y; v[4 * q + 2] = f.z; v[4 * q + 3] = f.w;
    }
#pragma unroll
    for (int l = 0; l < 3; ++l) {
      uint32_t w[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) w[q] = pack_bf16(v[2 * q], v[2 * q + 1]);
      *reinterpret_cast<uint4*>(out + l * limb + r * ld_out + c) = make_uint4(w[0], w[1], w[2], w[3]);
#pragma unroll
      for (int q = 0; q < 8; ++q) v[q] -= __bfloat162float(__float2bfloat16(v[q]));
    }
  }
}

template <int EPI, bool F32, bool PROMOTE>
cudaError_t launch_one(const UmmaParams& p, const Maps& maps, int pairs, cudaStream_t s) {
  static unsigned long long configured = 0;
  const cudaError_t e = allow_dynamic_smem(train_umma_kernel<EPI, F32, PROMOTE>, kSmemBytes, configured);
  if (e != cudaSuccess) return e;
  return launch_clusters(2, train_umma_kernel<EPI, F32, PROMOTE>, dim3(2 * pairs), dim3(kThreads), kSmemBytes, s, p, maps);
}

}  // namespace

int train_umma_lines(int M) { return (M + 31) / 32; }

cudaError_t launch_train_split(const float* in, int64_t ld_in, int rows, int cols, __nv_bfloat16* out, int64_t ld_out, int64_t limb, cudaStream_t s) {
  const int64_t total = (int64_t)rows * ((cols + 7) / 8);
  const int64_t want = (total + 255) / 256;
  return launch_pdl(train_split_kernel, dim3((unsigned)(want < 148 * 8 ? want : 148 * 8)), dim3(256), 0, s, in, ld_in, rows, cols, out, ld_out, limb);
}

cudaError_t launch_train_umma(const TrainUmma& t, cudaStream_t s) {
  const TrainGemm& g = t.g;
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return e;
  const int most = sms / 2 < kTrainUmmaPairs ? sms / 2 : kTrainUmmaPairs;
  UmmaParams p{};
  p.epi = g.epi;
  p.epilogue = g.epilogue;
  p.f32 = t.f32;
  p.tile_cols = g.epilogue == kEpiGateUp ? kCols / 2 : kCols;
  p.m_tiles = (g.M + kRows - 1) / kRows;
  p.n_tiles = (g.N + p.tile_cols - 1) / p.tile_cols;
  p.batch = g.batch;
  const long long tiles = (long long)p.m_tiles * p.n_tiles * g.batch;
  if (tiles > (1 << 30)) return cudaErrorInvalidValue;
  p.tiles = (int)tiles;
  p.blocks = (g.K + kDeep - 1) / kDeep;
  if (t.f32) p.blocks = (p.blocks + kLimbBlocks - 1) / kLimbBlocks * kLimbBlocks;
  const int parts = g.epilogue == kEpiGateUp ? 1 : g.parts;
  p.unit_blocks = t.f32 ? kLimbUnit : 1;
  p.units = parts * p.blocks / (t.f32 ? kLimbBlocks : 1);
  p.run_units = t.f32 ? 1 : kRunBlocks;
  p.a_mn = !g.a_major_k;
  p.b_mn = !g.b_major_k;
  p.partial = t.partial;
  p.counters = t.counters;
  p.status = t.status;
  p.budget = fused_test_knobs().wait_cycles;
  // Whole rounds of tiles, then the rest cut along K, unless a pair's share of it is so small that pieces cost more than they save.
  int pairs = most;
  p.whole = p.tiles / pairs * pairs;
  const int rest = p.tiles - p.whole;
  if (!t.partial || rest == 0 || (long long)rest * p.units < pairs || (long long)rest * p.units * p.unit_blocks < 16ll * pairs) {
    p.whole = p.tiles;
    if (p.tiles < pairs) pairs = p.tiles;
  }
  Maps maps;
  const int na = g.epilogue == kEpiGateUp ? 1 : g.batch > 1 ? g.batch : g.parts, nb = g.batch > 1 ? g.batch : g.parts;
  const int terms = t.f32 ? 3 : 1;
  for (int i = 0; i < 3; ++i) {
    const int ia = i < na ? i : 0, ib = i < nb ? i : 0;
    const bool fine = (g.a_major_k ? make_map(&maps.a[i], g.a[ia].data, g.K, g.M, g.a[ia].ld, terms, t.limb_a[ia], 128)
                                   : make_map(&maps.a[i], g.a[ia].data, g.M, g.K, g.a[ia].ld, terms, t.limb_a[ia], 64)) &&
                      (g.b_major_k ? make_map(&maps.b[i], g.b[ib].data, g.K, g.N, g.b[ib].ld, terms, t.limb_b[ib], 128)
                                   : make_map(&maps.b[i], g.b[ib].data, g.N, g.K, g.b[ib].ld, terms, t.limb_b[ib], 64));
    if (!fine) return cudaErrorInvalidValue;
  }
  if (t.f32) {
    if (g.epilogue == kEpiStore) return launch_one<kEpiStore, true, true>(p, maps, pairs, s);
    if (g.epilogue == kEpiGateUp) return launch_one<kEpiGateUp, true, true>(p, maps, pairs, s);
    return launch_one<kEpiHidden, true, true>(p, maps, pairs, s);
  }
  if (g.epilogue == kEpiStore) return launch_one<kEpiStore, false, false>(p, maps, pairs, s);
  if (g.epilogue == kEpiGateUp) return launch_one<kEpiGateUp, false, false>(p, maps, pairs, s);
  return launch_one<kEpiHidden, false, true>(p, maps, pairs, s);
}

}  // namespace sffn

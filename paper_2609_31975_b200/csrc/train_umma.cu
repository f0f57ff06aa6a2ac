// Products of the training calls in bf16 on the 5th-generation tensor cores (tcgen05.mma, accumulators in tensor memory).
//
// A pair of CTAs (cta_group::2) owns 256 rows of C = A B^T: each holds 128 rows of A and half of B's rows of a 64-deep K block
// in each of four stages (z and u, and dh, of up to 64 tokens: the rows of A that there are, in up to six).  Both operands may lie K-major or MN-major in memory (the tensor core takes either from the
// 128-byte-swizzled boxes that the tensor-map copies leave), so none of the six products of a training step needs a transposed copy.
//
//   kStore   512 columns: two accumulators of 256 fill tensor memory, and share A.  The copies into shared memory run at 10 TB/s at
//            most, from L2, and bound products in tiles of 256 columns; these move a quarter less for the same result.  The next
//            tile's products wait for the epilogue of a half, a twentieth of the tile's time at K = 4096.
//   kGateUp  z and u of 128 neurons, 256 columns: the even CTA's half of B is W_g, the odd one's W_up, so that z and u of a neuron are
//            in the same lane of tensor memory, 128 columns apart.  Two accumulators: one tile's epilogue runs under the next tile.
//   kHidden  dh of 256 neurons.  Its dz is summed over the tokens in fp32 (db_g), and the tensor cores truncate when they add onto an
//            accumulator: the sum comes out low by 5e-8 of its typical size for every 64 of K (3e-6 at K = 4096).  So runs of 768 k
//            get an accumulator of their own, eight warps add the runs up in registers, rounding to nearest (7e-7), and
//            put them into the other half of tensor memory, where four more warps make dz, du and h of them under the next tile.
//
// Epilogues leave through shared memory: boxes of 32 rows x 64 columns, 128-byte swizzle, which tensor-map stores take to the
// caller's rows, whatever their stride and alignment, cut off at the matrix's edges.
//
// Tiles are dealt to the pairs round robin.  What is left for a last, partly idle round is cut along K where that is shorter: a pair
// leaves its piece of a tile as fp32 in a workspace, and train_join_kernel adds up the pieces in their order in K and does the epilogue.
// Every wait is bounded by a cycle budget; on expiry the status word is set, all roles wind down and tensor memory is given back.
#include <cmath>

#include "fused_kernel.cuh"
#include "train_umma.cuh"

namespace sffn {
namespace {

using namespace tc;

constexpr int kStages = 4;           // of whole K blocks; the ring holds up to kMostStages of fewer rows of A
constexpr int kMostStages = 6, kFewRows = 64;
constexpr int kBoxBytes = 32 * 128;  // 32 rows x 64 bf16 columns
constexpr int kAdders = 8;           // warps 4-11

template <int EPI>
struct Form {
  static constexpr int kWide = EPI == kEpiStore ? 2 : 1;                       // accumulators of a tile
  static constexpr int kTileCols = EPI == kEpiGateUp ? 128 : 256 * kWide;      // output columns
  static constexpr int kStageBytes = (1 + kWide) * kHalfBytes;
  static constexpr int kThreads = EPI == kEpiHidden ? 512 : 384;
  static constexpr int kOutWarps = EPI == kEpiHidden ? 4 : 8;                  // that store boxes
  static constexpr int kBoxes = EPI == kEpiStore ? 1 : EPI == kEpiGateUp ? 3 : 5;  // of such a warp (kHidden: z and u too)
  static constexpr int kSmemBytes = kStages * kStageBytes + kOutWarps * kBoxes * kBoxBytes + 1024;
};
static_assert(Form<kEpiStore>::kSmemBytes <= 231 * 1024 && Form<kEpiGateUp>::kSmemBytes <= 231 * 1024 && Form<kEpiHidden>::kSmemBytes <= 231 * 1024, "shared memory");

struct Maps {
  CUtensorMap a[3], b[3];
  CUtensorMap out[3];  // kStore: of each product of a batch; kGateUp: z, u, h; kHidden: dz, du, h
  CUtensorMap in[2];   // kHidden: z, u
};

// Sixteen values of row `lane` into columns 16 q .. of a box.
__device__ __forceinline__ void box_put(uint32_t box, int lane, int q, const float* v) {
  const uint32_t row = box + lane * 128;
#pragma unroll
  for (int i = 0; i < 2; ++i)
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(row + (((2 * q + i) ^ (lane & 7)) << 4)), "r"(pack_bf16(v[8 * i], v[8 * i + 1])),
                 "r"(pack_bf16(v[8 * i + 2], v[8 * i + 3])), "r"(pack_bf16(v[8 * i + 4], v[8 * i + 5])), "r"(pack_bf16(v[8 * i + 6], v[8 * i + 7]))
                 : "memory");
}
struct Sixteen {
  uint32_t w[8];
  __device__ __forceinline__ void get_from(uint32_t box, int lane, int q) {
    const uint32_t row = box + lane * 128;
#pragma unroll
    for (int i = 0; i < 2; ++i)
      asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];"
                   : "=r"(w[4 * i]), "=r"(w[4 * i + 1]), "=r"(w[4 * i + 2]), "=r"(w[4 * i + 3])
                   : "r"(row + (((2 * q + i) ^ (lane & 7)) << 4))
                   : "memory");
  }
  __device__ __forceinline__ float get(int i) const { return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16); }
};
// Before a box is written again: its store has read it.  After it is written: one lane stores it.
__device__ __forceinline__ void boxes_free(int lane) {
  if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
  __syncwarp();
}
__device__ __forceinline__ void boxes_written() {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  __syncwarp();
}
// kStore: half boxes of 32 columns, 64-byte swizzle, two a warp: one is filled while the other's store reads it.
__device__ __forceinline__ void half_box_put(uint32_t box, int lane, int q, const float* v) {
  const uint32_t row = box + lane * 64;
#pragma unroll
  for (int i = 0; i < 2; ++i)
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(row + (((2 * q + i) ^ ((lane >> 1) & 3)) << 4)), "r"(pack_bf16(v[8 * i], v[8 * i + 1])),
                 "r"(pack_bf16(v[8 * i + 2], v[8 * i + 3])), "r"(pack_bf16(v[8 * i + 4], v[8 * i + 5])), "r"(pack_bf16(v[8 * i + 6], v[8 * i + 7]))
                 : "memory");
}
__device__ __forceinline__ void other_box_free(int lane) {
  if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
  __syncwarp();
}
__device__ __forceinline__ void box_store(const CUtensorMap* map, uint32_t box, int c0, int c1) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(c0), "r"(c1), "r"(box) : "memory");
}
__device__ __forceinline__ void boxes_leave() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void boxes_gone() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void box_load(uint32_t box, const CUtensorMap* map, int c0, int c1, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(box), "l"(map), "r"(c0),
               "r"(c1), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

template <int EPI>
__global__ void __launch_bounds__(Form<EPI>::kThreads, 1) train_umma_kernel(const __grid_constant__ UmmaParams p, const __grid_constant__ Maps maps) {
  using F = Form<EPI>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ int abort_word;
  __shared__ uint32_t tmem_slot;
  __shared__ __align__(8) uint64_t bars[2 * kMostStages + 4 + 2 + 4];
  volatile int* const abort_flag = &abort_word;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u, boxes = ring + kStages * F::kStageBytes;
  const uint32_t full = smem_u32(bars), empty = full + 8 * kMostStages, acc_full = empty + 8 * kMostStages, acc_empty = acc_full + 16;
  const uint32_t sums_full = acc_empty + 16, sums_empty = sums_full + 8, in_full = sums_empty + 8;  // kHidden
  const int rank = (int)cluster_rank(), pair = (int)blockIdx.x >> 1, pairs = (int)gridDim.x >> 1;

  if (tid == 0) {
    for (int s = 0; s < kMostStages; ++s) {
      mbar_init(full + 8 * s, 1);
      mbar_init(empty + 8 * s, 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(acc_full + 8 * b, 1);
      mbar_init(acc_empty + 8 * b, 2 * kAdders);
    }
    mbar_init(sums_full, kAdders);
    mbar_init(sums_empty, 4);
    for (int w = 0; w < 4; ++w) mbar_init(in_full + 8 * w, 1);
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

  const TrainEpilogue& e = p.epi;
  Walk walk(p, pairs, pair);
  Item it;
  // kStore: the accumulators of a tile that have columns
  auto halves_of = [&](const Place& at) { return F::kWide == 2 && at.n * F::kTileCols + 256 < e.N ? 2 : 1; };

  if (warp < 4) {
    if constexpr (EPI == kEpiHidden) asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    auto wait_all = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, p.status, p.budget)) != 0; };
    if (warp == 0) {
      const uint32_t a_bytes = p.a_rows * kDeep * 2;
      int s = 0, phase = 0, left_out = blockIdx.x == 0 ? p.drop : -1;
      bool ok = true;
      while (ok && walk.step(p, it)) {
        const Place at = place_of(p, it.tile);
        const int m0 = at.m * kPairRows + rank * 128, halves = halves_of(at);
        const int n0 = at.n * F::kTileCols + (EPI == kEpiGateUp ? 0 : rank * 128);
        for (int u = it.u0; u < it.u1; ++u) {
          ok = wait_all(empty + 8 * s, phase ^ 1);
          if (!ok) break;
          if (elect_one()) {
            const int part = u >= p.blocks ? 1 : 0, k0 = (u - part * p.blocks) * kDeep, which = p.batch > 1 ? at.batch : part;
            const CUtensorMap* ma = &maps.a[EPI == kEpiGateUp ? 0 : which];
            const CUtensorMap* mb = &maps.b[EPI == kEpiGateUp ? rank : which];
            const uint32_t bar = map_rank(full + 8 * s, 0), da = ring + s * p.stage_bytes;
            if (rank == 0) mbar_expect_tx(full + 8 * s, 2 * halves * kHalfBytes + (a_bytes < kHalfBytes ? 1 : 2) * a_bytes);
            if (left_out-- == 0 || (rank == 1 && a_bytes < kHalfBytes)) {
            } else if (p.a_mn) {
              tma_tile_3d(da, ma, m0, k0, 0, bar);
              tma_tile_3d(da + kHalfBytes / 2, ma, m0 + 64, k0, 0, bar);
            } else {
              tma_tile_3d(da, ma, k0, m0, 0, bar);
            }
            for (int h = 0; h < halves; ++h) {
              const uint32_t db = da + a_bytes + h * kHalfBytes;
              const int n = n0 + 256 * h;
              if (p.b_mn) {
                tma_tile_3d(db, mb, n, k0, 0, bar);
                tma_tile_3d(db + kHalfBytes / 2, mb, n + 64, k0, 0, bar);
              } else {
                tma_tile_3d(db, mb, k0, n, 0, bar);
              }
            }
          }
          __syncwarp();
          if (++s == p.stages) { s = 0; phase ^= 1; }
        }
      }
    } else if (warp == 1 && rank == 0) {
      const uint32_t idesc = idesc_bf16(kPairRows, 256, p.a_mn, p.b_mn);
      const uint64_t a0 = p.a_mn ? desc_mn_major(ring, kHalfBytes / 2) : desc_k_major(ring);
      const uint32_t ring_b = ring + p.a_rows * kDeep * 2;
      const uint64_t b0 = p.b_mn ? desc_mn_major(ring_b, kHalfBytes / 2) : desc_k_major(ring_b);
      const uint32_t a_step = p.a_mn ? 2048 >> 4 : 32 >> 4, b_step = p.b_mn ? 2048 >> 4 : 32 >> 4;  // sixteen k
      int s = 0, phase = 0, b = 0, acc_phase[2] = {1, 1};
      // the MMAs of a K block into one accumulator
      auto multiply = [&](int buffer, int h, uint32_t more) {
        const uint32_t off = (uint32_t)(s * p.stage_bytes) >> 4;
#pragma unroll
        for (int k = 0; k < kDeep / 16; ++k)
          umma_pair(tmem + buffer * 256, a0 + off + k * a_step, b0 + off + h * (kHalfBytes >> 4) + k * b_step, idesc, k > 0 ? 1u : more);
      };
      bool ok = true;
      while (ok && walk.step(p, it)) {
        const int halves = halves_of(place_of(p, it.tile));
        for (int u = it.u0; ok && u < it.u1;) {
          const int end = EPI == kEpiHidden ? min(it.u1, u + p.run_units) : it.u1;
          // the first block waits for the accumulators, half by half; where it is the only one, a half is handed over at once
          ok = wait_all(full + 8 * s, phase);
          if (!ok) break;
          for (int h = 0; h < halves; ++h) {
            const int buffer = F::kWide == 2 ? h : b;
            ok = wait_all(acc_empty + 8 * buffer, buffer ? acc_phase[1] : acc_phase[0]);
            if (!ok) break;
            if (buffer) acc_phase[1] ^= 1;
            else acc_phase[0] ^= 1;
            fence_after();
            if (elect_one()) {
              multiply(buffer, h, 0);
              if (end - u == 1) commit_pair(acc_full + 8 * buffer);
              if (h == halves - 1) commit_pair(empty + 8 * s);
            }
            __syncwarp();
          }
          if (!ok) break;
          if (++s == p.stages) { s = 0; phase ^= 1; }
          for (int n = u + 1; n < end; ++n) {
            ok = wait_all(full + 8 * s, phase);
            if (!ok) break;
            fence_after();
            if (elect_one()) {
              multiply(F::kWide == 2 ? 0 : b, 0, 1);
              if (F::kWide == 2 && halves == 2) multiply(1, 1, 1);
              commit_pair(empty + 8 * s);
              if (n == end - 1) {
                commit_pair(acc_full + 8 * (F::kWide == 2 ? 0 : b));
                if (F::kWide == 2 && halves == 2) commit_pair(acc_full + 8);
              }
            }
            __syncwarp();
            if (++s == p.stages) { s = 0; phase ^= 1; }
          }
          if (!ok) break;
          if (EPI == kEpiGateUp) b ^= 1;
          u = end;
        }
      }
    }
  } else if (warp < 12) {
    if constexpr (EPI == kEpiHidden) asm volatile("setmaxnreg.inc.sync.aligned.u32 160;");
    const int quad = warp & 3, half = (warp - 4) >> 2;
    const uint32_t lanes = (uint32_t)(32 * quad) << 16;
    constexpr int kChunks = 8;  // of sixteen columns, of a warp and accumulator
    // column (in the accumulator) of a chunk: kGateUp: a warp has z and u of 64 neurons, z's chunks first
    auto column = [&](int c) { return EPI == kEpiGateUp ? (c < 4 ? 0 : 128) + 64 * half + 16 * (c & 3) : 128 * half + 16 * c; };
    const uint32_t empty0 = map_rank(acc_empty, 0), box = boxes + (warp - 4) * F::kBoxes * kBoxBytes;
    int b = 0, full_phase[2] = {0, 0}, sums_phase = 1;
    bool ok = true;
    auto wait_full = [&](int buffer) {
      const bool there = __all_sync(0xffffffffu, mbar_wait(acc_full + 8 * buffer, buffer ? full_phase[1] : full_phase[0], abort_flag, p.status, p.budget));
      if (buffer) full_phase[1] ^= 1;
      else full_phase[0] ^= 1;
      fence_after();
      return there;
    };
    auto give_back = [&](int buffer) {
      fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(empty0 + 8 * buffer);
    };
    while (ok && walk.step(p, it)) {
      const Place at = place_of(p, it.tile);
      const int row0 = at.m * kPairRows + rank * 128 + 32 * quad;  // this warp's first row
      const bool rows = row0 < e.M;                                // has any: the others only keep step
      const bool cut = it.piece >= 0;
      float* const piece = cut ? piece_of(p, it.piece) + (size_t)(rank * 128 + 32 * quad + lane) * (256 * F::kWide) : nullptr;  // this lane's row
      if constexpr (EPI == kEpiHidden) {
        float acc[16 * kChunks];
#pragma unroll
        for (int i = 0; i < 16 * kChunks; ++i) acc[i] = 0.f;
#pragma unroll 1
        for (int u = it.u0; u < it.u1; u = min(it.u1, u + p.run_units)) {
          ok = wait_full(0);
          if (!ok) break;
          if (rows) {
#pragma unroll
            for (int c = 0; c < kChunks; ++c) {
              float v[16];
              tmem_ld16(tmem + lanes + column(c), v);
              tmem_arrived(v);
#pragma unroll
              for (int i = 0; i < 16; ++i) acc[16 * c + i] += v[i];
            }
          }
          give_back(0);
        }
        if (!ok) break;
        if (cut) {
#pragma unroll
          for (int c = 0; c < kChunks; ++c)
            if (rows) put_piece(piece + column(c), acc + 16 * c);
          continue;
        }
        ok = __all_sync(0xffffffffu, mbar_wait(sums_empty, sums_phase, abort_flag, p.status, p.budget));
        if (!ok) break;
        sums_phase ^= 1;
        if (rows) {
          fence_after();
#pragma unroll
          for (int c = 0; c < kChunks; ++c) tmem_st16(tmem + 256 + lanes + column(c), acc + 16 * c);
          tmem_stored();
          fence_before();
        }
        __syncwarp();
        if (lane == 0) arrive(sums_full);
      } else {
        const int halves = halves_of(at);
        for (int h = 0; h < halves; ++h) {
          const int buffer = F::kWide == 2 ? h : b;
          ok = wait_full(buffer);
          if (!ok) break;
          const uint32_t acc = tmem + lanes + buffer * 256;
          auto sums = [&](int c, float* v) {
            tmem_ld16(acc + column(c), v);
            tmem_arrived(v);
          };
          if (cut && rows) {
#pragma unroll 2
            for (int c = 0; c < kChunks; ++c) {
              float v[16];
              sums(c, v);
              put_piece(piece + 256 * h + column(c), v);
            }
          }
          if (rows && !cut) {
            if constexpr (EPI == kEpiStore) {
              const int n0 = at.n * F::kTileCols + 256 * h + 128 * half;
#pragma unroll 1
              for (int x = 0; x < 4; ++x) {
                const uint32_t to = box + (x & 1) * (kBoxBytes / 2);
                other_box_free(lane);
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                  float v[16];
                  sums(2 * x + q, v);
                  half_box_put(to, lane, q, v);
                }
                boxes_written();
                if (lane == 0) {
                  if (n0 + 32 * x < e.N) box_store(&maps.out[at.batch], to, n0 + 32 * x, row0);
                  boxes_leave();  // a group for each half box, so that all but the last one means the other one
                }
              }
            } else {
              const int n0 = at.n * F::kTileCols + 64 * half;
              boxes_free(lane);
#pragma unroll 1
              for (int q = 0; q < 4; ++q) {
                const int n = n0 + 16 * q;
                float z[16], u[16];
                sums(q, z);
                sums(q + 4, u);
                if (e.bias) {
                  const float bias = lane < 16 && n + lane < e.N ? e.bias[n + lane] : 0.f;
#pragma unroll
                  for (int i = 0; i < 16; ++i) z[i] += __shfl_sync(0xffffffffu, bias, i);
                }
                if (e.z) {
                  box_put(box, lane, q, z);
                  box_put(box + kBoxBytes, lane, q, u);
                }
                act16<true>(e.act, z, z);
                act16<true>(e.act_up, u, u);
#pragma unroll
                for (int i = 0; i < 16; ++i) z[i] *= u[i];
                box_put(box + 2 * kBoxBytes, lane, q, z);
              }
              boxes_written();
              // A tensor-map store cuts a row off at a multiple of 16 bytes: the last columns of an odd number go by themselves.
              const int even = e.N & ~7;
              if (e.z && even != e.N && n0 <= even && even < n0 + 64 && row0 + lane < e.M) {
                const uint32_t from = box + lane * 128 + ((((even - n0) >> 3) ^ (lane & 7)) << 4);
                const int64_t to = (int64_t)(row0 + lane) * e.ld_zu + even;
                for (int i = 0; i < e.N - even; ++i) {
                  uint16_t zv, uv;
                  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(zv) : "r"(from + 2 * i) : "memory");
                  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(uv) : "r"(from + kBoxBytes + 2 * i) : "memory");
                  static_cast<uint16_t*>(e.z)[to + i] = zv;
                  static_cast<uint16_t*>(e.u)[to + i] = uv;
                }
              }
              if (lane == 0 && n0 < e.N) {
                if (e.z && n0 < even) {
                  box_store(&maps.out[0], box, n0, row0);
                  box_store(&maps.out[1], box + kBoxBytes, n0, row0);
                }
                box_store(&maps.out[2], box + 2 * kBoxBytes, n0, row0);
                boxes_leave();
              }
            }
          }
          give_back(buffer);
        }
        if (EPI == kEpiGateUp) b ^= 1;
      }
    }
    if (EPI != kEpiHidden && lane == 0) boxes_gone();
  } else if constexpr (EPI == kEpiHidden) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 136;");
    const int quad = warp & 3;
    const uint32_t lanes = (uint32_t)(32 * quad) << 16;
    const uint32_t box = boxes + quad * F::kBoxes * kBoxBytes, zbox = box + 3 * kBoxBytes, ubox = box + 4 * kBoxBytes, bar = in_full + 8 * quad;
    int sums_phase = 0, in_phase = 0;
    bool ok = true;
    while (ok && walk.step(p, it)) {
      if (it.piece >= 0) continue;
      const Place at = place_of(p, it.tile);
      const int row0 = at.m * kPairRows + rank * 128 + 32 * quad;
      const bool rows = row0 < e.M;
      // z and u of a box come while the one before is being worked on, a tile's first while its sums are
      auto fetch = [&](int x) {
        if (lane != 0 || !rows) return;
        mbar_expect_tx(bar, 2 * kBoxBytes);
        box_load(zbox, &maps.in[0], at.n * 256 + 64 * x, row0, bar);
        box_load(ubox, &maps.in[1], at.n * 256 + 64 * x, row0, bar);
      };
      const int n_boxes = min(4, (e.N - at.n * 256 + 63) / 64);
      fetch(0);
      ok = __all_sync(0xffffffffu, mbar_wait(sums_full, sums_phase, abort_flag, p.status, p.budget));
      if (!ok) break;
      sums_phase ^= 1;
      fence_after();
      for (int x = 0; rows && x < n_boxes; ++x) {
        ok = __all_sync(0xffffffffu, mbar_wait(bar, in_phase, abort_flag, p.status, p.budget));
        if (!ok) break;
        in_phase ^= 1;
        const int n0 = at.n * 256 + 64 * x;
        boxes_free(lane);
#pragma unroll 1
        for (int q = 0; q < 4; ++q) {
          float dh[16], a[16], da[16], bv[16], db[16];
          tmem_ld16(tmem + 256 + lanes + 64 * x + 16 * q, dh);
          Sixteen t;
          t.get_from(zbox, lane, q);
          slope16<true>(e.act, t, a, da);
          t.get_from(ubox, lane, q);
          slope16<true>(e.act_up, t, bv, db);
          tmem_arrived(dh);
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            db[i] *= dh[i] * a[i];   // du
            da[i] *= dh[i] * bv[i];  // dz
            a[i] *= bv[i];           // h
          }
          if (e.dz) box_put(box, lane, q, da);
          if (e.du) box_put(box + kBoxBytes, lane, q, db);
          if (e.h) box_put(box + 2 * kBoxBytes, lane, q, a);
          if (e.db) {
            const float sum = column_sum(da, lane);
            const int n = n0 + 16 * q + (lane >> 1);
            if (!(lane & 1) && n < e.N) e.db[(int64_t)(row0 >> 5) * e.ld_h + n] = sum;
          }
        }
        boxes_written();
        if (x + 1 < n_boxes) fetch(x + 1);
        if (lane == 0) {
          if (e.dz) box_store(&maps.out[0], box, n0, row0);
          if (e.du) box_store(&maps.out[1], box + kBoxBytes, n0, row0);
          if (e.h) box_store(&maps.out[2], box + 2 * kBoxBytes, n0, row0);
          boxes_leave();
        }
      }
      if (!ok) break;
      fence_before();
      __syncwarp();
      if (lane == 0) arrive(sums_empty);
    }
    if (lane == 0) boxes_gone();
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

// A bf16 matrix [rows, width] in boxes of 64 (32) columns x 32 rows, 128- (64-) byte swizzle.
bool make_box_map(CUtensorMap* m, const void* base, int64_t width, int64_t rows, int64_t ld, bool half = false) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)width, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)ld * 2};
  const cuuint32_t box[2] = {half ? 32u : 64u, 32};
  const cuuint32_t steps[2] = {1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
            half ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int EPI>
cudaError_t launch_one(const TrainUmma& t, int pairs, cudaStream_t s) {
  using F = Form<EPI>;
  const TrainGemm& g = t.g;
  UmmaParams p{};
  pairs = plan_umma(t, F::kTileCols, p, pairs);
  static_assert(piece_cols(EPI, false) == 256 * F::kWide);
  // Few tokens: a CTA copies those rows of A in steps of 32 (what the epilogue's warps look at), and the ring holds more K blocks.  The
  // MMAs read 128 rows all the same: what lies behind, the same stage's rows of B, goes into rows of the accumulator that nobody reads.
  // bf16, without / with it: 1 and 5 tokens, 4096 x 14336, forward 107 / 92, 96 / 89 us, dh 58 / 43, 53 / 44; 16 tokens, 2048 x 8192,
  // forward 41 / 37; 60 tokens, 4096 x 14336, dh 49 / 46.  Plain products lose (8 tokens, 8192 x 20000, dx 118 / 141).
  p.a_rows = EPI != kEpiStore && g.a_major_k && g.M <= kFewRows ? (g.M + 31) & ~31 : 128;
  p.stage_bytes = F::kStageBytes - kHalfBytes + p.a_rows * kDeep * 2;
  p.stages = kStages * F::kStageBytes / p.stage_bytes;
  static_assert(kStages * F::kStageBytes / (F::kStageBytes - kHalfBytes + 32 * kDeep * 2) <= kMostStages);
  Maps maps;
  bool fine = pairs > 0 && make_operand_maps(t, p.a_rows, maps.a, maps.b);
  const TrainEpilogue& e = g.epi;
  void* const out[3] = {EPI == kEpiStore ? e.out[0] : EPI == kEpiGateUp ? e.z : e.dz, EPI == kEpiStore ? e.out[1] : EPI == kEpiGateUp ? e.u : e.du,
                        EPI == kEpiStore ? e.out[2] : e.h};
  for (int i = 0; i < 3; ++i)
    if (out[i]) fine = fine && make_box_map(&maps.out[i], out[i], EPI == kEpiGateUp && i < 2 ? g.N < 8 ? 8 : g.N & ~7 : g.N, g.M, EPI == kEpiStore ? e.ld_out : EPI == kEpiGateUp && i < 2 ? e.ld_zu : e.ld_h, EPI == kEpiStore);
  if (EPI == kEpiHidden) fine = fine && make_box_map(&maps.in[0], e.z, g.N, g.M, e.ld_zu) && make_box_map(&maps.in[1], e.u, g.N, g.M, e.ld_zu);
  if (!fine) return cudaErrorInvalidValue;
  static unsigned long long configured = 0;
  const cudaError_t err = allow_dynamic_smem(train_umma_kernel<EPI>, F::kSmemBytes, configured);
  if (err != cudaSuccess) return err;
  const cudaError_t launched = launch_clusters(2, train_umma_kernel<EPI>, dim3(2 * pairs), dim3(F::kThreads), F::kSmemBytes, s, p, maps);
  if (launched != cudaSuccess || p.whole == p.tiles) return launched;
  return launch_train_join(p, EPI, false, s);
}

}  // namespace

bool make_train_map(CUtensorMap* m, const void* base, int64_t width, int64_t rows, int64_t ld, int terms, int64_t limb, int box) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)width, (cuuint64_t)rows, (cuuint64_t)terms};
  const cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)(terms > 1 ? limb : ld * rows) * 2};
  const cuuint32_t boxes[3] = {(cuuint32_t)kDeep, (cuuint32_t)box, 1};
  const cuuint32_t steps[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool make_operand_maps(const TrainUmma& t, int a_rows, CUtensorMap* a, CUtensorMap* b) {
  const TrainGemm& g = t.g;
  const int na = g.epilogue == kEpiGateUp ? 1 : g.batch > 1 ? g.batch : g.parts, nb = g.batch > 1 ? g.batch : g.parts;
  const int terms = t.f32 ? 3 : 1;
  for (int i = 0; i < 3; ++i) {  // the first one again where there are fewer
    if (i >= na) a[i] = a[0];
    else if (!(g.a_major_k ? make_train_map(&a[i], g.a[i].data, g.K, g.M, g.a[i].ld, terms, t.limb_a[i], a_rows)
                           : make_train_map(&a[i], g.a[i].data, g.M, g.K, g.a[i].ld, terms, t.limb_a[i], 64))) return false;
    if (i >= nb) b[i] = b[0];
    else if (!(g.b_major_k ? make_train_map(&b[i], g.b[i].data, g.K, g.N, g.b[i].ld, terms, t.limb_b[i], 128)
                           : make_train_map(&b[i], g.b[i].data, g.N, g.K, g.b[i].ld, terms, t.limb_b[i], 64))) return false;
  }
  return true;
}

int plan_umma(const TrainUmma& t, int cols, UmmaParams& p, int pairs) {
  const TrainGemm& g = t.g;
  p.epi = g.epi;
  p.tile_cols = cols;
  p.m_tiles = (g.M + kPairRows - 1) / kPairRows;
  p.n_tiles = (g.N + cols - 1) / cols;
  p.batch = g.batch;
  const long long tiles = (long long)p.m_tiles * p.n_tiles * g.batch;
  if (tiles > (1 << 30)) return 0;
  p.tiles = (int)tiles;
  p.blocks = (g.K + kDeep - 1) / kDeep;
  p.units = (g.epilogue == kEpiGateUp ? 1 : g.parts) * p.blocks;
  p.run_units = t.f32 ? kLimbRun : g.epi.db ? kRunBlocks : p.units;  // (bf16: what is not summed in fp32 needs no runs)
  p.a_mn = !g.a_major_k;
  p.b_mn = !g.b_major_k;
  p.partial = t.partial;
  p.piece = (size_t)piece_rows(g.M) * piece_cols(g.epilogue, t.f32);
  p.status = t.status;
  p.budget = fused_test_knobs().wait_cycles;
  p.drop = fused_test_knobs().drop_stage;
  // Whole rounds of tiles, then the rest: whole too, or cut along K into `split` equal pieces a tile, dealt in rounds of their own.  What
  // is shortest, counted in K blocks of a product (half a microsecond): a piece's rows are written to the workspace (8 for 256 rows of
  // 256 columns), and a kernel of its own joins the pieces (5, and a half for each of a tile's).
  // 4096 x 14336, bf16: z and u of 1000 tokens, 448 tiles on 74 pairs, whole 213 us, cut 181 and 13 for the join; backward pass of 1000, 1500
  // and 2048 tokens with all pairs an equal share of the rest, wherever in K that starts, 689, 999, 1290 us, with equal pieces 650, 912,
  // 1164 (dx of 2048 tokens then reads 2.3 GB from memory, its operands six times over); 5 tokens 190 / 195.
  const int rest = p.tiles % pairs;
  p.whole = p.tiles;
  if (t.partial && rest > 0) {
    const double units = p.units, products = t.f32 ? kLimbProducts : 1, piece = 1.0 + (cols > 256 ? 16.0 : 8.0) * (g.M < kPairRows ? g.M : kPairRows) / kPairRows;
    double best = units * products;
    for (int split = 2; split <= p.units && rest * split <= kTrainPieces; ++split) {
      const int rounds = (rest * split + pairs - 1) / pairs;
      const double time = rounds * (std::ceil(units / split) * products + piece) + 5.0 + 0.5 * split;
      if (time < best) {
        best = time;
        p.split = split;
      }
    }
    if (p.split > 1) p.whole = p.tiles - rest;
  }
  const int pieces = (p.tiles - p.whole) * p.split, most = p.whole > pieces ? p.whole : pieces;
  if (most < pairs) pairs = most;
  return pairs;
}

// (A product has fewer tiles to cut than it has tiles, and a tile a piece for every block at most.)
size_t train_umma_partial_bytes(int epilogue, bool f32, int M, int N, long long blocks, int batch) {
  const int cols = epilogue == kEpiGateUp ? 128 : piece_cols(epilogue, f32);
  const long long tiles = (long long)((M + kPairRows - 1) / kPairRows) * ((N + cols - 1) / cols) * batch;
  const long long pieces = blocks < 2 ? 0 : tiles < kTrainPieces && tiles * blocks < kTrainPieces ? tiles * blocks : kTrainPieces;
  return (size_t)pieces * piece_rows(M) * piece_cols(epilogue, f32) * 4;
}

int train_umma_lines(int M) { return (M + 31) / 32; }

cudaError_t launch_train_umma(const TrainUmma& t, cudaStream_t s) {
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return e;
  const int pairs = sms / 2 < kTrainUmmaPairs ? sms / 2 : kTrainUmmaPairs;
  if (t.f32) return launch_train_umma_f32(t, pairs, s);
  return t.g.epilogue == kEpiStore ? launch_one<kEpiStore>(t, pairs, s)
         : t.g.epilogue == kEpiGateUp ? launch_one<kEpiGateUp>(t, pairs, s) : launch_one<kEpiHidden>(t, pairs, s);
}

}  // namespace sffn

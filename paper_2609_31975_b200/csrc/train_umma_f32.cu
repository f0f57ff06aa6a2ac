// Products of the training calls in fp32 on the tensor cores: every operand is three bf16 terms (24 bits), a product the six of
// the terms' products above 2^-27.
//
// Tiles (256 columns), roles and cut tiles as in train_umma.cu.  A K block's six operands, three terms of each, are in shared memory
// at once, 16 KB a CTA each, and all six products are taken from there: half the bytes of copying two operands for every product,
// which the copies (10 TB/s from L2 at most) would bound.  Two blocks fit; each operand's place is given back, and filled for
// the block after next, as soon as its last product is through, so the copies have at least half a block's time more.
// The tensor cores truncate when they add onto an accumulator (5e-8 of its size for every four MMAs): runs of two K blocks get an
// accumulator of their own, its small products first while it is small, and the epilogue warps add the runs up in registers, rounding
// to nearest.  Relative error of y (800 tokens, 512 x 1536, squared RELU) / time of a backward pass (500 tokens, 3840 x 14230): 6.2e-7
// / 1.84 ms, fp32 FMAs 8.0e-7; each block's six products in turn 1.6e-6 / 1.83, runs of one block 2.8e-7 / 1.96, both blocks'
// a0 b0 at the end 4.0e-7 / 1.87 (their places come back too late for the next run).
// Three products of 273, 460 and 664 us there, 1.2 to 1.5 PFLOP/s of bf16, and 295 us for the terms of weights and tokens.
#include "fused_kernel.cuh"
#include "train_umma.cuh"

namespace sffn {
namespace {

using namespace tc;

constexpr int kCols = 256;
constexpr int kPlaces = 12;  // of operands: a_0 a_1 a_2 b_0 b_1 b_2, of two K blocks
constexpr int kThreads = 384;
constexpr int kEpilogueWarps = 8;
constexpr int kSmemBytes = kPlaces * kHalfBytes + 1024 + 256;

struct Maps {
  CUtensorMap a[3], b[3];
};

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
__device__ __forceinline__ void store16(void* base, int64_t at, const float* v, int n, bool wide) {
  float* p = static_cast<float*>(base) + at;
  if (n == 16) {
    st8(p, reinterpret_cast<const uint32_t*>(v), wide);
    st8(p + 8, reinterpret_cast<const uint32_t*>(v) + 8, wide);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (i < n) p[i] = v[i];
  }
}
// The three bf16 terms of the first n of sixteen values (in a workspace: n is 8 or 16).
__device__ __forceinline__ void store16_limbs(void* base, int64_t at, int64_t limb, float* v, int n, bool wide) {
#pragma unroll
  for (int l = 0; l < 3; ++l) {
    __nv_bfloat16* p = static_cast<__nv_bfloat16*>(base) + l * limb + at;
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
    if (n == 16) st8(p, w, wide);
    else *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    if (l < 2) {
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] -= __bfloat162float(__float2bfloat16(v[i]));
    }
  }
}
struct Raw16 {
  float v[16];
  __device__ __forceinline__ void load(const void* base, int64_t at, int n, bool wide) {
    const float* p = static_cast<const float*>(base) + at;
    if (n == 16) {
      ld8(p, reinterpret_cast<uint32_t*>(v), wide);
      ld8(p + 8, reinterpret_cast<uint32_t*>(v) + 8, wide);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = i < n ? p[i] : 0.f;
    }
  }
  __device__ __forceinline__ float get(int i) const { return v[i]; }
};

template <int EPI>
__global__ void __launch_bounds__(kThreads, 1) train_umma_f32_kernel(const __grid_constant__ UmmaParams p, const __grid_constant__ Maps maps) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ int abort_word;
  __shared__ uint32_t tmem_slot;
  __shared__ __align__(8) uint64_t bars[2 * kPlaces + 4];
  volatile int* const abort_flag = &abort_word;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t full = smem_u32(bars), empty = full + 8 * kPlaces, acc_full = empty + 8 * kPlaces, acc_empty = acc_full + 16;
  const int rank = (int)cluster_rank(), pair = (int)blockIdx.x >> 1, pairs = (int)gridDim.x >> 1;

  if (tid == 0) {
    for (int s = 0; s < kPlaces; ++s) {
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
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    Walk walk(p, pairs, pair);
    Item it;
    auto wait_all = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, p.status, p.budget)) != 0; };
    uint32_t block = 0;  // K blocks so far: the places 6 (block mod 2) .., every other phase
    bool ok = true;
    if (warp == 0) {
      int left_out = blockIdx.x == 0 ? p.drop : -1;
      while (ok && walk.step(p, it)) {
        const Place at = place_of(p, it.tile);
        const int m0 = at.m * kPairRows + rank * 128;
        const int n0 = at.n * p.tile_cols + (EPI == kEpiGateUp ? 0 : rank * 128);
        for (int u = it.u0; ok && u < it.u1; ++u, ++block) {
          const int part = u >= p.blocks ? 1 : 0, k0 = (u - part * p.blocks) * kDeep, which = p.batch > 1 ? at.batch : part;
          const uint32_t first = 6 * (block & 1), phase = (block >> 1) & 1;
          // in the order of their first products
#pragma unroll
          for (int i = 0; i < 6; ++i) {
            constexpr int kOrder[6] = {1, 4, 2, 5, 3, 0};
            const int o = kOrder[i], term = o % 3;
            const uint32_t place = first + o;
            ok = wait_all(empty + 8 * place, phase ^ 1);
            if (!ok) break;
            if (elect_one()) {
              const bool of_a = o < 3, mn = of_a ? p.a_mn : p.b_mn;
              const CUtensorMap* map = of_a ? &maps.a[EPI == kEpiGateUp ? 0 : which] : &maps.b[EPI == kEpiGateUp ? rank : which];
              const uint32_t bar = map_rank(full + 8 * place, 0), to = ring + place * kHalfBytes;
              const int r0 = of_a ? m0 : n0;
              if (rank == 0) mbar_expect_tx(full + 8 * place, 2 * kHalfBytes);
              if (o == 0 && left_out-- == 0) {
              } else if (mn) {
                tma_tile_3d(to, map, r0, k0, term, bar);
                tma_tile_3d(to + kHalfBytes / 2, map, r0 + 64, k0, term, bar);
              } else {
                tma_tile_3d(to, map, k0, r0, term, bar);
              }
            }
            __syncwarp();
          }
        }
      }
    } else if (warp == 1 && rank == 0) {
      const uint32_t idesc = idesc_bf16(kPairRows, kCols, p.a_mn, p.b_mn);
      const uint64_t a0 = p.a_mn ? desc_mn_major(ring, kHalfBytes / 2) : desc_k_major(ring);
      const uint64_t b0 = (p.b_mn ? desc_mn_major(ring, kHalfBytes / 2) : desc_k_major(ring)) + 3 * (kHalfBytes >> 4);
      const uint32_t a_step = p.a_mn ? 2048 >> 4 : 32 >> 4, b_step = p.b_mn ? 2048 >> 4 : 32 >> 4;  // sixteen k
      int b = 0, b_phase = 0;
      while (ok && walk.step(p, it)) {
        for (int u = it.u0; ok && u < it.u1;) {
          static_assert(kLimbRun == 2);
          const int end = min(it.u1, u + p.run_units);
          ok = wait_all(acc_empty + 8 * b, b_phase ^ 1);
          if (!ok) break;
          fence_after();
          const uint32_t acc = tmem + b * kCols;
          const bool two = end - u == 2;
          // a1 b1, a1 b0, a2 b0, a0 b1, a0 b2 of both blocks, then a0 b0 of both; the first block's one product early, for its places
#pragma unroll
          for (int i = 0; i < 12; ++i) {
            constexpr int kBlock[12] = {0, 0, 0, 0, 0, 1, 1, 1, 1, 0, 1, 1};
            constexpr int kA[12] = {1, 1, 2, 0, 0, 1, 1, 2, 0, 0, 0, 0}, kB[12] = {1, 0, 0, 1, 2, 1, 0, 0, 1, 0, 2, 0};
            constexpr int kWait[12] = {1, 3, 2, 0, 5, 1, 3, 2, 0, -1, 5, -1}, kGive[12] = {-1, 1, 2, 4, 5, -1, 1, 2, 4, 0, 5, 0};
            if (kBlock[i] && !two) continue;
            const uint32_t at = block + kBlock[i], first = 6 * (at & 1), phase = (at >> 1) & 1, off = first * (kHalfBytes >> 4);
            if (kWait[i] == 1) ok = wait_all(full + 8 * (first + 4), phase);
            if (ok && kWait[i] >= 0) ok = wait_all(full + 8 * (first + kWait[i]), phase);
            if (!ok) break;
            fence_after();
            if (elect_one()) {
#pragma unroll
              for (int k = 0; k < kDeep / 16; ++k)
                umma_pair(acc, a0 + off + kA[i] * (kHalfBytes >> 4) + k * a_step, b0 + off + kB[i] * (kHalfBytes >> 4) + k * b_step, idesc, i > 0 || k > 0);
              if (kGive[i] >= 0) commit_pair(empty + 8 * (first + kGive[i]));
              if (kGive[i] == 0) commit_pair(empty + 8 * (first + 3));
              if (i == (two ? 11 : 9)) commit_pair(acc_full + 8 * b);
            }
            __syncwarp();
          }
          block += end - u;
          if (!ok) break;
          b ^= 1;
          if (b == 0) b_phase ^= 1;
          u = end;
        }
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    const TrainEpilogue& e = p.epi;
    const int quad = warp & 3, half = (warp - 4) >> 2;
    const uint32_t lanes = (uint32_t)(32 * quad) << 16;
    constexpr int kChunks = 8;                                   // of sixteen columns, of a warp
    constexpr int kOut = EPI == kEpiGateUp ? kChunks / 2 : kChunks;  // of sixteen output columns
    // column (in the accumulator) of a chunk: kGateUp: a warp has z and u of 64 neurons, z's chunks first
    auto column = [&](int c) { return EPI == kEpiGateUp ? (c < 4 ? 0 : 128) + 64 * half + 16 * (c & 3) : 128 * half + 16 * c; };
    const uint32_t empty0 = map_rank(acc_empty, 0);
    const uintptr_t wide_out = EPI == kEpiStore ? (uintptr_t)(e.ld_out * 4) : (uintptr_t)(e.ld_zu * 4) | reinterpret_cast<uintptr_t>(e.z) | reinterpret_cast<uintptr_t>(e.u);
    const bool wide_user = (wide_out & 31) == 0;
    const bool wide_own = EPI != kEpiStore && (e.ld_h & 15) == 0;
    int b = 0, b_phase = 0;
    bool ok = true;
    Walk walk(p, pairs, pair);
    Item it;
    while (ok && walk.step(p, it)) {
      const Place at = place_of(p, it.tile);
      const int m = at.m * kPairRows + rank * 128 + 32 * quad + lane;
      const int n0 = at.n * p.tile_cols + (EPI == kEpiGateUp ? 64 : 128) * half;  // first output column of this warp
      const bool row = m < e.M;
      // This item's sums, in tensor memory: as the MMAs left them, or added up over the runs and put back where the last run was.
      uint32_t tacc = 0;
      float acc[16 * kChunks];
#pragma unroll
      for (int i = 0; i < 16 * kChunks; ++i) acc[i] = 0.f;
#pragma unroll 1
      for (int u = it.u0; u < it.u1;) {
        const int end = min(it.u1, u + p.run_units);
        ok = __all_sync(0xffffffffu, mbar_wait(acc_full + 8 * b, b_phase, abort_flag, p.status, p.budget));
        if (!ok) break;
        fence_after();
        tacc = tmem + lanes + b * kCols;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
          float v[16];
          tmem_ld16(tacc + column(c), v);
          tmem_arrived(v);
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[16 * c + i] += v[i];
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
      auto own = [&](int c, float* v) {
        tmem_ld16(tacc + column(c), v);
        tmem_arrived(v);
      };
      // A tile that several pairs share: this warp's part of it is 16 KB of every piece.
      if (it.piece >= 0) {
        float* piece = piece_of(p, it.piece) + (size_t)(rank * 128 + 32 * quad + lane) * kCols;
#pragma unroll 2
        for (int c = 0; c < kChunks; ++c) {
          float v[16];
          own(c, v);
          if (row) put_piece(piece + column(c), v);
        }
      } else {
        if constexpr (EPI == kEpiStore) {
          void* out = e.out[at.batch];
          const bool wide = wide_user && (reinterpret_cast<uintptr_t>(out) & 31) == 0;
#pragma unroll 2
          for (int c = 0; c < kOut; ++c) {
            const int n = n0 + 16 * c;
            float v[16];
            own(c, v);
            if (row && n < e.N) store16(out, m * e.ld_out + n, v, min(16, e.N - n), wide);
          }
        } else if constexpr (EPI == kEpiGateUp) {
#pragma unroll 1
          for (int c = 0; c < kOut; ++c) {
            const int n = n0 + 16 * c;
            float z[16], u[16];
            own(c, z);
            own(c + 4, u);
            const int left = min(16, e.N - n);
            if (e.bias) {
              const float bias = lane < left ? e.bias[n + lane] : 0.f;
#pragma unroll
              for (int i = 0; i < 16; ++i) z[i] += __shfl_sync(0xffffffffu, bias, i);
            }
            if (row && left > 0) {
              if (e.z) {
                store16(e.z, m * e.ld_zu + n, z, left, wide_user);
                store16(e.u, m * e.ld_zu + n, u, left, wide_user);
              }
              act16<false>(e.act, z, z);
              act16<false>(e.act_up, u, u);
#pragma unroll
              for (int i = 0; i < 16; ++i) z[i] *= u[i];
              const int room = (int)min((int64_t)16, e.ld_h - n);
              store16_limbs(e.h, m * e.ld_h + n, e.limb, z, room, wide_own);
            }
          }
        } else {
          Raw16 rz, ru;
          auto fetch = [&](int c) {
            const int n = n0 + 16 * c, left = row ? min(16, e.N - n) : 0;
            rz.load(e.z, m * e.ld_zu + n, left, wide_user);
            ru.load(e.u, m * e.ld_zu + n, left, wide_user);
          };
          auto store = [&](void* to, int64_t at_h, float* v, int room) {
            if (!to || room <= 0) return;
            store16_limbs(to, at_h, e.limb, v, room, wide_own);
          };
          fetch(0);
#pragma unroll 1
          for (int c = 0; c < kOut; ++c) {
            const int n = n0 + 16 * c, room = row ? (int)min((int64_t)16, e.ld_h - n) : 0;
            const int64_t at_h = m * e.ld_h + n;
            float dh[16], a[16], da[16], bv[16], db[16];
            slope16<false>(e.act, rz, a, da);
            slope16<false>(e.act_up, ru, bv, db);
            if (c + 1 < kOut) fetch(c + 1);
            own(c, dh);
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
              const int line = at.m * (kPairRows / 32) + rank * 4 + quad, n_of = n + (lane >> 1);
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

template <int EPI>
cudaError_t launch_one(const UmmaParams& p, const Maps& maps, int pairs, cudaStream_t s) {
  static unsigned long long configured = 0;
  const cudaError_t e = allow_dynamic_smem(train_umma_f32_kernel<EPI>, kSmemBytes, configured);
  if (e != cudaSuccess) return e;
  const cudaError_t launched = launch_clusters(2, train_umma_f32_kernel<EPI>, dim3(2 * pairs), dim3(kThreads), kSmemBytes, s, p, maps);
  if (launched != cudaSuccess || p.whole == p.tiles) return launched;
  return launch_train_join(p, EPI, true, s);
}

}  // namespace

cudaError_t launch_train_split(const float* in, int64_t ld_in, int rows, int cols, __nv_bfloat16* out, int64_t ld_out, int64_t limb, cudaStream_t s) {
  const int64_t total = (int64_t)rows * ((cols + 7) / 8);
  const int64_t want = (total + 255) / 256;
  return launch_pdl(train_split_kernel, dim3((unsigned)(want < 148 * 8 ? want : 148 * 8)), dim3(256), 0, s, in, ld_in, rows, cols, out, ld_out, limb);
}

cudaError_t launch_train_umma_f32(const TrainUmma& t, int pairs, cudaStream_t s) {
  UmmaParams p{};
  pairs = plan_umma(t, t.g.epilogue == kEpiGateUp ? kCols / 2 : kCols, p, pairs);
  static_assert(piece_cols(kEpiStore, true) == kCols && piece_cols(kEpiGateUp, true) == kCols && piece_cols(kEpiHidden, true) == kCols);
  Maps maps;
  if (pairs <= 0 || !make_operand_maps(t, 128, maps.a, maps.b)) return cudaErrorInvalidValue;
  if (t.g.epilogue == kEpiStore) return launch_one<kEpiStore>(p, maps, pairs, s);
  if (t.g.epilogue == kEpiGateUp) return launch_one<kEpiGateUp>(p, maps, pairs, s);
  return launch_one<kEpiHidden>(p, maps, pairs, s);
}

}  // namespace sffn

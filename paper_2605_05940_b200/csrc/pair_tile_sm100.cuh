// Tensor-core tiles of a product D[m,n] = sum_k A[m,k] B[n,k] with an epilogue of the user's choice:
// the main loop behind the vocabulary cross entropy and the linear layer.
//
// Two CTAs on neighbouring SMs (a cluster of 2) work as a pair on a 256 x 256 (or narrower) tile with tcgen05
// .cta_group::2: each CTA stages its own 128 rows of A and its own 128 of the tile's 256 rows of B (both
// K-major bf16, 128-byte swizzle), and its tensor memory receives its own 128 rows of the tile for all 256
// columns.  Two accumulators (all 512 columns of tensor memory) let the epilogue of a tile run under the
// MMAs of the next one.  A stage of the operand ring is two k-steps of 64 deep (64 KB, eight MMAs per
// hand-off): a hand-off costs the tensor pipe about 120 clocks whatever the stage holds.  Three stages are what
// the 227 KB of shared memory hold.
//
// CTA = 576 threads, one CTA per SM, persistent over the tiles its pair's walk yields:
//   warp 0      TMA producer of this CTA's operand stages; the completion of both CTAs' loads is
//               counted on the leader's "full" barrier
//   warp 1      leader CTA (cluster rank 0) only: the MMA issuer of the pair.  In both CTAs this warp
//               owns the tensor memory
//   warps 2-17  epilogue: warp w reads tensor-memory lanes 32*(w%4).., columns of group (w-2)/4, so that
//               every thread owns one row and a quarter (64 columns wide tiles: half) of the tile's columns.  Sixteen warps, four per
//               scheduler: with eight (half a tile each) an epilogue with an activation was bound by its
//               own latencies and took longer than the MMAs of a K = 1536 tile
// An epilogue stores results the size of the tile from registers, 64 bytes of a row per thread and chunk
// (two full 32-byte sectors).  Staging them in shared memory for TMA stores was slower: the MMAs already
// take most of the shared memory's bandwidth, so staging traffic slows the main loop down.  Roles meet at
// mbarriers only, and every wait on one is bounded.
//
// Epi provides (Walk is evaluated by every role alike):
//   Params                     launch parameters, with `int* status` and `int ksteps`
//   rows(p)                    rows of A that exist
//   kBN                        columns of a tile
//   Walk(p, pair, pairs)       the tiles of a pair: bool next(PairTile&)
//   Epi(p, row_local, group)   per epilogue thread; then for every tile begin(tile), for every chunk of 32
//                              columns chunk(acc[32], col0), and end(tile)
#pragma once

#include "ptx_sm100.cuh"

namespace npd {

struct PairTile {
  int row0;         // first row of the pair's 256; this CTA's rows start at row0 + 128 * rank
  int tile;         // column tile (kBN columns)
  int run;          // epilogue's own number of the sequence of tiles this one belongs to
  bool first, last; // of that sequence
};

// 32 consecutive results of a row.  `n` of them exist; `wide` = the address is on a 32-byte boundary (it is on
// a 16-byte one in any case).
template <bool kF32>
__device__ __forceinline__ void store_row32(void* dst, const float (&v)[32], int n, bool wide) {
  constexpr int kWords = kF32 ? 32 : 16;
  uint32_t w[kWords];
#pragma unroll
  for (int i = 0; i < kWords; ++i)
    w[i] = kF32 ? __float_as_uint(v[i % 32]) : pack_bf16x2(v[(2 * i) % 32], v[(2 * i + 1) % 32]);
  uint32_t* p = static_cast<uint32_t*>(dst);
  if (n >= 32 && wide) {
#pragma unroll
    for (int i = 0; i < kWords; i += 8)
      asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p + i), "r"(w[i]), "r"(w[i + 1]), "r"(w[i + 2]),
                   "r"(w[i + 3]), "r"(w[i + 4]), "r"(w[i + 5]), "r"(w[i + 6]), "r"(w[i + 7])
                   : "memory");
  } else if (n >= 32) {
#pragma unroll
    for (int i = 0; i < kWords; i += 4) *reinterpret_cast<uint4*>(p + i) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
  } else {
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      if (i >= n) continue;
      if (kF32) p[i] = w[i % kWords];
      else reinterpret_cast<uint16_t*>(p)[i] = static_cast<uint16_t>(i & 1 ? w[i / 2] >> 16 : w[i / 2]);
    }
  }
}

// kBN = columns of a pair tile: 256, or 128 or 64 for problems that would not give every pair a tile otherwise.
template <int kBN>
struct PairCfg {
  static constexpr int BM = 128, BN = kBN, BK = 64, UK = 16;
  static constexpr int BNH = BN / 2;  // rows of B each CTA stages
  static constexpr int KS = 2, STAGES = BN == 256 ? 3 : (BN == 128 ? 4 : 5);
  static constexpr int A_BYTES = BM * BK * 2;
  static constexpr int B_BYTES = BNH * BK * 2;
  static constexpr int EPI_WARPS = 16;
  static constexpr int GROUPS = BN >= 128 ? 4 : 2;  // groups of four epilogue warps that have columns
  static constexpr int BNG = BN / GROUPS;           // columns of a group: 64 or 32
  static constexpr int THREADS = 64 + 32 * EPI_WARPS;
  static constexpr int TMEM_COLS = 2 * BN;
  static constexpr int OFF_A = 0;
  static constexpr int OFF_B = OFF_A + STAGES * KS * A_BYTES;
  static constexpr int OFF_BAR = OFF_B + STAGES * KS * B_BYTES;
  static constexpr int NUM_BARS = 2 * STAGES + 4;
  static constexpr int SMEM_BYTES = OFF_BAR + NUM_BARS * 8 + 16 + 1024;
};

template <class Epi>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(PairCfg<Epi::kBN>::THREADS, 1)
pair_tile_kernel(const __grid_constant__ CUtensorMap tmap_a, const __grid_constant__ CUtensorMap tmap_b,
                 const typename Epi::Params p) {
  using L = PairCfg<Epi::kBN>;
  constexpr int BM = L::BM, BN = L::BN, BK = L::BK, UK = L::UK, BNH = L::BNH, KS = L::KS, STAGES = L::STAGES, A_BYTES = L::A_BYTES,
                B_BYTES = L::B_BYTES, GROUPS = L::GROUPS, BNG = L::BNG, OFF_A = L::OFF_A, OFF_B = L::OFF_B, OFF_BAR = L::OFF_BAR,
                NUM_BARS = L::NUM_BARS, TMEM_COLS = L::TMEM_COLS;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + OFF_BAR);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + NUM_BARS);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();  // 0 = leader of the pair
  const uint32_t full0 = smem_u32(bars);
  const uint32_t empty0 = full0 + 8 * STAGES;
  const uint32_t tfull0 = empty0 + 8 * STAGES;
  const uint32_t tempty0 = tfull0 + 16;

  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(full0 + 8 * s, 1);
      mbar_init(empty0 + 8 * s, 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(tfull0 + 8 * b, 1);
      mbar_init(tempty0 + 8 * b, 2 * 4 * GROUPS);  // the epilogue warps of both CTAs, counted in the leader
    }
    *abort_flag = 0;
    fence_mbar_init();
    prefetch_tmap(&tmap_a);
    prefetch_tmap(&tmap_b);
  }
  if (warp == 1) tmem_alloc_pair(smem_u32(tmem_slot), TMEM_COLS);
  tc_fence_before_sync();
  __syncthreads();
  cluster_sync_all();  // the peer's barriers are initialised before anything is sent to them
  tc_fence_after_sync();
  const uint32_t tmem_base = *tmem_slot;
  const uint32_t full_leader = mapa_shared(full0, 0);
  const uint32_t tempty_leader = mapa_shared(tempty0, 0);

  // Everything above touched only this CTA's own resources; what follows reads what earlier kernels
  // of the stream wrote and overwrites what they read.
  grid_dependency_wait();
  grid_launch_dependents();

  typename Epi::Walk walk(p, static_cast<int>(blockIdx.x >> 1), static_cast<int>(gridDim.x >> 1));
  PairTile t;

  if (warp == 0) {
    // ---------------------- operand producer ----------------------
    if (lane == 0) {
      uint32_t it = 0;
      bool ok = true;
      const int rows = Epi::rows(p);
      while (ok && walk.next(t)) {
        const int ra = t.row0 + static_cast<int>(rank) * BM;
        const int rb = t.tile * BN + static_cast<int>(rank) * BNH;
        // A CTA whose rows do not exist fetches none: what its rows of the tile hold is never stored.
        const bool mine = ra < rows, both = t.row0 + BM < rows;
        const uint32_t step_bytes = (both ? 2 : 1) * A_BYTES + 2 * B_BYTES;
        for (int ks = 0; ks < p.ksteps; ks += KS, ++it) {
          const uint32_t st = it % STAGES, ph = (it / STAGES) & 1;
          const int nk = min(KS, p.ksteps - ks);
          if (!(ok = mbar_wait(empty0 + 8 * st, ph ^ 1, abort_flag))) break;
          // the leader's barrier counts the bytes of both CTAs' loads of this stage
          if (rank == 0) mbar_arrive_expect_tx(full0 + 8 * st, nk * step_bytes);
          const uint32_t fb = full_leader + 8 * st;
          for (int h = 0; h < nk; ++h) {
            if (mine) tma_load_2d_pair(smem_u32(smem + OFF_A + (st * KS + h) * A_BYTES), &tmap_a, fb, (ks + h) * BK, ra);
            tma_load_2d_pair(smem_u32(smem + OFF_B + (st * KS + h) * B_BYTES), &tmap_b, fb, (ks + h) * BK, rb);
          }
        }
      }
      // Drain: a stage is released only after its loads landed and the MMAs that read it finished, so
      // waiting for the release of the last stages covers both.
      const uint32_t last = it < STAGES ? it : STAGES;
      for (uint32_t j = 0; j < last && ok; ++j) {
        const uint32_t i2 = it - 1 - j;
        ok = mbar_wait(empty0 + 8 * (i2 % STAGES), (i2 / STAGES) & 1, abort_flag);
      }
      if (!ok) {
        // Aborted: nobody may be left to release the stages, but the loads already issued still land
        // in this CTA's shared memory.  The leader's "full" barriers count both CTAs' bytes; the peer
        // cannot wait on them and lets the grace period pass instead.
        if (rank == 0) {
          for (uint32_t j = 0; j < last; ++j) {
            const uint32_t i2 = it - 1 - j;
            mbar_wait_drain(full0 + 8 * (i2 % STAGES), (i2 / STAGES) & 1);
          }
        } else {
          grace_sleep();
        }
      }
    }
  } else if (warp == 1) {
    // ---------------------- MMA issuer ----------------------
    if (rank == 0 && lane == 0) {
      constexpr uint32_t idesc = umma_idesc_bf16(2 * BM, BN, false, false);
      uint32_t it = 0, tile = 0;
      bool ok = true;
      for (; ok && walk.next(t); ++tile) {
        const uint32_t buf = tile & 1, tph = (tile >> 1) & 1;
        if (!(ok = mbar_wait(tempty0 + 8 * buf, tph ^ 1, abort_flag))) break;
        tc_fence_after_sync();
        const uint32_t d_tmem = tmem_base + buf * BN;
        for (int ks = 0; ks < p.ksteps; ks += KS, ++it) {
          const uint32_t st = it % STAGES, ph = (it / STAGES) & 1;
          const int nk = min(KS, p.ksteps - ks);
          if (!(ok = mbar_wait(full0 + 8 * st, ph, abort_flag))) break;
          tc_fence_after_sync();
          for (int h = 0; h < nk; ++h) {
            const uint32_t sa = smem_u32(smem + OFF_A + (st * KS + h) * A_BYTES);
            const uint32_t sb = smem_u32(smem + OFF_B + (st * KS + h) * B_BYTES);
#pragma unroll
            for (int k = 0; k < BK / UK; ++k)
              umma_bf16_pair(d_tmem, umma_desc_sw128(sa + k * (UK * 2), 16, 1024),
                             umma_desc_sw128(sb + k * (UK * 2), 16, 1024), idesc, (ks > 0 || h > 0 || k > 0) ? 1u : 0u);
          }
          umma_commit_pair(empty0 + 8 * st);
        }
        if (ok) umma_commit_pair(tfull0 + 8 * buf);
      }
    }
  } else if (warp < 2 + 4 * GROUPS) {
    // ---------------------- epilogue ----------------------
    const int lg = warp & 3;            // the lane group of tensor memory this warp may read
    const int group = (warp - 2) >> 2;  // which BNG columns of the tile
    Epi epi(p, static_cast<int>(rank) * BM + lg * 32 + lane, group);
    uint32_t tile = 0;
    bool ok = true;
    for (; ok && walk.next(t); ++tile) {
      const uint32_t buf = tile & 1, tph = (tile >> 1) & 1;
      epi.begin(t);
      if (!(ok = __all_sync(0xffffffffu, mbar_wait(tfull0 + 8 * buf, tph, abort_flag)))) break;
      tc_fence_after_sync();
      const uint32_t taddr = tmem_base + (static_cast<uint32_t>(lg * 32) << 16) + buf * BN + group * BNG;
#pragma unroll 1
      for (int c = 0; c < BNG / 32; ++c) {
        uint32_t acc[32];
        __syncwarp();  // the epilogue's branches may have parted the warp
        tmem_ld32(taddr + c * 32, acc);
        tmem_ld_wait();
        if (c == BNG / 32 - 1) {
          // everything this warp needs of the accumulator is in registers: it may be overwritten
          tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster(tempty_leader + 8 * buf);
        }
        epi.chunk(acc, t.tile * BN + group * BNG + c * 32);
      }
      epi.end(t);
    }
  }

  // ---------------------- teardown ----------------------
  // Neither CTA may leave (or free tensor memory) while its peer can still send it barrier arrivals or
  // have MMAs reading its shared memory.
  tc_fence_before_sync();
  __syncthreads();
  cluster_sync_all();
  tc_fence_after_sync();
  if (warp == 1) {
    __syncwarp();
    tmem_dealloc_pair(tmem_base, TMEM_COLS);
  }
  if (threadIdx.x == 0 && *abort_flag != 0) report_timeout(p.status);
}

}  // namespace npd

// Tensor-core tiles of a product D[m,n] = sum_k A[m,k] B[n,k] with an epilogue of the user's choice:
// the main loop behind the vocabulary cross entropy and the linear layer.
//
// Two CTAs on neighbouring SMs (a cluster of 2) work as a pair on a 256 x 256 tile with tcgen05
// .cta_group::2: each CTA stages its own 128 rows of A and its own 128 of the tile's 256 rows of B (both
// K-major bf16, 128-byte swizzle), and its tensor memory receives its own 128 rows of the tile for all 256
// columns.  Two accumulators (all 512 columns of tensor memory) let the epilogue of a tile run under the
// MMAs of the next one.  A stage of the operand ring is two k-steps of 64 deep (64 KB, eight MMAs per
// hand-off): a hand-off costs the tensor pipe about 120 clocks whatever the stage holds.  Three stages, and
// 32 KB for the output staging, fill the 227 KB of shared memory.
//
// CTA = 384 threads, one CTA per SM, persistent over the tiles its pair's walk yields:
//   warp 0      TMA producer of this CTA's operand stages; the completion of both CTAs' loads is
//               counted on the leader's "full" barrier
//   warp 1      leader CTA (cluster rank 0) only: the MMA issuer of the pair.  In both CTAs this warp
//               owns the tensor memory
//   warps 2, 3  one storing thread each, for the left and the right half of a tile's columns
//   warps 4-11  epilogue: warp w reads tensor-memory lanes 32*(w%4).., columns 128*((w-4)/4).., so that
//               every thread owns one row and half of the tile's columns
// An epilogue with results the size of the tile writes them, 128 rows x 64 bytes at a time, to a ring of
// two staging buffers per half (64-byte swizzle); the storing thread hands them to TMA stores, which
// clip them at the matrix's edges.  Roles meet at mbarriers only, and every wait is bounded.
//
// Epi provides (all evaluated by every role alike unless said otherwise):
//   Params                     launch parameters, with `int* status` and `int ksteps`
//   Walk(p, pair, pairs, rank) the tiles of a pair: bool next(PairTile&)
//   kOuts                      tile-sized results per tile (0, 1 or 2); kF32 = the first is fp32, else bf16
//                              (a second one is always bf16)
//   steps(p, tile, half, row0) 32-column chunks of this half that have to be stored (0 .. 4)
//   keeps(p, tile, col)        whether a staging buffer whose first column is `col` of the tile is stored
//   out_col(p, tile)           column of the results that the tile's column 0 goes to
//   Epi(p, row_local, half)    per epilogue thread; then for every tile begin(tile), for every chunk
//                              chunk(acc[32], col0, out), and end(tile); out[i] is the i-th staging buffer's
//                              64 bytes of this row: the first result's one (bf16) or two (fp32), then the second's
#pragma once

#include "ptx_sm100.cuh"

namespace npd {

struct PairTile {
  int row0;         // first row of the pair's 256; this CTA's rows start at row0 + 128 * rank
  int tile;         // column tile (256 columns)
  int run;          // epilogue's own number of the sequence of tiles this one belongs to
  bool first, last; // of that sequence
};

namespace pair_cfg {
constexpr int BM = 128, BN = 256, BK = 64, UK = 16;
constexpr int BNH = BN / 2;
constexpr int KS = 2, STAGES = 3;
constexpr int A_BYTES = BM * BK * 2;
constexpr int B_BYTES = BNH * BK * 2;
constexpr int OUT_BYTES = 128 * 64;  // one staging buffer
constexpr int OUT_BUFS = 2;          // per half
constexpr int THREADS = 384;
constexpr int TMEM_COLS = 512;
constexpr int OFF_A = 0;
constexpr int OFF_B = OFF_A + STAGES * KS * A_BYTES;
constexpr int OFF_OUT = OFF_B + STAGES * KS * B_BYTES;
constexpr int OFF_BAR = OFF_OUT + 2 * OUT_BUFS * OUT_BYTES;
constexpr int NUM_BARS = 2 * STAGES + 4 + 4 * OUT_BUFS;
constexpr int SMEM_BYTES = OFF_BAR + NUM_BARS * 8 + 16 + 1024;
}  // namespace pair_cfg

template <class Epi>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(pair_cfg::THREADS, 1)
pair_tile_kernel(const __grid_constant__ CUtensorMap tmap_a, const __grid_constant__ CUtensorMap tmap_b,
                 const __grid_constant__ CUtensorMap tmap_o0, const __grid_constant__ CUtensorMap tmap_o1,
                 const typename Epi::Params p) {
  using namespace pair_cfg;
  constexpr int kOuts = Epi::kOuts;
  constexpr int kSub = Epi::kF32 ? 2 : 1;                                     // staging buffers per chunk: first result,
  constexpr int kPer = kOuts == 0 ? 1 : kSub + (kOuts > 1 ? 1 : 0);          // all results
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
  const uint32_t ofull0 = tempty0 + 16;               // [half][OUT_BUFS]
  const uint32_t oempty0 = ofull0 + 8 * 2 * OUT_BUFS;  // [half][OUT_BUFS]

  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(full0 + 8 * s, 1);
      mbar_init(empty0 + 8 * s, 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(tfull0 + 8 * b, 1);
      mbar_init(tempty0 + 8 * b, 16);  // 8 epilogue warps of each CTA, counted in the leader
    }
    for (int i = 0; i < 2 * OUT_BUFS; ++i) {
      mbar_init(ofull0 + 8 * i, 4);   // the four warps of the half
      mbar_init(oempty0 + 8 * i, 1);  // the half's storing thread
    }
    *abort_flag = 0;
    fence_mbar_init();
    prefetch_tmap(&tmap_a);
    prefetch_tmap(&tmap_b);
    if (kOuts > 0) prefetch_tmap(&tmap_o0);
    if (kOuts > 1) prefetch_tmap(&tmap_o1);
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
      while (ok && walk.next(t)) {
        const int ra = t.row0 + static_cast<int>(rank) * BM;
        const int rb = t.tile * BN + static_cast<int>(rank) * BNH;
        for (int ks = 0; ks < p.ksteps; ks += KS, ++it) {
          const uint32_t st = it % STAGES, ph = (it / STAGES) & 1;
          const int nk = min(KS, p.ksteps - ks);
          if (!(ok = mbar_wait(empty0 + 8 * st, ph ^ 1, abort_flag))) break;
          // the leader's barrier counts the bytes of both CTAs' loads of this stage
          if (rank == 0) mbar_arrive_expect_tx(full0 + 8 * st, 2 * nk * (A_BYTES + B_BYTES));
          const uint32_t fb = full_leader + 8 * st;
          for (int h = 0; h < nk; ++h) {
            tma_load_2d_pair(smem_u32(smem + OFF_A + (st * KS + h) * A_BYTES), &tmap_a, fb, (ks + h) * BK, ra);
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
  } else if (warp < 4) {
    // ---------------------- storing threads ----------------------
    if (kOuts > 0 && lane == 0) {
      const int half = warp - 2;
      uint32_t oit = 0;
      int prev = -1;  // buffer of the copy in flight
      bool ok = true;
      while (ok && walk.next(t)) {
        const int row0 = t.row0 + static_cast<int>(rank) * BM;
        const int n = Epi::steps(p, t, half, row0);
        for (int j = 0; j < n * kPer && ok; ++j, ++oit) {
          const int b = half * OUT_BUFS + static_cast<int>(oit % OUT_BUFS);
          if (!(ok = mbar_wait(ofull0 + 8 * b, (oit / OUT_BUFS) & 1, abort_flag))) break;
          const int c = j / kPer, which = j % kPer < kSub ? 0 : 1, sub = which == 0 ? j % kPer : 0;
          const int col = half * BNH + c * 32 + sub * 16;  // within the tile
          if (Epi::keeps(p, t, col))
            tma_store_2d(which == 0 ? &tmap_o0 : &tmap_o1, smem_u32(smem + OFF_OUT + b * OUT_BYTES),
                         Epi::out_col(p, t) + col, row0);
          tma_store_commit();
          if (prev >= 0) {
            tma_store_wait_read<1>();  // the copy before this one has read its buffer
            mbar_arrive(oempty0 + 8 * prev);
          }
          prev = b;
        }
      }
      tma_store_wait_read<0>();
      if (prev >= 0) mbar_arrive(oempty0 + 8 * prev);
      tma_store_wait_all<0>();
    }
  } else {
    // ---------------------- epilogue ----------------------
    const int e = warp - 4;
    const int lg = e & 3;     // == warp % 4: the lane group of tensor memory this warp may read
    const int half = e >> 2;  // which 128 columns of the tile
    const int row_local = lg * 32 + lane;
    const uint32_t swz = static_cast<uint32_t>((row_local >> 1) & 3);  // 64-byte swizzle
    Epi epi(p, static_cast<int>(rank) * BM + row_local, half);
    uint32_t tile = 0, oit = 0;
    bool ok = true;
    for (; ok && walk.next(t); ++tile) {
      const uint32_t buf = tile & 1, tph = (tile >> 1) & 1;
      const int row0 = t.row0 + static_cast<int>(rank) * BM;
      epi.begin(t);
      if (!(ok = __all_sync(0xffffffffu, mbar_wait(tfull0 + 8 * buf, tph, abort_flag)))) break;
      tc_fence_after_sync();
      const uint32_t taddr = tmem_base + (static_cast<uint32_t>(lg * 32) << 16) + buf * BN + half * BNH;
      const int n = kOuts > 0 ? Epi::steps(p, t, half, row0) : BNH / 32;
      // once everything this warp needs of an accumulator is in registers it may be overwritten
      auto release = [&]() {
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(tempty_leader + 8 * buf);
      };
      if (n == 0) release();
#pragma unroll 1
      for (int c = 0; c < n && ok; ++c) {
        uint32_t acc[32];
        __syncwarp();  // the epilogue's branches may have parted the warp
        tmem_ld32(taddr + c * 32, acc);
        tmem_ld_wait();
        if (c == n - 1) release();
        uint32_t out[kPer][16];
        epi.chunk(acc, t.tile * BN + half * BNH + c * 32, out);
        if (kOuts > 0) {
#pragma unroll
          for (int s = 0; s < kPer; ++s, ++oit) {
            const int b = half * OUT_BUFS + static_cast<int>(oit % OUT_BUFS);
            if (!(ok = __all_sync(0xffffffffu, mbar_wait(oempty0 + 8 * b, ((oit / OUT_BUFS) & 1) ^ 1, abort_flag)))) break;
            uint8_t* orow = smem + OFF_OUT + b * OUT_BYTES + row_local * 64;
            const uint32_t* w = out[s];
#pragma unroll
            for (int q = 0; q < 4; ++q)
              *reinterpret_cast<uint4*>(orow + ((static_cast<uint32_t>(q) ^ swz) << 4)) =
                  make_uint4(w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(ofull0 + 8 * b);
          }
        }
      }
      if (!ok) break;
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
  if (threadIdx.x == 0 && *abort_flag != 0 && p.status != nullptr) atomicCAS(p.status, 0, kStatusTimeout);
}

}  // namespace npd

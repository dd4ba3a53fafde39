// The bf16 GEMM's tile through registers and two buffers in LDS (sk_bf16_gemm.hip says what it is made for).
#pragma once
#include "sk_bf16_finish.h"
#include "sk_bf16_tile.h"

namespace sk {

// One tile configuration of the GEMM: its work-group size, its LDS footprint and its body
// (the work of one work-group, given the group's index in the launch and LDS of at
// least LDS_BYTES).  The body is a device function so that one launch can carry the
// work-groups of two independent GEMMs (dual_gemm_kernel below).
// ACT: 0 and more for a dense layer's results (sk_bf16_finish.h) in place of the product's.
template <int BM, int BN, bool A_KC, bool B_KC, typename OutT, bool COLSUM, int ACT = -1>
struct GemmTile {
  static constexpr int NTH = 256, WAVES_N = 2;
  typedef OpTile<BM, A_KC, BK, NTH> TA;
  typedef OpTile<BN, B_KC, BK, NTH> TB;
  static constexpr int WM = BM / 2, WN = BN / 2, TM = WM / 32, TN = WN / 32;
  static constexpr int STAGE = TA::ELEMS + TB::ELEMS;
  static constexpr int LDS_BYTES = 2 * STAGE * 2;
  // bf16 results leave through a wave-private strip of LDS (32 rows of the wave's sub-tile at
  // a time, see the epilogue), carved out of a main buffer that is idle by then.
  static constexpr int WAVE_STRIP = 32 * WN * 2;
  static_assert((NTH / 64) * WAVE_STRIP <= STAGE * 2, "the waves' strips fit one main buffer");
  static_assert(ACT < 0 || (sizeof(OutT) == 2 && 4 * FinishStrip<TN>::BYTES <= LDS_BYTES), "a dense layer's strips");
  static __device__ __forceinline__ void run(const GemmArgs& p, int block, unsigned char* smem, const FinishArgs& f = FinishArgs{});
};

template <int BM, int BN, bool A_KC, bool B_KC, typename OutT, bool COLSUM, int ACT>
__device__ __forceinline__ void
GemmTile<BM, BN, A_KC, B_KC, OutT, COLSUM, ACT>::run(const GemmArgs& p, int block, unsigned char* const smem, const FinishArgs& f) {
  bf16* const lds = reinterpret_cast<bf16*>(smem);

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = wave / WAVES_N, wn = wave % WAVES_N;

  const int tiles = p.tiles_m * p.tiles_n;
  const int id = xcd_remap(block, tiles * p.splits);
  const int split = id / tiles;
  int tile_m, tile_n;
  tile_coords(id - split * tiles, p.tiles_m, p.tiles_n, tile_m, tile_n);
  const int m0 = tile_m * BM, n0 = tile_n * BN;
  const int k_begin = split * p.k_per_split;
  const int k_end = (k_begin + p.k_per_split < p.K) ? k_begin + p.k_per_split : p.K;
  const int nk = (k_end - k_begin + BK - 1) / BK;

  const bf16* __restrict__ A = static_cast<const bf16*>(p.A);
  const bf16* __restrict__ B = static_cast<const bf16*>(p.B);

  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  f32x16 csum[COLSUM ? TN : 1];
  if (COLSUM) {
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) csum[j][r] = 0.f;
  }
  // Column sums of B ride on the MFMA: an all-ones fragment in place of A's.
  const bool do_colsum = COLSUM && p.colsum != nullptr && tile_m == 0 && wm == 0;
  bf16x8 ones;
#pragma unroll
  for (int j = 0; j < 8; ++j) ones[j] = (bf16)1.0f;

  // One k step (16 wide): fragments of the four steps of a chunk are read one step
  // ahead of the MFMAs that use them (two fragment sets), so LDS latency hides
  // behind the matrix pipe.
  bf16x8 fa0[TM], fb0[TN], fa1[TM], fb1[TN];
  auto read = [&](const bf16* As, int ks, bf16x8 (&fa)[TM], bf16x8 (&fb)[TN]) {
    const bf16* Bs = As + TA::ELEMS;
#pragma unroll
    for (int i = 0; i < TM; ++i) fa[i] = read_frag<A_KC, TA::LD>(As, wm * WM + i * 32, ks, lane);
#pragma unroll
    for (int j = 0; j < TN; ++j) fb[j] = read_frag<B_KC, TB::LD>(Bs, wn * WN + j * 32, ks, lane);
  };
  auto mma = [&](const bf16x8 (&fa)[TM], const bf16x8 (&fb)[TN]) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[j], fa[i], acc[i][j], 0, 0, 0);
    if (COLSUM) {
      if (do_colsum) {
#pragma unroll
        for (int j = 0; j < TN; ++j)
          csum[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[j], ones, csum[j], 0, 0, 0);
      }
    }
  };
  // Work per chunk and thread: NMMA MFMAs and NDSR fragment reads per k step.  Each k step is one scheduling
  // phase in which the other instructions are spread evenly between the MFMAs
  // (sched_phase), so they issue in the shadow of the matrix pipe instead of in a
  // burst that stalls it (the texture path takes 16 cycles per 16-byte-per-lane load).
  constexpr int NDSR = (A_KC ? TM : 2 * TM) + (B_KC ? TN : 2 * TN);
  constexpr int NMMA = TM * TN;

  // This lane's bias values (four columns per 8-column group of each 32-column block),
  // fetched before the main loop so the epilogue does not wait for them; through a
  // buffer window of N elements (none without a bias), so no lane needs a branch.
  constexpr bool HAS_BIAS = sizeof(OutT) == 2 && ACT < 0;
  uint2 bias_r[HAS_BIAS ? TN : 1][4];
  if constexpr (HAS_BIAS) {
    const GWindow bias_w = make_window(p.bias, 0, p.bias != nullptr ? p.N : 0, 2);
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
        const int gn = n0 + wn * WN + j * 32 + q * 8 + (lane >> 5) * 4;
        const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(bias_w.rsrc, gn * 2, 0, 0);
        bias_r[j][q] = make_uint2(v.x, v.y);
      }
  }

  {
    // An iteration is too short to cover a load's latency, so two
    // register sets keep the loads of chunk kc + 2 in flight while chunk kc + 1,
    // loaded one iteration earlier, is stored.  (Four and six sets were measured on the
    // shapes of this layer and were no faster.)
    uint4 ra0[TA::PIECES], rb0[TB::PIECES], ra1[TA::PIECES], rb1[TB::PIECES];
    TA::load(ra0, A, p.lda, m0, p.M, k_begin, k_end, p.K, tid);
    TB::load(rb0, B, p.ldb, n0, p.N, k_begin, k_end, p.K, tid);
    TA::load(ra1, A, p.lda, m0, p.M, k_begin + BK, k_end, p.K, tid);
    TB::load(rb1, B, p.ldb, n0, p.N, k_begin + BK, k_end, p.K, tid);
    TA::store(lds, ra0, tid);
    TB::store(lds + TA::ELEMS, rb0, tid);
    __syncthreads();
    auto iteration = [&](const bf16* As, bf16* An, uint4 (&la)[TA::PIECES], uint4 (&lb)[TB::PIECES],
                         uint4 (&sa)[TA::PIECES], uint4 (&sb)[TB::PIECES], int k0) {
      // loads into (la, lb) for chunk k0, A's during k step 0 and B's during k step 1 (in
      // one burst they hold the waves at the memory pipe's queue; measured 1 % on the
      // [8192 x 1024..4096] shapes); stores from (sa, sb), loaded an iteration ago
      __builtin_amdgcn_sched_barrier(0);
      read(As, 1, fa1, fb1);
      TA::load(la, A, p.lda, m0, p.M, k0, k_end, p.K, tid);
      mma(fa0, fb0);
      sched_phase<NMMA, NDSR, TA::PIECES, 0>();
      read(As, 2, fa0, fb0);
      TB::load(lb, B, p.ldb, n0, p.N, k0, k_end, p.K, tid);
      mma(fa1, fb1);
      TA::store(An, sa, tid);
      sched_phase<NMMA, NDSR, TB::PIECES, TA::PIECES>();
      read(As, 3, fa1, fb1);
      mma(fa0, fb0);
      TB::store(An + TA::ELEMS, sb, tid);
      sched_phase<NMMA, NDSR, 0, TB::PIECES>();
      // the barrier one k step before the end of the chunk: the first fragments of the
      // next chunk come in behind the last step's MFMAs, not behind the barrier
      __syncthreads();
      read(An, 0, fa0, fb0);
      mma(fa1, fb1);
      sched_phase<NMMA, NDSR, 0, 0>();
    };
    read(lds, 0, fa0, fb0);
    for (int kc = 0; kc < nk; kc += 2) {
      iteration(lds, lds + STAGE, ra0, rb0, ra1, rb1, k_begin + (kc + 2) * BK);
      // an all-zero chunk when nk is odd
      iteration(lds + STAGE, lds, ra1, rb1, ra0, rb0, k_begin + (kc + 3) * BK);
    }
  }

  // ---- epilogue: accumulators -> global ----
  // Lane l owns output row l % 32 of each 32-row block and, for q = 0..3, the four
  // columns 8 q + 4 (l / 32) .. +3 of each 32-column block.
  //   fp32: those 16 bytes are stored as they are (32-byte row segments, merged by the L2).
  //   bf16: the two half-waves exchange the halves of neighbouring column groups
  //     (v_permlane32_swap), after which every lane holds eight consecutive columns; the
  //     wave then turns each 32-row block of its sub-tile over through a strip of LDS that
  //     only it touches (no barrier: one wave's LDS operations execute in order), so that
  //     eight consecutive lanes hold one whole row of the sub-tile and a store instruction
  //     writes complete 128-byte lines.  Stored straight from registers the same data left as
  //     32 scattered 32-byte segments per instruction, which the store path takes four
  //     times as long to work through: with the stores switched off the [8192 x 512] .
  //     [512 x 4096] product of BERT-large took 37 us instead of 50, and most of that gap
  //     stayed when the stores went to a cache-resident scratch target instead, i.e. it was
  //     the instructions, not the bytes.  Pieces are XOR-swizzled by row so that neither the
  //     column-wise writes nor the row-wise reads collide on LDS banks.
  OutT* __restrict__ C = static_cast<OutT*>(p.C) +
                         (sizeof(OutT) == 4 ? (int64_t)split * p.M * p.ldc : (int64_t)0);
  const float scale = p.scale;
  const int wn0 = n0 + wn * WN;  // first global column of this wave
  const int n_store = p.n_store > 0 ? p.n_store : p.N;

  if constexpr (ACT >= 0) {
    uint4 bias[FinishStrip<TN>::STEPS];
    finish_bias<TN>(bias, p.bias, wn0, p.N, lane);
    __syncthreads();   // (the strips lie in the main buffers)
#pragma unroll
    for (int i = 0; i < TM; ++i)
      finish_rows<ACT, TN>(acc[i], f, bias, p.C, p.ldc, m0 + wm * WM + i * 32, wn0, p.M, p.N, smem + wave * FinishStrip<TN>::BYTES, lane);
  } else if constexpr (sizeof(OutT) == 4) {
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int gm = m0 + wm * WM + i * 32 + (lane & 31);
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int gn = wn0 + j * 32 + q * 8 + (lane >> 5) * 4;
          if (gm < p.M && gn < n_store)
            *reinterpret_cast<float4*>(reinterpret_cast<float*>(C) + (int64_t)gm * p.ldc + gn) =
                make_float4(acc[i][j][q * 4 + 0] * scale, acc[i][j][q * 4 + 1] * scale,
                            acc[i][j][q * 4 + 2] * scale, acc[i][j][q * 4 + 3] * scale);
        }
    }
  } else {
    constexpr int PPRW = WN / 8;        // 16-byte pieces per row of the wave's sub-tile
    constexpr int RPI = 64 / PPRW;      // rows one store instruction covers
    constexpr int ROW_BYTES = WN * 2;
    // The strips live in the main buffer.  The last k step still read fragments after the
    // loop's last barrier, so one more comes first.
    __syncthreads();
    unsigned char* const strip = smem + wave * WAVE_STRIP;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int row_w = lane & 31;
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int pr = 0; pr < 2; ++pr) {
          uint2 w[2];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int q = 2 * pr + h;
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = acc[i][j][q * 4 + e] * scale;
            const uint2 bb = bias_r[j][q];
            v[0] += bf16_bits_to_float(bb.x & 0xffffu);
            v[1] += bf16_bits_to_float(bb.x >> 16);
            v[2] += bf16_bits_to_float(bb.y & 0xffffu);
            v[3] += bf16_bits_to_float(bb.y >> 16);
            w[h].x = pack_bf16x2(v[0], v[1]);
            w[h].y = pack_bf16x2(v[2], v[3]);
          }
          typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
          const u32x2 s0 = __builtin_amdgcn_permlane32_swap(w[0].x, w[1].x, false, false);
          const u32x2 s1 = __builtin_amdgcn_permlane32_swap(w[0].y, w[1].y, false, false);
          // columns j * 32 + 16 pr + 8 (l / 32) .. + 7 of the sub-tile: piece 4 j + 2 pr + l / 32
          const int piece = j * 4 + pr * 2 + (lane >> 5);
          *reinterpret_cast<uint4*>(strip + row_w * ROW_BYTES + ((piece ^ (row_w & (PPRW - 1))) * 16)) =
              make_uint4(s0.x, s1.x, s0.y, s1.y);
        }
#pragma unroll
      for (int r0 = 0; r0 < 32; r0 += RPI) {
        const int row_r = r0 + lane / PPRW, piece = lane % PPRW;
        const uint4 v = *reinterpret_cast<const uint4*>(strip + row_r * ROW_BYTES + ((piece ^ (row_r & (PPRW - 1))) * 16));
        const int gm = m0 + wm * WM + i * 32 + row_r;
        const int gn = wn0 + piece * 8;
        if (gm < p.M && gn < n_store)
          *reinterpret_cast<uint4*>(reinterpret_cast<bf16*>(C) + (int64_t)gm * p.ldc + gn) = v;
      }
    }
  }

  if (COLSUM) {
    // every D column of csum holds the same sums; lanes 0 and 32 write them out
    if (do_colsum && (lane & 31) == 0) {
      float* out = p.colsum + (int64_t)split * p.N;
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int gn = wn0 + j * 32 + q * 8 + (lane >> 5) * 4;
          if (gn < p.N)
            *reinterpret_cast<float4*>(out + gn) = make_float4(
                csum[j][q * 4 + 0], csum[j][q * 4 + 1], csum[j][q * 4 + 2], csum[j][q * 4 + 3]);
        }
    }
  }
}

}  // namespace sk

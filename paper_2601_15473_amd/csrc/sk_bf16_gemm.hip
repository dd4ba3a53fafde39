// bf16 MFMA GEMM with fp32 accumulation for gfx950: the contraction every
// two-pass plan of the SKLinear forward/backward is made of.
//
//   C[M, N] = scale * (A . B) (+ bias[n]),   or raw fp32 split-K partial slabs.
//
// (The 256 x 256 tile is a kernel of its own: sk_bf16_gemm256.hip.)  One work-group of 2 x 2
// waves owns a BM x BN tile; each wave a (BM/2) x (BN/2) sub-tile of 32x32 MFMA blocks.
// Operands go global -> registers -> LDS (double buffered, one barrier per 64-wide k chunk), or
// straight into a ring of chunks in LDS (sk_bf16_ring.h), and are read from LDS directly in the
// MFMA fragment layout; operands whose contiguous dimension is not k are read with
// the LDS transpose read.  Results leave straight from registers: fp32 as 16-byte
// pieces, bf16 in whole lines through a wave-private strip of LDS.
#include "sk_bf16_ring.h"
#include "sk_bf16_staged.h"
#include "sk_launch.h"

namespace sk {

// RING: the tile on a ring of chunks, for launches of one round.
template <int BM, int BN, bool A_KC, bool B_KC, typename OutT, bool COLSUM, bool RING = false>
__global__ __launch_bounds__(256) void gemm_bf16_kernel(const GemmArgs p) {
  typedef typename std::conditional<RING, RingTile<BM, BN, A_KC, B_KC, OutT, COLSUM>, GemmTile<BM, BN, A_KC, B_KC, OutT, COLSUM>>::type G;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[G::LDS_BYTES];
  G::run(p, blockIdx.x, smem);
}

// Whether a tile has a ring, for the launches of one round on which it is ahead.  Past a round two or more staged
// work-groups on a CU hide each other's waits as well, and a ring takes their room ([11752 x 3344] . [3344 x 2032] and the like on
// 128 x 128 rings in place of 256 x 256 tiles or staged ones: 4 to 10 % behind).  It is behind for bf16 results of 128 x 64
// ([4001 x 384] . [384 x 768] 9.8 : 8.5 us) and for 64 x 128 (dY . U^T of [4096 x 3072], R = 128, in four ranges 12.3 : 12.0).
template <int BM, int BN, typename OutT>
constexpr bool has_ring() { return BM == BN || (BM == 128 && sizeof(OutT) == 4); }

// Two independent GEMMs in one launch: the first `groups_a` work-groups run GA on `a`, the
// rest run GB on `b`.  For small problems a kernel's fixed cost (launch, first trip to
// memory, drain) is as large as its work, and two kernels that do not depend on each
// other can share it; the chip co-schedules both kinds of work-group on every CU.
template <class GA, class GB>
__global__ __launch_bounds__(256) void dual_gemm_kernel(const GemmArgs a, const GemmArgs b,
                                                        const int groups_a) {
  constexpr int BYTES = GA::LDS_BYTES > GB::LDS_BYTES ? GA::LDS_BYTES : GB::LDS_BYTES;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[BYTES];
  if ((int)blockIdx.x < groups_a) GA::run(a, blockIdx.x, smem);
  else GB::run(b, (int)blockIdx.x - groups_a, smem);
}

// Sums the split-K slabs in index order; see ReduceArgs.
// (One piece per thread and no bounds test inside the slab loop: as many work-groups as
// pieces allow matters more here than loads per thread.)
__global__ __launch_bounds__(256) void reduce_splits_kernel(const ReduceArgs p) {
  int64_t i4 = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  const float* __restrict__ part = p.part;
  float* __restrict__ out = p.out;
  int64_t n = p.n;
  float scale = p.scale;
  int splits = p.splits;
  if (i4 >= n) {  // second segment
    i4 -= n;
    part = p.part2; out = p.out2; n = p.n2; scale = p.scale2; splits = p.splits2;
    if (i4 >= n) return;
  }
  float4 s = sum_slabs(part + i4, n, splits);
  s.x *= scale; s.y *= scale; s.z *= scale; s.w *= scale;
  *reinterpret_cast<float4*>(out + i4) = s;
}

// Sum of split-K slabs in index order, rounded once to bf16 (an intermediate that the
// next GEMM reads as an operand).
// (`second` is for two products of one launch; the sum of one alone takes 0.3 us longer with it as an argument.)
__device__ __forceinline__ void reduce_to_bf16(const RoundedSum& p, int64_t i4) {
  const float4 s = sum_slabs(p.part + i4, p.n, p.splits);
  uint2 w;
  w.x = pack_bf16x2(s.x, s.y);
  w.y = pack_bf16x2(s.z, s.w);
  *reinterpret_cast<uint2*>(static_cast<bf16*>(p.out) + i4) = w;
}
__global__ __launch_bounds__(256) void reduce_to_bf16_kernel(const RoundedSum p) {
  const int64_t i4 = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i4 < p.n) reduce_to_bf16(p, i4);
}
__global__ __launch_bounds__(256) void reduce_two_to_bf16_kernel(const RoundedSum p, const RoundedSum second) {
  const int64_t i4 = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i4 < p.n) reduce_to_bf16(p, i4);
  else if (i4 - p.n < second.n) reduce_to_bf16(second, i4 - p.n);
}

// Up to three fp32 arrays, whole or in slabs, rounded to bf16, one behind the other over the work-groups.  Bound by the launch:
// 246 k numbers (a two-sided BERT-base layer's gradients) 2.7 us, through torch's fused copy 13.6.  The sums of their ranges here instead of
// ahead of it are two launches less of that layer's six backward.
__global__ __launch_bounds__(256) void round_gradients_kernel(const RoundArgs p) {
  int64_t i4 = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
#pragma unroll
  for (int s = 0; s < RoundArgs::MAX; ++s) {
    if (i4 < p.n[s]) {
      const float* const from = p.from[s] + i4;
      unsigned short* const to = p.to[s] + i4;
      if (i4 + 4 <= p.n[s]) {
        float4 v = sum_slabs(from, p.stride[s], p.splits[s]);
        v.x *= p.scale[s]; v.y *= p.scale[s]; v.z *= p.scale[s]; v.w *= p.scale[s];
        *reinterpret_cast<uint2*>(to) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
      } else {
        for (int e = 0; i4 + e < p.n[s]; ++e) to[e] = (unsigned short)pack_bf16x2(from[e] * p.scale[s], 0.f);
      }
      return;
    }
    i4 -= (p.n[s] + 3) / 4 * 4;
  }
}

template <typename OutT>
static std::string out_label() { return sizeof(OutT) == 2 ? "bf16" : "float"; }

template <int BM, int BN, bool A_KC, bool B_KC, typename OutT, bool COLSUM>
static hipError_t launch_cfg(GemmArgs a, hipStream_t s) {
  a.tiles_m = (a.M + BM - 1) / BM;
  a.tiles_n = (a.N + BN - 1) / BN;
  const long long total = (long long)a.tiles_m * a.tiles_n * a.splits;
  if (total <= 0 || total > 0x7fffffffLL || (A_KC && !within_window(BM, a.lda, BK, 2)) || (B_KC && !within_window(BN, a.ldb, BK, 2)))
    return hipErrorInvalidValue;
  note_gemm(a, A_KC, B_KC, 2, sizeof(OutT), sizeof(OutT) == 4);
  static const std::string name = kernel_label("gemm_bf16_kernel", {lbl(BM), lbl(BN), lbl(A_KC), lbl(B_KC), out_label<OutT>(), lbl(COLSUM)});
  const Work work = gemm_work(a, 2, sizeof(OutT), sizeof(OutT) == 4);
  if constexpr (has_ring<BM, BN, OutT>()) {
    if (total <= NUM_CUS * RingTile<BM, BN, A_KC, B_KC, OutT, COLSUM>::PER_CU) {
      static const std::string ring = kernel_label("gemm_bf16_kernel", {lbl(BM), lbl(BN), lbl(A_KC), lbl(B_KC), out_label<OutT>(), lbl(COLSUM), lbl(true)});
      return launch_kernel(ring.c_str(), work, gemm_bf16_kernel<BM, BN, A_KC, B_KC, OutT, COLSUM, true>, dim3((unsigned)total), dim3(256), s, a);
    }
  }
  return launch_kernel(name.c_str(), work, gemm_bf16_kernel<BM, BN, A_KC, B_KC, OutT, COLSUM>, dim3((unsigned)total), dim3(256), s, a);
}

// Tiles that have a ring only.
template <int BM, int BN, bool A_KC, bool B_KC>
static hipError_t launch_ring(GemmArgs a, hipStream_t s) {
  a.tiles_m = (a.M + BM - 1) / BM;
  a.tiles_n = (a.N + BN - 1) / BN;
  const long long total = (long long)a.tiles_m * a.tiles_n;
  if (a.splits != 1 || total <= 0 || total > 0x7fffffffLL || (A_KC && !within_window(BM, a.lda, BK, 2)) || (B_KC && !within_window(BN, a.ldb, BK, 2)))
    return hipErrorInvalidValue;
  note_gemm(a, A_KC, B_KC, 2, 2, false);
  static const std::string name = kernel_label("gemm_bf16_kernel", {lbl(BM), lbl(BN), lbl(A_KC), lbl(B_KC), "bf16", lbl(false), lbl(true)});
  return launch_kernel(name.c_str(), gemm_work(a, 2, 2, false), gemm_bf16_kernel<BM, BN, A_KC, B_KC, bf16, false, true>, dim3((unsigned)total), dim3(256), s, a);
}

template <bool A_KC, bool B_KC, typename OutT, bool COLSUM>
static hipError_t launch_tiles(int tile, const GemmArgs& a, hipStream_t s) {
  switch (tile) {
    case TILE_128x128: return launch_cfg<128, 128, A_KC, B_KC, OutT, COLSUM>(a, s);
    case TILE_128x64: return launch_cfg<128, 64, A_KC, B_KC, OutT, COLSUM>(a, s);
    case TILE_64x128: return launch_cfg<64, 128, A_KC, B_KC, OutT, COLSUM>(a, s);
    case TILE_64x64: return launch_cfg<64, 64, A_KC, B_KC, OutT, COLSUM>(a, s);
    default: return hipErrorInvalidValue;
  }
}

hipError_t launch_gemm_bf16(GemmKind kind, int tile, const GemmArgs& a, hipStream_t s) {
  if (tile == TILE_256x256) return launch_gemm256_bf16(kind, a, s);
  if (tile == TILE_256x128 && kind == GEMM_NN) return launch_ring<256, 128, true, false>(a, s);
  if (tile == TILE_256x128 && kind == GEMM_NT) return launch_ring<256, 128, true, true>(a, s);
  if (tile == TILE_256x128 && kind == GEMM_TN) return launch_ring<256, 128, false, false>(a, s);
  switch (kind) {
    case GEMM_NN: return launch_tiles<true, false, bf16, false>(tile, a, s);
    case GEMM_NT: return launch_tiles<true, true, bf16, false>(tile, a, s);
    case GEMM_TN_F32: return launch_tiles<false, false, float, true>(tile, a, s);
    case GEMM_TN_F32_PLAIN: return launch_tiles<false, false, float, false>(tile, a, s);
    case GEMM_NN_F32: return launch_tiles<true, false, float, false>(tile, a, s);
    case GEMM_TT: return launch_tiles<false, true, bf16, false>(tile, a, s);
    case GEMM_TN: return launch_tiles<false, false, bf16, false>(tile, a, s);
    case GEMM_NN_F32_COLSUM: return launch_tiles<true, false, float, true>(tile, a, s);
    case GEMM_NT_F32: return launch_tiles<true, true, float, false>(tile, a, s);
    case GEMM_TT_F32: return launch_tiles<false, true, float, false>(tile, a, s);
    default: return hipErrorInvalidValue;
  }
}

namespace {
typedef GemmTile<64, 64, true, true, bf16, false> NT_64x64;
typedef GemmTile<128, 64, true, true, bf16, false> NT_128x64;
typedef GemmTile<128, 128, true, true, bf16, false> NT_128x128;
typedef GemmTile<64, 64, true, true, float, false> NTF_64x64;
typedef GemmTile<64, 128, true, true, float, false> NTF_64x128;
typedef GemmTile<128, 128, true, true, float, false> NTF_128x128;
typedef GemmTile<64, 64, false, true, bf16, false> TT_64x64;
typedef GemmTile<128, 128, false, true, bf16, false> TT_128x128;
typedef GemmTile<64, 64, false, true, float, false> TTF_64x64;
typedef GemmTile<64, 128, false, true, float, false> TTF_64x128;
typedef GemmTile<128, 64, false, true, float, false> TTF_128x64;
typedef GemmTile<128, 128, false, true, float, false> TTF_128x128;
typedef GemmTile<128, 64, true, false, float, true> NNFC_128x64;
typedef GemmTile<128, 128, true, false, float, true> NNFC_128x128;
typedef RingTile<64, 64, true, true, bf16, false> RING_NT_64x64;
typedef RingTile<64, 64, true, true, float, false> RING_NTF_64x64;
typedef RingTile<64, 64, false, true, bf16, false> RING_TT_64x64;
typedef RingTile<64, 64, false, true, float, false> RING_TTF_64x64;

// The pairs of (kind, tile) the dual kernel is built for, the ones the backward pass's plans produce, with the kernel
// of each and, for those on 64 x 64 tiles, the one on rings.  The first should be the longer-running GEMM: its
// work-groups are dispatched first and the other's fill in beside them.
typedef void (*DualKernel)(GemmArgs, GemmArgs, int);
struct DualPair { GemmKind ka; int ta; GemmKind kb; int tb; DualKernel staged, ring; };
const DualPair kDualPairs[] = {
    // narrow sketch: R in 65..128, R <= 64; of a long input, Z^T in ranges as well
    {GEMM_NT_F32, TILE_64x128, GEMM_TT, TILE_64x64, dual_gemm_kernel<NTF_64x128, TT_64x64>, nullptr},
    {GEMM_NT_F32, TILE_64x64, GEMM_TT, TILE_64x64, dual_gemm_kernel<NTF_64x64, TT_64x64>, dual_gemm_kernel<RING_NTF_64x64, RING_TT_64x64>},
    {GEMM_NT_F32, TILE_64x64, GEMM_TT_F32, TILE_64x128, dual_gemm_kernel<NTF_64x64, TTF_64x128>, nullptr},
    {GEMM_NT_F32, TILE_64x128, GEMM_TT_F32, TILE_128x128, dual_gemm_kernel<NTF_64x128, TTF_128x128>, nullptr},
    {GEMM_NT_F32, TILE_64x128, GEMM_TT_F32, TILE_128x64, dual_gemm_kernel<NTF_64x128, TTF_128x64>, nullptr},
    // wide sketch, dY.U^T beside Z^T: both whole, the one, the other or both in ranges
    {GEMM_NT, TILE_128x128, GEMM_TT, TILE_128x128, dual_gemm_kernel<NT_128x128, TT_128x128>, nullptr},
    {GEMM_NT_F32, TILE_128x128, GEMM_TT, TILE_128x128, dual_gemm_kernel<NTF_128x128, TT_128x128>, nullptr},
    {GEMM_NT, TILE_128x128, GEMM_TT_F32, TILE_128x128, dual_gemm_kernel<NT_128x128, TTF_128x128>, nullptr},
    {GEMM_NT_F32, TILE_128x128, GEMM_TT_F32, TILE_128x128, dual_gemm_kernel<NTF_128x128, TTF_128x128>, nullptr},
    {GEMM_NT, TILE_64x64, GEMM_TT, TILE_64x64, dual_gemm_kernel<NT_64x64, TT_64x64>, dual_gemm_kernel<RING_NT_64x64, RING_TT_64x64>},
    {GEMM_NT, TILE_64x64, GEMM_TT_F32, TILE_64x64, dual_gemm_kernel<NT_64x64, TTF_64x64>, dual_gemm_kernel<RING_NT_64x64, RING_TTF_64x64>},
    {GEMM_NT_F32, TILE_64x64, GEMM_TT_F32, TILE_64x64, dual_gemm_kernel<NTF_64x64, TTF_64x64>, dual_gemm_kernel<RING_NTF_64x64, RING_TTF_64x64>},
    // wide sketch, Z^T.dY beside G.S^T
    {GEMM_NN_F32_COLSUM, TILE_128x64, GEMM_NT, TILE_128x128, dual_gemm_kernel<NNFC_128x64, NT_128x128>, nullptr},
    {GEMM_NN_F32_COLSUM, TILE_128x128, GEMM_NT, TILE_128x128, dual_gemm_kernel<NNFC_128x128, NT_128x128>, nullptr},
    {GEMM_NN_F32_COLSUM, TILE_128x64, GEMM_NT, TILE_128x64, dual_gemm_kernel<NNFC_128x64, NT_128x64>, nullptr},
    {GEMM_NN_F32_COLSUM, TILE_128x64, GEMM_NT, TILE_64x64, dual_gemm_kernel<NNFC_128x64, NT_64x64>, nullptr},
};
const DualPair* dual_pair(GemmKind ka, int ta, GemmKind kb, int tb) {
  for (const DualPair& p : kDualPairs)
    if (p.ka == ka && p.ta == ta && p.kb == kb && p.tb == tb) return &p;
  return nullptr;
}
}  // namespace

bool dual_gemm_supported(GemmKind kind_a, int tile_a, GemmKind kind_b, int tile_b) {
  return dual_pair(kind_a, tile_a, kind_b, tile_b) != nullptr;
}

hipError_t launch_dual_gemm_bf16(GemmKind kind_a, int tile_a, GemmArgs a, GemmKind kind_b, int tile_b,
                                 GemmArgs b, hipStream_t s) {
  const DualPair* const pair = dual_pair(kind_a, tile_a, kind_b, tile_b);
  if (pair == nullptr) return hipErrorInvalidValue;
  int bm, bn;
  tile_dims(tile_a, bm, bn);
  a.tiles_m = (a.M + bm - 1) / bm;
  a.tiles_n = (a.N + bn - 1) / bn;
  tile_dims(tile_b, bm, bn);
  b.tiles_m = (b.M + bm - 1) / bm;
  b.tiles_n = (b.N + bn - 1) / bn;
  const long long ga = (long long)a.tiles_m * a.tiles_n * a.splits;
  const long long gb = (long long)b.tiles_m * b.tiles_n * b.splits;
  if (ga <= 0 || gb <= 0 || ga + gb > 0x7fffffffLL) return hipErrorInvalidValue;
  const dim3 grid((unsigned)(ga + gb)), block(256);
  Work work;
  {
    bool akc, bkc, f32;
    gemm_kind_traits(kind_a, akc, bkc, f32);
    note_gemm(a, akc, bkc, 2, f32 ? 4 : 2, f32);
    work = gemm_work(a, 2, f32 ? 4 : 2, f32);
    gemm_kind_traits(kind_b, akc, bkc, f32);
    note_gemm(b, akc, bkc, 2, f32 ? 4 : 2, f32);
    const Work wb = gemm_work(b, 2, f32 ? 4 : 2, f32);
    work.flops += wb.flops;
    work.bytes += wb.bytes;
  }
  // 64 x 64 tiles in one round, two work-groups to a CU: on the ring, as a product by itself.  Backward pass, us, staged : ring,
  // narrow sketches: 2925 tokens, 1584 -> 2480, R = 64 29.6 : 26.6; 1024, 1024 -> 1024, R = 64 19.6 : 17.5; 2901, 304 -> 3824, R = 16 20.1 : 20.4;
  // wide ones: 1600, 2464 -> 1536, R = 256 30.6 : 25.3; 1507, 3120 -> 464, R = 512 36.9 : 31.6; 4096, 768 -> 768, R = 256 (512
  // work-groups) 24.5 : 23.5.  (On rings of their own the 128 x 64 and the 128 x 128 tiles of the other pairs are level with the staged
  // ones: 150 layers with the latter, 1.0000 of the time, 0.98 to 1.02.)
  const bool ring = pair->ring != nullptr && ga + gb <= NUM_CUS * RING_NT_64x64::PER_CU;
  return launch_kernel(ring ? "dual_gemm_kernel<ring>" : "dual_gemm_kernel", work, ring ? pair->ring : pair->staged, grid, block, s, a, b, (int)ga);
}

__global__ __launch_bounds__(256) void reduce_splits_2d_kernel(const float* __restrict__ part,
                                                               float* __restrict__ out, int rows, int cols,
                                                               int64_t ld_out, int splits, float scale) {
  const int c = (blockIdx.x * 256 + threadIdx.x) * 4;
  const int r = blockIdx.y;
  if (c >= cols) return;
  const int64_t n = (int64_t)rows * cols, at = (int64_t)r * cols + c;
  const float4 s = sum_slabs(part + at, n, splits);
  *reinterpret_cast<float4*>(out + (int64_t)r * ld_out + c) =
      make_float4(s.x * scale, s.y * scale, s.z * scale, s.w * scale);
}

hipError_t launch_reduce_splits_2d(const float* part, float* out, int rows, int cols, int64_t ld_out,
                                   int splits, float scale, hipStream_t s) {
  if (rows < 1 || rows > 65535 || cols < 4 || (cols & 3) != 0 || splits < 1) return hipErrorInvalidValue;
  const dim3 grid((unsigned)((cols / 4 + 255) / 256), (unsigned)rows);
  note_matrix(part, (int64_t)splits * rows, cols, cols, 4, false);
  note_matrix(out, rows, cols, ld_out, 4, true);
  return launch_kernel("reduce_splits_2d_kernel", Work{0.0, 4.0 * rows * cols * (splits + 1)}, reduce_splits_2d_kernel, grid, dim3(256), s, part, out, rows,
                       cols, ld_out, splits, scale);
}

hipError_t launch_reduce_to_bf16(const RoundedSum& a, const RoundedSum& b, hipStream_t s) {
  const int64_t groups = ((a.n + b.n) / 4 + 255) / 256;
  if (groups == 0) return hipSuccess;
  if (a.n < 0 || b.n < 0 || ((a.n | b.n) & 3) != 0 || (a.n > 0 && a.splits < 1) || (b.n > 0 && b.splits < 1) || groups > 0x7fffffffLL) return hipErrorInvalidValue;
  Work work{0.0, 0.0};
  for (const RoundedSum& r : {a, b}) {
    if (r.n == 0) continue;
    note_matrix(r.part, r.splits, r.n, r.n, 4, false);
    note_matrix(r.out, 1, r.n, r.n, 2, true);
    work.bytes += (double)r.n * (4.0 * r.splits + 2.0);
  }
  if (a.n > 0 && b.n > 0) return launch_kernel("reduce_two_to_bf16_kernel", work, reduce_two_to_bf16_kernel, dim3((unsigned)groups), dim3(256), s, a, b);
  return launch_kernel("reduce_to_bf16_kernel", work, reduce_to_bf16_kernel, dim3((unsigned)groups), dim3(256), s, a.n > 0 ? a : b);
}

hipError_t launch_reduce_splits(const ReduceArgs& a, hipStream_t s) {
  const int64_t groups = ((a.n + a.n2) / 4 + 255) / 256;
  if (groups <= 0) return hipSuccess;
  note_reduce(a);
  return launch_kernel("reduce_splits_kernel", reduce_work(a), reduce_splits_kernel, dim3((unsigned)groups), dim3(256), s, a);
}

hipError_t launch_round_gradients(const RoundArgs& a, hipStream_t s) {
  int64_t pieces = 0;
  Work work{0.0, 0.0};
  for (int i = 0; i < RoundArgs::MAX; ++i) {
    if (a.n[i] == 0) continue;
    if (a.n[i] < 0 || a.splits[i] < 1 || (a.splits[i] > 1 && (a.n[i] & 3) != 0)) return hipErrorInvalidValue;
    pieces += (a.n[i] + 3) / 4;
    note_matrix(a.from[i], a.splits[i], a.n[i], a.stride[i], 4, false);
    note_matrix(a.to[i], 1, a.n[i], a.n[i], 2, true);
    work.bytes += (double)a.n[i] * (4.0 * a.splits[i] + 2.0);
  }
  const int64_t groups = (pieces + 255) / 256;
  if (groups <= 0) return hipSuccess;
  if (groups > 0x7fffffffLL) return hipErrorInvalidValue;
  return launch_kernel("round_gradients_kernel", work, round_gradients_kernel, dim3((unsigned)groups), dim3(256), s, a);
}

}  // namespace sk

// bf16 matrix products of the decoder stage: the kernels, the choice of a tile form and the checks of arguments.  The tiles, their
// pipelines and epilogues are in gemm_core.h.
#include "gemm_core.h"

namespace {

template <int BM, int BN, int BK, int NS, int NW, int WPE, bool AKM, bool BKM, int EPI>
__global__ __launch_bounds__(64 * NW, WPE) void gemm_dtl_kernel(const uint16_t* __restrict__ A, int64_t lda, int64_t a_bs,
                                                                 const uint16_t* __restrict__ B, int64_t ldb, int64_t b_bs,
                                                                 int M, int N, int K, int tiles_m, int tiles_n,
                                                                 int band_rows, Epi e) {
  int bm, bn;
  tile_of_block(tiles_m, tiles_n, band_rows, bm, bn);
  gemm_dtl_body<BM, BN, BK, NS, NW, AKM, BKM, EPI>(A, lda, a_bs, B, ldb, b_bs, M, N, K, bm, bn, e);
}

template <int BM, int BN, int G, int NW, int NS, bool AKM, bool BKM, int EPI>
__global__ __launch_bounds__(64 * NW * G, NW * G / 4) void gemm_split_kernel(const uint16_t* __restrict__ A, int64_t lda, int64_t a_bs,
                                                                const uint16_t* __restrict__ B, int64_t ldb, int64_t b_bs, int M, int N, int K,
                                                                int tiles_m, int tiles_n, Epi e) {
  int ks, bm, bn;
  split_tile(tiles_m, tiles_n, 1, ks, bm, bn);
  gemm_split_body<BM, BN, G, NW, NS, AKM, BKM, EPI>(A, lda, a_bs, B, ldb, b_bs, M, N, K, bm, bn, e);
}

// ---- few tiles and a long contraction: split over workgroups as well ------------------------
// A product of so few tiles that most CUs have none is cut into S stretches of k-tiles, a workgroup to each tile of each: every
// one stores its sum as fp32 to part[stretch][M][N], and the kernel that reads the result - a LayerNorm, which passes over
// whole rows anyway - adds the S of them in order (norm.hip): no exchange between workgroups, no launch of its own.
template <int BM, int BN, int G, int NW, int NS, bool BKM>
__global__ __launch_bounds__(64 * NW * G, NW * G / 4) void gemm_part_kernel(const uint16_t* __restrict__ A, int64_t lda, int64_t a_bs,
                                                               const uint16_t* __restrict__ B, int64_t ldb, int64_t b_bs, int M, int N, int K,
                                                               int tiles_m, int tiles_n, int S, float* part) {
  int ks, bm, bn;
  split_tile(tiles_m, tiles_n, S, ks, bm, bn);
  const int nk = K / 32, t0 = nk * ks / S, t1 = nk * (ks + 1) / S;
  Epi e{part + (int64_t)ks * M * N, N, nullptr, nullptr, nullptr, 0, nullptr, nullptr, 0.f, nullptr, 0, 0};
  gemm_split_body<BM, BN, G, NW, NS, false, BKM, EPI_F32>(A + t0 * a_bs, lda, a_bs, B + t0 * (BKM ? 32 * ldb : b_bs), ldb, b_bs,
                                                          M, N, (t1 - t0) * 32, bm, bn, e);
}

// Several independent products of one kind in a single launch (the four weight-gradient
// products of a decoder block): a workgroup finds its problem from the running tile count.
// One launch fills the chip where four small grids would each leave most CUs idle.
struct GroupedProblem {
  const uint16_t* A; const uint16_t* B; float* out;
  float* upd_w; uint16_t* upd_ver; float eta;
  int lda, a_bs, ldb, b_bs, ldo, ldv, bsv, M, N, K, tiles_m, tiles_n, first_tile;   // ldv, bsv: of the weight version
};
template <int MAX>
struct GroupedArgs {
  GroupedProblem p[MAX];
  int count;
};

// the problem, tile row and tile column of a workgroup
template <int MAX>
__device__ __forceinline__ const GroupedProblem& grouped_tile(const GroupedArgs<MAX>& ga, int& bm, int& bn) {
  // Workgroup ids are dealt to the 8 XCDs in turn, and each XCD pulls its operand panels
  // through its own L2.  Give XCD g a CONTIGUOUS range of the tile numbering (so it works on
  // one problem at a time, not on a slice of all of them) and number a problem's tiles in bands
  // of two tile rows, column by column (so a run of 8 tiles is a 2 x 4 patch: 6 operand panels).
  const int total = gridDim.x, base = total / 8, rem = total % 8;
  const int g = blockIdx.x % 8, i = blockIdx.x / 8;
  const int v = g * base + (g < rem ? g : rem) + i;
  int pi = 0;
#pragma unroll
  for (int k = 1; k < MAX; ++k)
    if (k < ga.count && v >= ga.p[k].first_tile) pi = k;
  const GroupedProblem& q = ga.p[pi];
  const int local = v - q.first_tile;
  constexpr int GB = 2;
  const int band = local / (GB * q.tiles_n), first_row = band * GB;
  const int rows = q.tiles_m - first_row < GB ? q.tiles_m - first_row : GB;
  const int in = local - band * GB * q.tiles_n;
  bm = first_row + in % rows;
  bn = in / rows;
  return q;
}
__device__ __forceinline__ Epi grouped_epi(const GroupedProblem& q) {
  return Epi{q.out, q.ldo, q.upd_ver, nullptr, nullptr, 0, nullptr, q.upd_w, q.eta, nullptr, q.ldv, q.bsv};
}

template <int BM, int BN, int BK, int NS, int NW, int WPE>
__global__ __launch_bounds__(64 * NW, WPE) void gemm_dtl_grouped_wgrad_kernel(GroupedArgs<RV_GEMM_GROUP_BLOCK> ga) {
  int bm, bn;
  const GroupedProblem& q = grouped_tile(ga, bm, bn);
  gemm_dtl_body<BM, BN, BK, NS, NW, true, true, EPI_F32_UPD>(q.A, q.lda, q.a_bs, q.B, q.ldb, q.b_bs, q.M, q.N, q.K, bm, bn, grouped_epi(q));
}
template <int BM, int BN, int G, int NW, int NS, int MAX>
__global__ __launch_bounds__(64 * NW * G, NW * G / 4) void gemm_split_grouped_wgrad_kernel(GroupedArgs<MAX> ga) {
  int bm, bn;
  const GroupedProblem& q = grouped_tile(ga, bm, bn);
  gemm_split_body<BM, BN, G, NW, NS, true, true, EPI_F32_UPD>(q.A, q.lda, q.a_bs, q.B, q.ldb, q.b_bs, q.M, q.N, q.K, bm, bn, grouped_epi(q));
}

template <int BM, int BN, int BK, int NS, int NW, int WPE, bool AKM, bool BKM, int EPI>
rv_status launch_dtl(const rv_gemm_args& g, hipStream_t st) {
  constexpr int ring = NS * (dtl_tile_bytes(BM, BK) + dtl_tile_bytes(BN, BK));
  // the GELU' epilogue keeps two rows of fp32 column sums (one per wave row) behind the image
  constexpr int image = staged_epi(EPI) ? BM * stage_pitch(BN) + (EPI == EPI_BF16_DGELU ? 2 * BN * 4 : 0)
                        : (epi_has_resid(EPI) && NW == 8 && BM == 256 && BN == 256 ? upd_image_bytes(BM, BN) : 0);
  constexpr int smem = ring > image ? ring : image;
  auto kern = gemm_dtl_kernel<BM, BN, BK, NS, NW, WPE, AKM, BKM, EPI>;
  // once per instantiation; a function-local static is initialised exactly once, also under threads
  static const hipError_t configured =
      hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (configured != hipSuccess) return RV_E_DEVICE;
  int tm = (g.M + BM - 1) / BM, tn = (g.N + BN - 1) / BN;
  Epi e{g.out, g.ldo, g.out2, g.bias, g.resid, g.ldr, g.zin, nullptr, 0.f, g.epi == EPI_BF16_DGELU ? g.colpart : nullptr,
        g.bsv ? 32 : g.ldo, g.bsv ? g.bsv : 32};
  g.colpart_rows = (g.M + BM - 1) / BM;
  const int ntiles = tm * tn;
  // Measured: alone, the XCD-banded map pays only for the small tile.  Inside a stage step a
  // launch holds about a third of every XCD's CUs, and what an XCD runs of it at one time should
  // share operand panels: bands of 8 tile rows (2 for 32 or more tile rows, either tile size)
  // against the natural order: stage steps -1.3 % / -0.6 % / -1.9 % (d 1600 / 2048 / 1024).
  int band = 8;
  if (g.sharing != 0) band = tm >= 32 ? 2 : 8;
  else if (!(BM == 128 && BN == 128)) tm = -tm;
  hipLaunchKernelGGL(kern, dim3(ntiles), dim3(64 * NW), smem, st, g.A, g.lda, g.a_bs, g.B, g.ldb, g.b_bs, g.M, g.N, g.K,
                     tm, tn, band, e);
  return rv_launch_status();
}

template <int BM, int BN, int G, int NW, int NS, bool AKM, bool BKM, int EPI>
rv_status launch_split(const rv_gemm_args& g, hipStream_t st) {
  constexpr int smem = split_lds<BM, BN, G, NS>();
  static_assert(smem <= 160 * 1024, "LDS of one CU");
  auto kern = gemm_split_kernel<BM, BN, G, NW, NS, AKM, BKM, EPI>;
  static const hipError_t configured =
      hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (configured != hipSuccess) return RV_E_DEVICE;
  const int tm = (g.M + BM - 1) / BM, tn = (g.N + BN - 1) / BN;
  Epi e{g.out, g.ldo, g.out2, g.bias, g.resid, g.ldr, g.zin, nullptr, 0.f, g.epi == EPI_BF16_DGELU ? g.colpart : nullptr,
        g.bsv ? 32 : g.ldo, g.bsv ? g.bsv : 32};
  g.colpart_rows = tm;
  hipLaunchKernelGGL(kern, dim3(tm * tn), dim3(64 * NW * G), smem, st, g.A, g.lda, g.a_bs, g.B, g.ldb, g.b_bs, g.M, g.N, g.K, tm, tn, e);
  return rv_launch_status();
}

template <int BM, int BN, int G, int NW, int NS, bool BKM>
rv_status launch_part(const rv_gemm_args& g, int S, float* part, hipStream_t st) {
  constexpr int smem = split_lds<BM, BN, G, NS>();
  static_assert(smem <= 160 * 1024, "LDS of one CU");
  auto kern = gemm_part_kernel<BM, BN, G, NW, NS, BKM>;
  static const hipError_t configured =
      hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (configured != hipSuccess) return RV_E_DEVICE;
  const int tm = (g.M + BM - 1) / BM, tn = (g.N + BN - 1) / BN;
  hipLaunchKernelGGL(kern, dim3(tm * tn * S), dim3(64 * NW * G), smem, st, g.A, g.lda, g.a_bs, g.B, g.ldb, g.b_bs, g.M, g.N, g.K, tm, tn, S, part);
  return rv_launch_status();
}
template <bool BKM>
rv_status pick_part(const rv_gemm_args& g, int S, float* part, hipStream_t st) {
  switch (g.tile) {
    case 1032: return launch_part<32, 64, 8, 2, 3, BKM>(g, S, part, st);
    case 1064: return launch_part<64, 64, 4, 4, 4, BKM>(g, S, part, st);
    case 1065: return launch_part<64, 64, 2, 4, 4, BKM>(g, S, part, st);
    case 1128: return launch_part<128, 128, 2, 4, 4, BKM>(g, S, part, st);
  }
  return RV_E_INVAL;
}

// Tile choice (codes: 5256, 2256, 2192, 2128, 1128, 1065, 1064, 1032).
//   5256  256x256, eight waves of 128x64, BK 32, ring of four slots run in the pipelined form
//         (three tiles in flight, loads dealt out behind the MFMAs), one workgroup per CU:
//         lowest LDS traffic per MFMA, two waves per SIMD cover each other's stalls;
//   2192  128x256, four waves of 64x128, ring of three slots, two workgroups per CU;
//   2128  128x128, four waves of 64x64, ring of four slots, two workgroups per CU;
//   1128  128x128, 1065 / 1064 64x64, 1032 32x64: the contraction split inside the workgroup over
//         2, 2 / 4 and 8 groups of waves.
// The automatic choice among the first three minimises  rounds * tile area * workgroups per CU / efficiency,
// rounds = ceil(tiles / (256 CUs * workgroups per CU)), efficiencies ratios of times before 2192 and 2128 had
// the pipelined ring, 2192's 0.92 -> 0.98 with it (us, bound loads / ring: 4096x1024x4096 2128 43.7 / 38.0, 4096x6144x2048 2192 116 / 98,
// 8192x1600x6400 2192 189 / 154; 5256 75, 103, 150).  Over 200 launches of 512 .. 8192 rows and 256 .. 8192 in k alone on average 2.1 % above
// the best of the three (0.3 % before the ring; 3.0 % from 64 tiles of 256x256 on), most on short contractions: 6784x7552x256 with GELU 91 where
// 2128 takes 69, 5120x6848x1024 85 / 72 (2192).
// Whether the contraction is split is decided by the modelled time, us,
//   rounds * (f + turns * t) + out * M N / 1e6,  turns = k-tiles per group,
// t between t0 (a launch that leaves most CUs idle) and t1 (one that fills them; with 2192 and 2128 as they were before the pipelined ring:
// with 0.88 of their times four microbatches of 6 blocks of d 768, 1152 tokens take 0.2 - 0.5 % longer), fitted to 488 launches of 64 .. 8192 rows
// alone, operands in blocks of columns, weights cold.  A product of few tiles is one walk along K: 256x448x1792 takes 43 us
// with 5256, 22 with 2128 and 7 with 1032; 512x4096x1024 with GELU' 32 / 17 / 11 (1065); 1152x768x3072 65 / 36 / 14 (1064);
// 1152x2048x8192 152 / 108 / 72 (1128); 2048x1024x4096 82 / 44 / 29 (1065); 8192x6400x1600 183 / 204 / 261.
// A split form is taken where the model has it a tenth faster, on the shape alone, so that a product has the same bits beside
// other streams as by itself; and not from 64 tiles of 256x256 on: it takes more CU time per flop, which the other streams
// of a step could have used.  Stage steps, split where a tenth faster / not from 64 tiles on / nowhere, us:
//   4 blocks d 1024, 4096 tokens 1762 / 1718 / 1714    6 blocks d 768, 1152 tokens, 4 microbatches 4847 / 4850 / 5260
//   8 blocks d 832, 2048 tokens  1535 / 1443           9 blocks d 896, 4032 tokens (64 tiles)     3382 / 3520
//   12 blocks d 640, 2880 tokens 2230 / - / 2400       7 blocks d 1536, 1536 tokens, 2 microbatches 5890 / - / 6230
struct TileForm { int code, bm, bn, k, per_cu; float f, t0, t1, out; };
constexpr TileForm kForms[] = {
    {5256, 256, 256, 32, 1, 8.9f, 0.51f, 0.64f, 0.63f}, {2192, 128, 256, 32, 2, 6.1f, 0.45f, 0.77f, 0.66f},
    {2128, 128, 128, 64, 2, 3.1f, 0.65f, 0.91f, 0.77f}, {1128, 128, 128, 64, 1, 4.3f, 0.47f, 0.48f, 0.68f},
    {1065, 64, 64, 64, 2, 3.1f, 0.27f, 0.37f, 0.50f},   {1064, 64, 64, 128, 1, 3.9f, 0.43f, 0.40f, 0.11f},
    {1032, 32, 64, 256, 1, 3.3f, 0.66f, 0.57f, 0.f}};
// the modelled time of a form whose contraction is cut into S stretches
float form_time(const TileForm& c, int M, int N, int K, int S) {
  const float tiles = (float)((M + c.bm - 1) / c.bm) * ((N + c.bn - 1) / c.bn) * S, slots = 256.f * c.per_cu;
  const float fill = tiles < slots ? tiles / slots : 1.f;
  return ceilf(tiles / slots) * (c.f + ceilf((float)K / S / c.k) * (c.t0 + (c.t1 - c.t0) * fill * fill)) + c.out * 1e-6f * M * N * S;
}
int in_order_form(int M, int N) {
  auto cost = [&](int bm, int bn, int bpc, double eff) {
    const long tiles = (long)((M + bm - 1) / bm) * ((N + bn - 1) / bn);
    return (double)((tiles + 256 * bpc - 1) / (256 * bpc)) * bm * bn * bpc / eff;
  };
  const double c256 = cost(256, 256, 1, 1.0), c192 = cost(128, 256, 2, 0.98), c128 = cost(128, 128, 2, 0.83);
  return c256 <= c192 && c256 <= c128 ? 5256 : c192 <= c128 ? 2192 : 2128;
}
// the form of a whole product where nobody shares the chip, and its modelled time (k32: form 1032 is there)
int whole_form(int M, int N, int K, bool k32, float& time) {
  int best = in_order_form(M, N);
  for (const TileForm& c : kForms)
    if (c.code == best) time = form_time(c, M, N, K, 1);
  if (((M + 255) / 256) * ((N + 255) / 256) >= 64) return best;
  float least = 0.9f * time;
  for (const TileForm& c : kForms) {
    if (c.code >= 2000 || (c.code == 1032 && !k32)) continue;
    const float t = form_time(c, M, N, K, 1);
    if (t < least) { best = c.code; least = time = t; }
  }
  return best;
}

template <bool AKM, bool BKM, int EPI>
rv_status pick_tile(const rv_gemm_args& g, hipStream_t st) {
  int tile = g.tile;
  if (tile == 0) {
    float time;   // (whether the contraction is split: by the shape alone)
    tile = whole_form(g.M, g.N, g.K, !AKM, time);
    const long t256 = (long)((g.M + 255) / 256) * ((g.N + 255) / 256);
    // Measured inside the stage step (d = 1024, 1600, 2048): what a launch leaves of the chip is
    // used by the other streams, so CU time per flop counts for more than its own duration.
    if (tile >= 2000 && (g.sharing == 2 || (g.sharing && t256 >= 128))) tile = 5256;
  }
  if constexpr (!AKM) {
    if (tile == 1032) return launch_split<32, 64, 8, 2, 3, AKM, BKM, EPI>(g, st);
  }
  if (tile == 1064) return launch_split<64, 64, 4, 4, 4, AKM, BKM, EPI>(g, st);
  if (tile == 1065) return launch_split<64, 64, 2, 4, 4, AKM, BKM, EPI>(g, st);
  if (tile == 1128) return launch_split<128, 128, 2, 4, 4, AKM, BKM, EPI>(g, st);
  if (tile == 2256) return launch_dtl<256, 256, 32, 4, 4, 1, AKM, BKM, EPI>(g, st);
  if (tile == 2192) return launch_dtl<128, 256, 32, 3, 4, 2, AKM, BKM, EPI>(g, st);
  if (tile == 2128) return launch_dtl<128, 128, 32, 4, 4, 2, AKM, BKM, EPI>(g, st);
  if (tile == 5256) return launch_dtl<256, 256, 32, 4, 8, 2, AKM, BKM, EPI>(g, st);
  return RV_E_INVAL;
}

}  // namespace

namespace {
// tile offsets are kept in 32 bits, and a matrix in blocks of columns is whole blocks
bool operand_fits(const rv_gemm_args& g) {
  auto fits = [](int64_t rows, int64_t cols, int64_t ld, int64_t bs) {
    if (bs == 32) return rows * ld < (1ll << 31);
    return ld == 32 && bs == rows * 32 && cols % 32 == 0 && rows * cols < (1ll << 31);
  };
  return (g.a_kmajor ? fits(g.K, g.M, g.lda, g.a_bs) : fits(g.M, g.K, g.lda, g.a_bs)) &&
         (g.b_kmajor ? fits(g.K, g.N, g.ldb, g.b_bs) : fits(g.N, g.K, g.ldb, g.b_bs)) &&
         (!g.bsv || (g.bsv == (int64_t)g.M * 32 && g.N % 32 == 0 && (int64_t)g.M * g.N < (1ll << 31)));
}
}  // namespace

rv_status rv_gemm_bf16(const rv_gemm_args& g, hipStream_t st) {
  if (!g.A || !g.B || !g.out || g.M < 8 || g.N < 8 || g.K < 64) return RV_E_INVAL;
  if (g.K % 64 || g.N % 8 || g.M % 8 || g.lda % 8 || g.ldb % 8 || g.ldo % 4) return RV_E_INVAL;
  if ((((uintptr_t)g.A) | ((uintptr_t)g.B) | ((uintptr_t)g.out)) & 15) return RV_E_INVAL;
  // bf16 outputs (and the pre-activation input of GELU') move in 16-byte row pieces: pitch % 8
  if ((staged_epi(g.epi) || g.epi == EPI_F32_BIAS_RESID_BF16) && g.ldo % 8) return RV_E_INVAL;
  if (staged_epi(g.epi) && g.epi == EPI_BF16_BIAS_GELU && (((uintptr_t)g.out2) & 15)) return RV_E_INVAL;
  if (g.epi == EPI_BF16_DGELU && (((uintptr_t)g.zin) & 15)) return RV_E_INVAL;
  if (!operand_fits(g)) return RV_E_INVAL;
  const bool need_bias = g.epi == EPI_BF16_BIAS || g.epi == EPI_F32_BIAS_RESID ||
                         g.epi == EPI_BF16_BIAS_GELU || g.epi == EPI_F32_BIAS_RESID_BF16;
  if (need_bias && (!g.bias || (((uintptr_t)g.bias) & 7))) return RV_E_INVAL;
  if ((g.epi == EPI_F32_BIAS_RESID || g.epi == EPI_F32_BIAS_RESID_BF16) &&
      (!g.resid || g.ldr % 4 || (((uintptr_t)g.resid) & 15)))
    return RV_E_INVAL;
  if ((g.epi == EPI_BF16_BIAS_GELU || g.epi == EPI_F32_BIAS_RESID_BF16) && !g.out2) return RV_E_INVAL;
  if (g.epi == EPI_BF16_DGELU && !g.zin) return RV_E_INVAL;
  // only the layout/epilogue pairs the stage uses are instantiated
  if (!g.a_kmajor && g.b_kmajor) {          // forward products
    switch (g.epi) {
      case EPI_BF16_BIAS: return pick_tile<false, true, EPI_BF16_BIAS>(g, st);
      case EPI_F32_BIAS_RESID: return pick_tile<false, true, EPI_F32_BIAS_RESID>(g, st);
      case EPI_F32_BIAS_RESID_BF16: return pick_tile<false, true, EPI_F32_BIAS_RESID_BF16>(g, st);
      case EPI_BF16_BIAS_GELU: return pick_tile<false, true, EPI_BF16_BIAS_GELU>(g, st);
    }
  } else if (!g.a_kmajor && !g.b_kmajor) {  // input-gradient products
    switch (g.epi) {
      case EPI_BF16: return pick_tile<false, false, EPI_BF16>(g, st);
      case EPI_BF16_DGELU: return pick_tile<false, false, EPI_BF16_DGELU>(g, st);
    }
  } else if (g.a_kmajor && g.b_kmajor) {    // weight-gradient products
    if (g.epi == EPI_F32) return pick_tile<true, true, EPI_F32>(g, st);
  }
  return RV_E_INVAL;
}

// The form and the number of stretches of a product whose partial sums the next kernel can add: the least modelled time,
// with 4 bytes per partial sum read back at 5 TB/s, if that takes a tenth off the best whole product; S = 1: none does.
// Weights cold, best whole form / cut (with the reading back), us: 64x2048x8192 30.1 / 11.3 (64x64 tiles, S 8), 128x1024x4096
// 11.6 / 7.1 (32x64, 4), 1024x2048x8192 66.9 / 46.0 (128x128, 2), 1152x1600x6400 50.2 / 35.7,
// 256x448x1792 7.2 / 5.9.  Over 130 products of 64 .. 2048 rows the modelled ratio is below the measured one by 0.1 .. 0.2 on the
// short walks and above it by as much on the long ones; a modelled tenth was 0 .. 30 % measured.
// Four stages of 4 blocks of d 1024 on 128 tokens, forward and backward, with their average 3137 -> 2761 us, stage step of 12
// blocks of d 448 on 256 tokens 924 -> 852 us (with what split_tile and the early requests give).
// Not from 64 tiles of 256x256 on, as with the split forms of whole products.  Stage steps, cut / whole, us: 4 blocks d 2048, 2048 tokens
// 3367 / 3069, 2 of d 4096, 4608 tokens 11080 / 9200 (separate calls 11530 / 10910), 3 of d 4096, 1024 tokens 4537 / 4262 (separate
// calls 4853 / 5017: the one form that loses).  Below, cut against the forms without: 4 of d 2048, 1024 tokens 2100 / 2550, of
// d 1600, 2048 tokens (56 tiles) 2170 / 2344, of d 1024, 3072 tokens (48) 1390 / 1513.
rv_part_form rv_gemm_part_form(int M, int N, int K) {
  float whole;
  whole_form(M, N, K, true, whole);
  rv_part_form best = {0, 1};
  if (((M + 255) / 256) * ((N + 255) / 256) >= 64) return best;
  float least = 0.9f * whole;
  for (const TileForm& c : kForms) {
    if (c.code >= 2000) continue;
    for (int S = 2; S <= RV_GEMM_PARTS_MAX && S * c.k <= K; S *= 2) {
      const float time = form_time(c, M, N, K, S) + (float)M * N * S * 4.f / 5e6f;   // (written: in the form's own time)
      if (time < least) { least = time; best = {c.code, S}; }
    }
  }
  return best;
}

// the product's operands as in g (a_kmajor 0), its sums over S stretches of the contraction to part[S][M][N]
rv_status rv_gemm_part(const rv_gemm_args& g, int S, float* part, hipStream_t st) {
  if (!g.A || !g.B || !part || g.a_kmajor || g.M < 8 || g.N < 8 || g.K < 64 || S < 1 || S > RV_GEMM_PARTS_MAX || S > g.K / 32) return RV_E_INVAL;
  if (g.K % 64 || g.N % 8 || g.M % 8 || g.lda % 8 || g.ldb % 8) return RV_E_INVAL;
  if ((((uintptr_t)g.A) | ((uintptr_t)g.B) | ((uintptr_t)part)) & 15) return RV_E_INVAL;
  if (!operand_fits(g)) return RV_E_INVAL;
  return g.b_kmajor ? pick_part<true>(g, S, part, st) : pick_part<false>(g, S, part, st);
}

namespace {
template <int MAX>
rv_status launch_grouped(void (*kern)(GroupedArgs<MAX>), int BM, int BN, int threads, int smem, const rv_gemm_args* gs, int count,
                         hipStream_t st) {
  GroupedArgs<MAX> ga;
  int tiles = 0;
  for (int k = 0; k < count; ++k) {
    const rv_gemm_args& g = gs[k];
    GroupedProblem& q = ga.p[k];
    q.A = g.A; q.B = g.B; q.out = g.store_out ? (float*)g.out : nullptr;
    q.upd_w = g.upd_w; q.upd_ver = g.upd_ver; q.eta = g.upd_eta;
    q.lda = (int)g.lda; q.a_bs = (int)g.a_bs; q.ldb = (int)g.ldb; q.b_bs = (int)g.b_bs; q.ldo = (int)g.ldo;
    q.ldv = (int)(g.bsv ? 32 : g.ldo); q.bsv = (int)(g.bsv ? g.bsv : 32);
    q.M = g.M; q.N = g.N; q.K = g.K;
    q.tiles_m = (g.M + BM - 1) / BM;
    q.tiles_n = (g.N + BN - 1) / BN;
    q.first_tile = tiles;
    tiles += q.tiles_m * q.tiles_n;
  }
  for (int k = count; k < MAX; ++k) ga.p[k] = ga.p[0];
  ga.count = count;
  hipLaunchKernelGGL(kern, dim3(tiles), dim3(threads), smem, st, ga);
  return rv_launch_status();
}
template <int BM, int BN, int BK, int NS, int NW>
rv_status launch_grouped_dtl(const rv_gemm_args* gs, int count, hipStream_t st) {
  constexpr int ring = NS * (dtl_tile_bytes(BM, BK) + dtl_tile_bytes(BN, BK));
  constexpr int smem = ring > upd_image_bytes(BM, BN) ? ring : upd_image_bytes(BM, BN);
  static_assert(smem <= 160 * 1024, "LDS of one CU");
  auto kern = gemm_dtl_grouped_wgrad_kernel<BM, BN, BK, NS, NW, 2>;
  static const hipError_t configured =
      hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (configured != hipSuccess) return RV_E_DEVICE;
  return launch_grouped(kern, BM, BN, 64 * NW, smem, gs, count, st);
}
template <int BM, int BN, int G, int NW, int NS, int MAX>
rv_status launch_grouped_split(const rv_gemm_args* gs, int count, hipStream_t st) {
  constexpr int smem = split_lds<BM, BN, G, NS>();
  static_assert(smem <= 160 * 1024, "LDS of one CU");
  auto kern = gemm_split_grouped_wgrad_kernel<BM, BN, G, NW, NS, MAX>;
  static const hipError_t configured =
      hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (configured != hipSuccess) return RV_E_DEVICE;
  return launch_grouped(kern, BM, BN, 64 * NW * G, smem, gs, count, st);
}
}  // namespace

namespace {
int tiles_of(int count, const int* M, const int* N, int edge) {
  int tiles = 0;
  for (int k = 0; k < count; ++k) tiles += ((M[k] + edge - 1) / edge) * ((N[k] + edge - 1) / edge);
  return tiles;
}
}  // namespace

// 256x256 tiles, eight waves (measured against 128x128 and 128x256 tiles, alone and inside the
// stage step of d 1024, 2048 and 1600: fewest LDS bytes per MFMA, so it takes the least CU time
// from the kernels that run beside it, and the step is 3-4 % shorter)
// A block whose 256x256 tiles do not cover the chip and whose walk along the tokens is short takes
// 128x128 tiles with the walk split in two, four times as many: 24 -> 12 us (d 448, ffn 1792, 256
// tokens, 44 tiles), 37 -> 34 us (768, 3072, 1152 tokens, 108); even at 30 us with 128 tokens of a
// 1024-wide block, where the update's 126 MB bound it.  Longer walks keep the CU time per flop down: stage steps of
// four blocks, ms, split / in order (the separate calls differ the same way):
//   tokens           512          1024         1536         2048         3072         4096
//   d 1024   0.710/0.732  0.870/0.876  1.090/1.074  1.240/1.220  1.584/1.535  1.979/1.881
//   d 768    0.514/0.520  0.656/0.651  0.772/0.786  0.917/0.904  1.156/1.095  1.377/1.357
//   d 448    0.390/0.410  0.425/0.443  0.486/0.496  0.531/0.568  0.669/0.690  0.786/0.818
// From RV_WGRAD_SPLIT_K tokens on the split form where the model of the forms has the whole block a quarter faster: that is a narrow
// one, whose 256x256 tiles are a tenth of the chip.  Stage steps, in order / split, us: d 128, 4032 tokens 726 / 539; d 320, 6272 tokens 2266 /
// 2000; d 256, 2688 tokens 1226 / 1164; d 448, 4160 tokens, four microbatches in separate calls 4340 / 3915; the one
// seen to lose, d 384 on 3584 tokens in separate calls, 2443 / 2500.
// Asked for the four products of a block together, however many launches they leave in (the few tiles that a wide block sends by
// themselves share the chip with the others: dWo of d 1600, 8192 tokens, 49 tiles, split 11 ms of CU time, in order 7; stage step
// 21.53 / 21.43 and, another run, 21.39 / 21.37 ms),
// and for what leaves last by itself, with nothing behind it to share the chip (decoder.hip).
rv_wgrad_form rv_gemm_wgrad_form(int count, const int* M, const int* N, int K) {
  const int tiles = tiles_of(count, M, N, 256), small = tiles_of(count, M, N, 128);
  const float whole = ceilf(tiles / 256.f) * (8.9f + K / 32 * 0.55f), split = ceilf(small / 256.f) * (4.3f + K / 64 * 0.48f);
  return tiles < 256 && (K < RV_WGRAD_SPLIT_K || split < 0.75f * whole) ? RV_WGRAD_SPLIT : RV_WGRAD_IN_ORDER;
}

rv_status rv_gemm_wgrad_grouped(const rv_gemm_args* gs, int count, hipStream_t st, rv_wgrad_form form) {
  if (!gs || count < 1 || count > (form == RV_WGRAD_SPLIT ? RV_GEMM_GROUP_MAX : RV_GEMM_GROUP_BLOCK)) return RV_E_INVAL;
  for (int k = 0; k < count; ++k) {
    const rv_gemm_args& g = gs[k];
    if (!g.A || !g.B || !g.out || !g.a_kmajor || !g.b_kmajor || g.epi != EPI_F32) return RV_E_INVAL;
    if (g.M < 8 || g.N < 8 || g.K < 64 || g.K % 64 || g.N % 8 || g.M % 8 || g.lda % 8 || g.ldb % 8 || g.ldo % 4)
      return RV_E_INVAL;
    if ((((uintptr_t)g.A) | ((uintptr_t)g.B) | ((uintptr_t)g.out)) & 15) return RV_E_INVAL;
    if (!operand_fits(g)) return RV_E_INVAL;
    if ((g.upd_w != nullptr) != (g.upd_ver != nullptr)) return RV_E_INVAL;
    if (!g.upd_w && !g.store_out) return RV_E_INVAL;
    if ((((uintptr_t)g.upd_w) & 15) || (((uintptr_t)g.upd_ver) & 7)) return RV_E_INVAL;
  }
  if (form == RV_WGRAD_BY_TOKENS) {
    int M[RV_GEMM_GROUP_BLOCK], N[RV_GEMM_GROUP_BLOCK];
    for (int k = 0; k < count; ++k) { M[k] = gs[k].M; N[k] = gs[k].N; }
    form = gs[0].K < RV_WGRAD_SPLIT_K && tiles_of(count, M, N, 256) < 256 ? RV_WGRAD_SPLIT : RV_WGRAD_IN_ORDER;
  }
  if (form == RV_WGRAD_IN_ORDER) return launch_grouped_dtl<256, 256, 32, 4, 8>(gs, count, st);
  return count > RV_GEMM_GROUP_BLOCK ? launch_grouped_split<128, 128, 2, 4, 4, RV_GEMM_GROUP_MAX>(gs, count, st)
                                     : launch_grouped_split<128, 128, 2, 4, 4, RV_GEMM_GROUP_BLOCK>(gs, count, st);
}

extern "C" rv_status rv_k_gemm_bf16(const void* A, int64_t lda, int a_kmajor, const void* B, int64_t ldb,
                                    int b_kmajor, int M, int N, int K, int epilogue, void* out, int64_t ldo,
                                    void* out2, const void* bias, const float* resid, int64_t ldr,
                                    const void* zin, int tile, void* stream) {
  rv_gemm_args g;
  g.A = (const uint16_t*)A; g.lda = lda; g.a_kmajor = a_kmajor;
  g.B = (const uint16_t*)B; g.ldb = ldb; g.b_kmajor = b_kmajor;
  g.M = M; g.N = N; g.K = K; g.epi = epilogue; g.out = out; g.ldo = ldo; g.out2 = out2;
  g.bias = (const uint16_t*)bias; g.resid = resid; g.ldr = ldr; g.zin = (const uint16_t*)zin; g.tile = tile;
  return rv_gemm_bf16(g, (hipStream_t)stream);
}

extern "C" rv_status rv_k_gemm_bf16_blocks(const void* A, int a_blocks, int a_kmajor, const void* B, int b_blocks, int b_kmajor, int M,
                                           int N, int K, int epilogue, void* out, void* out2, int out_blocks, const void* bias,
                                           const float* resid, const void* zin, int tile, int parts, void* stream) {
  if (M < 1 || N < 1 || K < 1 || (out_blocks && epilogue != EPI_BF16_BIAS_GELU && epilogue != EPI_BF16_DGELU)) return RV_E_INVAL;
  auto operand = [](const void* p, int blocks, int64_t rows, int64_t cols) { return blocks ? rv_blocks(p, rows) : rv_rows(p, cols); };
  const rv_mat a = a_kmajor ? operand(A, a_blocks, K, M) : operand(A, a_blocks, M, K);
  const rv_mat b = b_kmajor ? operand(B, b_blocks, K, N) : operand(B, b_blocks, N, K);
  rv_gemm_args g;
  g.A = a.p; g.lda = a.ld; g.a_bs = a.bs; g.a_kmajor = a_kmajor;
  g.B = b.p; g.ldb = b.ld; g.b_bs = b.bs; g.b_kmajor = b_kmajor;
  g.M = M; g.N = N; g.K = K; g.epi = epilogue; g.out = out; g.ldo = N; g.out2 = out2; g.bsv = out_blocks ? (int64_t)M * 32 : 0;
  g.bias = (const uint16_t*)bias; g.resid = resid; g.ldr = N; g.zin = (const uint16_t*)zin; g.tile = tile;
  return parts ? rv_gemm_part(g, parts, (float*)out, (hipStream_t)stream) : rv_gemm_bf16(g, (hipStream_t)stream);
}

extern "C" rv_status rv_k_gemm_part_form(int M, int N, int K, int* tile, int* parts) {
  if (!tile || !parts || M < 8 || N < 8 || K < 64) return RV_E_INVAL;
  const rv_part_form form = rv_gemm_part_form(M, N, K);
  *tile = form.tile;
  *parts = form.S;
  return RV_OK;
}

extern "C" rv_status rv_k_gemm_part(const void* A, int64_t lda, const void* B, int64_t ldb, int b_kmajor, int M, int N, int K,
                                    int tile, int parts, float* part, void* stream) {
  rv_gemm_args g;
  g.A = (const uint16_t*)A; g.lda = lda; g.B = (const uint16_t*)B; g.ldb = ldb; g.b_kmajor = b_kmajor;
  g.M = M; g.N = N; g.K = K; g.tile = tile;
  return rv_gemm_part(g, parts, part, (hipStream_t)stream);
}

extern "C" rv_status rv_k_gemm_wgrad_grouped(int count, const void* const* X, const int64_t* lda,
                                             const void* const* dY, const int64_t* ldb, const int* M, const int* N,
                                             int K, float* const* dW, void* stream) {
  if (count < 1 || count > RV_GEMM_GROUP_BLOCK || !X || !lda || !dY || !ldb || !M || !N || !dW) return RV_E_INVAL;
  rv_gemm_args g[RV_GEMM_GROUP_BLOCK];
  for (int k = 0; k < count; ++k) {
    g[k].A = (const uint16_t*)X[k]; g[k].lda = lda[k]; g[k].a_kmajor = 1;
    g[k].B = (const uint16_t*)dY[k]; g[k].ldb = ldb[k]; g[k].b_kmajor = 1;
    g[k].M = M[k]; g[k].N = N[k]; g[k].K = K; g[k].epi = EPI_F32; g[k].out = dW[k]; g[k].ldo = N[k];
  }
  return rv_gemm_wgrad_grouped(g, count, (hipStream_t)stream, RV_WGRAD_IN_ORDER);
}

extern "C" rv_status rv_k_gemm_wgrad_update(int count, const void* const* X, const int64_t* lda, const void* const* dY,
                                            const int64_t* ldb, const int* M, const int* N, int K, float* const* dW,
                                            float* const* w, void* const* ver, float eta, void* stream) {
  if (count < 1 || count > RV_GEMM_GROUP_BLOCK || !X || !lda || !dY || !ldb || !M || !N || (!dW && !w) || !w != !ver) return RV_E_INVAL;
  rv_gemm_args g[RV_GEMM_GROUP_BLOCK];
  for (int k = 0; k < count; ++k) {
    g[k].A = (const uint16_t*)X[k]; g[k].lda = lda[k]; g[k].a_kmajor = 1;
    g[k].B = (const uint16_t*)dY[k]; g[k].ldb = ldb[k]; g[k].b_kmajor = 1;
    g[k].M = M[k]; g[k].N = N[k]; g[k].K = K; g[k].epi = EPI_F32; g[k].ldo = N[k];
    g[k].out = dW ? dW[k] : w[k];   // (not written without dW)
    g[k].store_out = dW != nullptr;
    if (w) { g[k].upd_w = w[k]; g[k].upd_ver = (uint16_t*)ver[k]; g[k].upd_eta = eta; }
  }
  return rv_gemm_wgrad_grouped(g, count, (hipStream_t)stream, RV_WGRAD_BY_TOKENS);
}

// The loss at the end of a chain of peers: softmax cross entropy of every token against a vocabulary, and its gradients.
//
//   z = x W^T           x bf16 [T, d], W bf16 [V, d], z in fp32 registers only
//   loss_t = lse_t - z[t, y_t],   lse_t = ln sum_v exp z[t, v]
//   dz[t, v] = r_t (exp(z[t, v] - lse_t) - [v = y_t])      r: the caller's weight of a row
//   dx = s dz W,  dW = s dz^T x                              s: the caller's scale, on the fp32 sums (in dz, where labels' entries are
//                                                            near -1, its rounding would be that of all of them: a bias)
// Three products of 2 T V d flop each; the forward alone is one.
//
// The logits are never written.  A wave of the first product holds 64 columns of the vocabulary - a strip - of its rows; it takes
// each row's maximum over the strip, m, and writes the pair (m, sum of exp2((z - m) log2 e + 15)) in fp32 and, for the
// gradients, the exponentials e themselves in fp16: they are at most 2^15 whatever the logits are, keep 11 bits down to 2^-29 of the
// strip's largest and are off by less than 2^-40 of it below.  (Logits in 16 bits would move a probability by |z| 2^-9 of itself, e in
// bf16 by 2^-8: with the rounding of dz the gradients were then 1.6 times as far from 64 bits as their own rounding, now 1.2.)  The pairs of
// a row's strips are joined to its largest logit, top, and the sum of its exponentials, and  dz = e exp2((m - top) log2 e) r / sum  overwrites e
// in place, rounded to bf16, which is what the matrix instructions take.
// Maximum and sum stay two numbers: differences are formed of logits, before anything is multiplied or added, so that what they lose
// does not grow with the logits (m log2 e or lse in ONE fp32 number is off by 2^-24 of itself, and a probability by that many powers of e).
// loss = (top - z_y) + ln sum has two terms that are not negative, and the label's own column of dz is  r expm1(-loss):
// p - 1 from a rounded p would have fewer digits where the model is nearly certain.
// Computing z again for the gradients instead of keeping e would be a fourth product: 2 bytes of e written and 4 moved by the pass
// that makes dz of it are 1.2 ps a logit at 5 TB/s, the product 2 d / 1.3 PFLOP/s = 1.6 ps at d 1024, 3.2 ps at 2048.
// One piece of rows is kept at a time (e, strips and dx's sums of `rows` rows; where the caller leaves the choice 2^30 elements of e or of dx at
// most, but 128 rows at least, and twice that of e where a batch of up to 256 rows may need its dz in two parts), so what grows with T
// is the copy of x alone; from the second piece on the weight gradient is added up in fp32.
//
// Rows whose label lies outside [0, V) - prompts, padding - take no part: a first kernel gathers the others, in order, into a copy of
// x without gaps, in blocks of 32 columns (rv_mat), and all kernels behind it go by the number of rows it counted.  So a batch that is half
// prompt costs half.  A batch of up to 256 rows, whose products are bound by the weights, is not gathered: a launch less, and the rows that take
// no part become zeros where dz and its copy of x are made.  Either way nothing such a row holds (NaN of an unwritten buffer) reaches an output.
#include <math.h>
#include "gemm_core.h"

namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr int STRIP = 64;
constexpr int kTop = 15;                 // a strip's largest exponential is 2^15
constexpr int64_t kMostE = 1ll << 30;    // elements of e, and of dx, of a piece's rows, where the caller leaves the choice

// what a row of the piece needs in the backward
struct RowInfo { float top, g, at_label; int label; };    // largest logit; weight over the sum of exponentials; dz of the label

struct CutForm { int tile, S; };
struct Plan {
  int T, d, V, Vp, P, R, pieces;         // V rounded up to whole strips; rows of a piece, of a block of e; number of pieces
  bool grads, few;                       // few: up to kFewRows rows, not gathered
  int64_t ldw;
  CutForm dx;                            // tile and stretches of dx; stretches of dW
  int S_w;
  size_t count, pos, idx, lab, info, target, stat, xw, tail, e, part, acc, bytes;
};

__host__ __device__ inline int div_up(int a, int b) { return (a + b - 1) / b; }
__host__ __device__ inline int round_up(int a, int b) { return div_up(a, b) * b; }

// The rows that the kernels work on, in pieces of P.  Gathered (count != null): *count rows without gaps, lab and idx their labels and places.
// Up to kFewRows rows stay where they are, and those that take no part become zeros where dz is made.
struct Rows {
  const int* count; const int* lab; const int* idx; const int* pos;
  const int64_t* label;
  int T, V, p, P;
  int R;                                   // rows of a block of columns of e and of the copy of x: P, or more where dz may have two parts
  int twice;                               // dW of dz in two parts (dz_kernel)
};
constexpr int kFewRows = 256;
__device__ __forceinline__ int rows_of(const Rows& r) {
  const int left = (r.count ? *r.count : r.T) - r.p * r.P;
  return left < r.P ? left : r.P;
}
// k-tiles of dW's product over them, one of zeros where there is none
__device__ __forceinline__ int row_tiles(const Rows& r, int M) { return div_up(M > 0 ? M : 1, 32) << r.twice; }
// the label of a token, of a row of the piece, -1: takes no part
__device__ __forceinline__ int label_at(const Rows& r, int t) {
  const int64_t y = r.label[t];
  return y >= 0 && y < r.V ? (int)y : -1;
}
__device__ __forceinline__ int label_of(const Rows& r, int row) {
  return r.count ? r.lab[r.p * r.P + row] : label_at(r, r.p * r.P + row);
}

// row r of the tail of W: the rows from V / 32 * 32 on, zeros behind the last (see input_grad_body)
__device__ __forceinline__ void copy_tail(const uint16_t* __restrict__ w, int64_t ldw, int d, int V, uint16_t* __restrict__ tail, int r) {
  const int v = V / 32 * 32 + r;
  for (int c = threadIdx.x; c < d / 8; c += 256) {
    u32x4 u = {0u, 0u, 0u, 0u};
    if (v < V) u = *reinterpret_cast<const u32x4*>(w + (int64_t)v * ldw + c * 8);
    *reinterpret_cast<u32x4*>(tail + (int64_t)r * ldw + c * 8) = u;
  }
}

// ---- rows that take part ----------------------------------------------------------------------
// A block takes `per` consecutive rows, 64 at a time; where they go follows from the number of labels before them that take part, which
// it counts itself: at most a thousand blocks do it, 8 T bytes each out of L2, and a scan of its own would be a launch more.
// pos[t] = place among the rows kept or -1; idx, lab: the other way round.  The block of the last rows leaves their number.
// Behind the row blocks: the tail of W.  Bound by memory: 8192 rows of d 2048 18 us, 3.6 TB/s.
__global__ __launch_bounds__(256) void gather_kernel(const uint16_t* __restrict__ x, int64_t ldx, const int64_t* __restrict__ label, int T,
                                                     int d, int V, int P, int per, int* __restrict__ count, int* __restrict__ pos,
                                                     int* __restrict__ idx, int* __restrict__ lab, uint16_t* __restrict__ xw,
                                                     float* __restrict__ loss, float* __restrict__ lse, const uint16_t* __restrict__ w,
                                                     int64_t ldw, uint16_t* __restrict__ tail, int row_blocks) {
  const int tid = threadIdx.x, l = tid & 63;
  if ((int)blockIdx.x >= row_blocks) {
    copy_tail(w, ldw, d, V, tail, blockIdx.x - row_blocks);
    return;
  }
  __shared__ int part[4], place[64];
  const int t0 = blockIdx.x * per, t1 = T - t0 < per ? T : t0 + per;
  auto takes = [&](int64_t y) { return y >= 0 && y < V; };
  int before = 0;
  for (int t = tid; t < t0; t += 8 * 256) {   // (eight on the way at a time)
    int64_t y[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) y[k] = label[t + k * 256 < t0 ? t + k * 256 : t];
#pragma unroll
    for (int k = 0; k < 8; ++k) before += t + k * 256 < t0 && takes(y[k]) ? 1 : 0;
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) before += __shfl_xor(before, o, 64);
  if (l == 0) part[tid >> 6] = before;
  __syncthreads();
  before = part[0] + part[1] + part[2] + part[3];
  for (int first = t0; first < t1; first += 64) {
    const int rows = t1 - first < 64 ? t1 - first : 64;
    if (tid < 64) {
      const int64_t y = l < rows ? label[first + l] : -1;
      const bool in = takes(y);
      const uint64_t all = __builtin_amdgcn_ballot_w64(in);
      const int j = before + __popcll(all & ((1ull << l) - 1));
      place[l] = in ? j : -1;
      if (l < rows) {
        pos[first + l] = in ? j : -1;
        if (in) { idx[j] = first + l; lab[j] = (int)y; }
        else { loss[first + l] = 0.f; if (lse) lse[first + l] = 0.f; }
      }
      before += __popcll(all);
      if (l == 0 && first + rows == T) *count = before;
    }
    __syncthreads();
    const int chunks = rows * (d / 8);
    for (int i = tid; i < chunks; i += 256) {
      // four chunks of a block of 32 columns in neighbouring lanes, then the next row: what is written is runs of 64 bytes a row
      const int q = i & 3, r = (i >> 2) % rows, cb = (i >> 2) / rows, j = place[r];
      if (j < 0) continue;
      const int p = j / P, jr = j - p * P;
      const u32x4 u = *reinterpret_cast<const u32x4*>(x + (int64_t)(first + r) * ldx + cb * 32 + q * 8);
      *reinterpret_cast<u32x4*>(xw + (int64_t)p * P * d + (int64_t)cb * 32 * P + 32 * jr + q * 8) = u;
    }
    __syncthreads();
  }
}

// Workgroup ids go to the 8 XCDs in turn; this gives each a contiguous range of a list of n, whose neighbours read the same operands.  The
// operands do not fit an L2, and what eight of them fetch of the same panels comes out of the power that bounds the products: us, ids as they
// come / ranges, V 128000, d 2048, 8192 rows: logits 3674 / 3458, dx 3209 / 3008, dW 3169 / 2978.
__device__ __forceinline__ int xcd_range(int id, int n) {
  const int base = n / 8, rem = n % 8, x = id % 8;
  return x * base + (x < rem ? x : rem) + id / 8;
}
// number in a list of vm x vn tiles -> tile: bands of kBand tile rows, column by column, so that the 32 workgroups an XCD holds are a patch
constexpr int kBand = 4;
__device__ __forceinline__ void band_tile(int i, int vm, int vn, int& bm, int& bn) {
  const int band = i / (kBand * vn), first = band * kBand, rows = vm - first < kBand ? vm - first : kBand, in = i - first * vn;
  bm = first + in % rows;
  bn = in / rows;
}
// Of a list of tiles of 256x256, those that are handed out whole: where the last round has work for up to half of the CUs its tiles go
// to two workgroups each, upper and lower half, which take three quarters of a whole one's time.  us, without / with: half of 4096 tokens,
// V 50257, d 1024 (logits 6.2 rounds, dW 3.1) 717 / 690; update, 1024, V 20000, d 1024 (1.2, 1.2) 220 / 209; 3001, V 50257, d 1600, logits
// alone (8.5) 394 / 391.  (Quarters would gain a few percent of such a round more, and only where it has 64 tiles or fewer.)
__host__ __device__ inline int whole_tiles(int tiles) { return tiles > 256 && tiles % 256 <= 128 ? tiles - tiles % 256 : tiles; }
__host__ __device__ inline int halved_grid(int tiles) { return 2 * tiles - whole_tiles(tiles); }
// workgroup of halved_grid -> number in the list; half: -1, or which
__device__ __forceinline__ int dealt_tile(int id, int tiles, int& half) {
  const int whole = whole_tiles(tiles);
  half = -1;
  if (id < whole) return xcd_range(id, whole);
  id = xcd_range(id - whole, 2 * (tiles - whole));
  half = id & 1;
  return whole + id / 2;
}

// ---- the logits' product ----------------------------------------------------------------------
// Bound by the matrix cores at the board's power cap: 7783 rows, V 128000, d 2048 3.37 ms, 1.21 PFLOP/s (a library product of 8192^3 1.37); of that
// 0.35 ms are the epilogue, exponentials and stores about half each.  (Tiles of 128x256, two to a CU, whose epilogues run beside walks: the whole
// step 11.03 ms to 10.77.)
// (The tiles are dealt out over the tile rows that are there: a map over the rows of all tokens would leave whole XCDs without work where half
// of the rows are out.)
struct LogitsOut {
  uint16_t* e;         // [Vp / 32][R][32]
  float2* stat;        // [Vp / 64][P]
  float* target;       // [P] the label's logit
  int P, R, V, Vp;
};

// max and sum over the four lanes (l / 16) that share a row, left in all of them: lane rows swapped with their neighbours, then halves
__device__ __forceinline__ float quad_max(float v) {
  auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
  s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float quad_sum(float v) {
  auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
  s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {   // round to nearest even
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, f16x2));
}

// label: of the lane's rows, -1 where there is none.  Rows behind the last one are written like the others (P is whole tiles) and never read.
template <bool STORE, int TM, int TN>
__device__ __forceinline__ void strip_epilogue(const f32x4 (&acc)[TM][TN], const LogitsOut& o, const int (&label)[TM], int mw, int nw, int M) {
  static_assert(TN * 16 == STRIP, "a wave's columns are one strip");
  if (nw >= o.Vp || mw >= M) return;
  const int l = threadIdx.x & 63, grp = l >> 4, strip = nw / STRIP, row0 = mw + (l & 15);
  f32x4 a[TM][TN];
  bool hit = false;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
#pragma unroll
    for (int c = 0; c < TN; ++c) a[i][c] = acc[i][c];
    hit |= (unsigned)(label[i] - nw) < (unsigned)STRIP;
  }
  // One branch for all rows each: a branch for every one of them would keep the rows' chains of instructions apart.
  if (nw + STRIP > o.V) {                                  // (wave-uniform) the last strip ends inside
    asm volatile("");
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int c = 0; c < TN; ++c)
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (nw + c * 16 + 4 * grp + k >= o.V) a[i][c][k] = -INFINITY;
  }
  if (__builtin_amdgcn_ballot_w64(hit)) {                  // few strips hold a label of their rows
    asm volatile("");
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int y = label[i] - nw;
#pragma unroll
      for (int c = 0; c < TN; ++c)
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (y == c * 16 + 4 * grp + k) o.target[row0 + i * 16] = a[i][c][k];
    }
  }
  float2* stat = o.stat + (int64_t)strip * o.P + row0;
  uint16_t* e = o.e + ((int64_t)2 * strip * o.R + row0) * 32 + (grp & 1 ? 16 + 4 * (grp - 1) : 4 * grp);
  const int64_t block = 32ll * o.R;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    float m = a[i][0][0];
#pragma unroll
    for (int c = 0; c < TN; ++c)
#pragma unroll
      for (int k = 0; k < 4; ++k) m = fmaxf(m, a[i][c][k]);
    m = quad_max(m);
    const float base = m == -INFINITY ? 0.f : m;           // (a strip of -inf alone: its sum is zero)
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < TN; ++c)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        a[i][c][k] = __builtin_amdgcn_exp2f(__fmaf_rn(a[i][c][k] - base, kLog2e, (float)kTop));
        sum += a[i][c][k];
      }
    sum = quad_sum(sum);
    if (grp == 0) stat[i * 16] = float2{m, sum};
    if (STORE) {
      // Two quads of a lane are 16 columns apart; the swap of lane rows of 16 gives even rows eight consecutive columns of the first
      // quad and odd ones of the second, and a wave's 16 bytes a lane are one run of 1 KiB of the block of 32 columns.
#pragma unroll
      for (int b = 0; b < TN / 2; ++b) {
        u32x4 v;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const auto s = __builtin_amdgcn_permlane16_swap(pack_f16(a[i][2 * b][2 * h], a[i][2 * b][2 * h + 1]),
                                                          pack_f16(a[i][2 * b + 1][2 * h], a[i][2 * b + 1][2 * h + 1]), false, false);
          v[h] = s[0]; v[2 + h] = s[1];
        }
        *reinterpret_cast<u32x4*>(e + b * block + i * 512) = v;
      }
    }
  }
}

template <int BM, int BN, int NS, int NW, bool STORE>
__global__ __launch_bounds__(64 * NW, 2) void logits_kernel(const uint16_t* __restrict__ x, int64_t ldx, int64_t x_bs, const uint16_t* __restrict__ w,
                                                            int64_t ldw, int d, Rows rows, LogitsOut o) {
  const int M = rows_of(rows);
  if (M <= 0) return;
  const int vm = div_up(M, BM), vn = div_up(o.Vp, BN), tiles = vm * vn;
  int bm, bn, half = -1;
  if ((int)blockIdx.x >= (BM == 256 ? halved_grid(tiles) : tiles)) return;
  band_tile(BM == 256 ? dealt_tile(blockIdx.x, tiles, half) : xcd_range(blockIdx.x, tiles), vm, vn, bm, bn);
  auto tile = [&](auto rows_of_tile, int bm) {
    constexpr int BT = rows_of_tile, TM = BT / 2 / 16;
    // the labels of this lane's rows, asked for here: behind the walk along d each would be a round trip of its own
    const int first = bm * BT + (threadIdx.x >> 6 & 1) * (BT / 2) + (threadIdx.x & 15);
    int label[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) label[i] = first + i * 16 < M ? label_of(rows, first + i * 16) : -1;
    auto own = [&](const auto& acc, int m0, int n0, int wm0, int wn0) { strip_epilogue<STORE>(acc, o, label, m0 + wm0, n0 + wn0, M); };
    gemm_dtl_body<BT, BN, 32, NS, NW, false, false, EPI_OWN>(x, ldx, x_bs, w, ldw, 32, M, o.V, d, bm, bn, Epi{}, nullptr, 0, own);
  };
  if (BM == 128 || half < 0) tile(std::integral_constant<int, BM>{}, bm);
  else if ((2 * bm + half) * 128 < M) tile(std::integral_constant<int, 128>{}, 2 * bm + half);
}

// ---- strips joined to rows ----------------------------------------------------------------------
// 16 rows to a block, 64 lanes to a row: a strip's pairs of 16 rows are one line.  Bound by memory and, with few rows, by its chain of round
// trips: 7783 rows of V 128000 40 us, 3.1 TB/s; one row of V 32000 4 us.
__global__ __launch_bounds__(1024) void join_kernel(const float2* __restrict__ stat, const float* __restrict__ target, Rows rows, int strips,
                                                    const float* __restrict__ row_scale, float* __restrict__ loss, float* __restrict__ lse,
                                                    RowInfo* __restrict__ info) {
  __shared__ float2 part[64][17];
  const int P = rows.P, M = rows_of(rows), r = threadIdx.x & 15, sl = threadIdx.x >> 4, row = blockIdx.x * 16 + r;
  if ((int)blockIdx.x * 16 >= M) return;
  auto join = [](float2 a, float2 b) {
    const float m = fmaxf(a.x, b.x), base = m == -INFINITY ? 0.f : m;
    return float2{m, a.y * __builtin_amdgcn_exp2f((a.x - base) * kLog2e) + b.y * __builtin_amdgcn_exp2f((b.x - base) * kLog2e)};
  };
  float2 v = {-INFINITY, 0.f};
  if (row < M) {
#pragma unroll 4
    for (int s = sl; s < strips; s += 64) v = join(v, stat[(int64_t)s * P + row]);
  }
  part[sl][r] = v;
  __syncthreads();
  for (int n = 32; n; n >>= 1) {
    if (sl < n) part[sl][r] = join(part[sl][r], part[sl + n][r]);
    __syncthreads();
  }
  if (sl != 0 || row >= M) return;
  v = part[0][r];
  const int at_piece = rows.p * P + row, t = rows.count ? rows.idx[at_piece] : at_piece, y = label_of(rows, row);
  if (y < 0) {                                    // (not gathered) whatever its logits were
    loss[t] = 0.f;
    if (lse) lse[t] = 0.f;
    if (info) info[row] = RowInfo{0.f, 0.f, 0.f, -1};
    return;
  }
  // (the largest logit's own exponential is exactly 2^kTop and nothing is taken away from a sum: the log is not negative)
  const float ln = logf(v.y * (1.0f / (1 << kTop))), each = (v.x - target[row]) + ln;
  loss[t] = each;
  if (lse) lse[t] = v.x + ln;
  if (info) {
    const float g = row_scale ? row_scale[t] : 1.0f;
    info[row] = RowInfo{v.x, g / v.y, g * expm1f(-each), y};
  }
}

// ---- e -> dz, in place ----------------------------------------------------------------------
// Bound by memory: 7783 rows of V 128000 780 us, 5.1 TB/s, a large copy's rate.
// 64 rows to a block, four lanes to a row's 64 bytes of a block of columns, `per` strips one after the other.  Rows that take no part, and those
// from the last one up to whole tiles of 32, become zeros, of dz here and of the copy of x that the weight gradient's product walks over.
// Two parts (`twice`: an update by a batch of up to 256 rows, dW of up to 64, however they are cut into pieces): what dz loses to bf16 is rounded
// itself and stands, with the same rows of x, behind the rows, so that dW has 16 bits of the labels' entries, which are most of it, and the 11
// of e of the others - the fp32 master would otherwise be off by up to 2^-9 of a single token's whole step.  The product is bound by the weights
// there.  Larger batches would pay for it with another product of dW's size; an update by them has the labels' entries alone in two parts
// (labels_rest), the others with the one rounding that a stage's own gradients have.
// Where rows are not gathered the copy is made here, by the blocks behind the strips', and the tail of W by those behind them.
__global__ __launch_bounds__(256) void dz_kernel(uint16_t* __restrict__ e, const float2* __restrict__ stat, const RowInfo* __restrict__ info, Rows rows,
                                                 int strips, int per, int strip_blocks, uint16_t* __restrict__ xw, int d, const uint16_t* __restrict__ x,
                                                 int64_t ldx, const uint16_t* __restrict__ w, int64_t ldw, uint16_t* __restrict__ tail) {
  const int P = rows.P;
  int M = rows_of(rows);
  if (M <= 0) {
    if (rows.p) return;
    M = 0;                                        // no row at all: one tile of zeros
  }
  const int row = blockIdx.x * 64 + threadIdx.x / 4, q = threadIdx.x & 3;
  const int end = round_up(M > 0 ? M : 1, 32);
  const u32x4 zero = {0u, 0u, 0u, 0u};
  if ((int)blockIdx.y >= strip_blocks) {          // (rows not gathered) 8 blocks of 32 columns of x each, then a row of the tail each
    const int c0 = (blockIdx.y - strip_blocks) * 8, copies = div_up(d / 32, 8);
    if ((int)blockIdx.y - strip_blocks >= copies) {
      if (blockIdx.x == 0) copy_tail(w, ldw, d, rows.V, tail, blockIdx.y - strip_blocks - copies);
      return;
    }
    if (row >= end) return;
    const bool in = row < M && label_of(rows, row) >= 0;
    for (int cb = c0; cb < c0 + 8 && cb < d / 32; ++cb) {
      const u32x4 v = in ? *reinterpret_cast<const u32x4*>(x + (int64_t)row * ldx + cb * 32 + q * 8) : zero;
      uint16_t* to = xw + ((int64_t)cb * rows.R + row) * 32 + q * 8;
      *reinterpret_cast<u32x4*>(to) = v;
      if (rows.twice) *reinterpret_cast<u32x4*>(to + end * 32) = v;
    }
    return;
  }
  if (row >= end) return;
  const int s0 = blockIdx.y * per, s1 = s0 + per < strips ? s0 + per : strips;
  uint16_t* base = e + (int64_t)row * 32 + q * 8;
  const int64_t bs = 32ll * rows.R;
  if (row >= M || info[row].label < 0) {
    for (int s = s0; s < s1; ++s) {
      *reinterpret_cast<u32x4*>(base + 2 * s * bs) = zero;
      *reinterpret_cast<u32x4*>(base + (2 * s + 1) * bs) = zero;
      if (rows.twice) {
        *reinterpret_cast<u32x4*>(base + 2 * s * bs + end * 32) = zero;
        *reinterpret_cast<u32x4*>(base + (2 * s + 1) * bs + end * 32) = zero;
      }
    }
    if (rows.count && blockIdx.y == 0) {
      for (int cb = 0; cb < d / 32; ++cb) *reinterpret_cast<u32x4*>(xw + ((int64_t)cb * rows.R + row) * 32 + q * 8) = zero;
    }
    return;
  }
  const RowInfo r = info[row];
#pragma unroll 2
  for (int s = s0; s < s1; ++s) {
    const float f = r.g * __builtin_amdgcn_exp2f((stat[(int64_t)s * P + row].x - r.top) * kLog2e);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      u32x4* at = reinterpret_cast<u32x4*>(base + (2 * s + h) * bs);
      f32x4 v[2];
      const u32x4 packed = *at;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t pair = packed[k];          // (a bit cast of a vector's element reads element 0)
        const f32x2 two = __builtin_convertvector(__builtin_bit_cast(f16x2, pair), f32x2);
        v[k >> 1][2 * (k & 1)] = two.x; v[k >> 1][2 * (k & 1) + 1] = two.y;
      }
      const int y = r.label - ((2 * s + h) * 32 + q * 8);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k >> 2][k & 3] = y == k ? r.at_label : v[k >> 2][k & 3] * f;
      const u32x4 rounded = f32_to_bf16x8(v);
      *at = rounded;
      if (rows.twice) {
        f32x4 back[2];
        bf16x8_to_f32(back, rounded);
        v[0] -= back[0]; v[1] -= back[1];
        at[end * 4] = f32_to_bf16x8(v);
      }
    }
  }
}

// ---- dx ----------------------------------------------------------------------
// dx has few tiles and a contraction as long as the vocabulary: it is cut into S stretches, whose fp32 sums a second kernel adds.  Tile and
// S are the host's choice by modelled time for all rows (cut_form below); where fewer rows take part, the device, which alone knows,
// makes as many more stretches of the walk as there are tile rows less, so that the launch fills the chip as far as it was to.
constexpr int kMostParts = 64;
__device__ __forceinline__ int stretches(int S, int tiles_m, int vm, int nk) {
  int n = S * tiles_m / vm;
  n = n < kMostParts ? n : kMostParts;
  n = n * 8 <= nk ? n : nk / 8;
  return n > S ? n : S;
}
struct GradArgs {
  const uint16_t* dz; const uint16_t* xw; const uint16_t* w;
  int64_t ldw;
  Rows rows;
  int d, Vp;
  int S_dx, tiles_m, dx_grid;             // dx: stretches for all rows, their tile rows, workgroups
  const uint16_t* tail; float* part;
  int S_w, w_first;                       // dW; its workgroups in front of those of dx (both_grads_kernel)
  float* sums; uint16_t* dw; const float* master; float* master_out; uint16_t* version;
  float scale, eta;                       // eta: times scale
  const RowInfo* info;                    // of an update by gathered rows (labels_rest), else null
};
// BM 256: tiles of 256x256, eight waves, in order of k; 128: of 128x128, the walk split over two groups of four waves.  The last k-tiles, which
// end behind the last row of W, come from its copy with zeros behind (there is nothing behind W that could be read).  7783 rows, V 128000,
// d 2048 3.0 ms, 1.36 PFLOP/s; 2048 rows, V 50257, d 1024, in eight stretches, 0.18 ms, 1.15.
template <int BM>
__device__ __forceinline__ void input_grad_body(const GradArgs& a, int id) {
  const int d = a.d, V = a.rows.V, M = rows_of(a.rows);
  if (M <= 0) return;
  const int vm = div_up(M, BM), vn = div_up(d, BM), tiles = vm * vn, nk = a.Vp / 32;
  const int S = stretches(a.S_dx, a.tiles_m, vm, nk);
  if (id >= tiles * S) return;
  id = xcd_range(id, tiles * S);
  const int s = id / tiles;
  int bm, bn;
  band_tile(id - s * tiles, vm, vn, bm, bn);
  const int k0 = (int)((int64_t)nk * s / S), k1 = (int)((int64_t)nk * (s + 1) / S);
  Epi out{};
  out.out = a.part + (int64_t)s * vm * BM * d; out.ldo = d;
  const uint16_t* A = a.dz + (int64_t)k0 * 32 * a.rows.R;
  const int64_t bs = 32ll * a.rows.R;
  const uint16_t* B = a.w + (int64_t)k0 * 32 * a.ldw;
  if constexpr (BM == 256)
    gemm_dtl_body<256, 256, 32, 4, 8, false, true, EPI_F32, true>(A, 32, bs, B, a.ldw, 32, M, d, (k1 - k0) * 32, bm, bn, out, a.tail, V / 32 - k0);
  else
    gemm_split_body<128, 128, 2, 4, 4, false, true, EPI_F32, true>(A, 32, bs, B, a.ldw, 32, M, d, (k1 - k0) * 32, bm, bn, out, a.tail, V / 32 - k0);
}
template <int BM>
__global__ __launch_bounds__(512, 2) void input_grad_kernel(GradArgs a) { input_grad_body<BM>(a, blockIdx.x); }
// the stretches' sums, added in a fixed order and rounded, to the rows they belong to; zeros to the rows that take no part.  LANES lanes share
// eight columns of a row: with dozens of stretches one lane's walk over them is a chain of round trips (256 rows of 448
// columns, 64 stretches: 25 us with one lane).  The host chooses by the stretches for all rows; where few of them take part the device makes
// more and one lane may walk over up to 64 sums, but of that many rows less.
template <int LANES>
__global__ __launch_bounds__(256) void input_grad_join_kernel(const float* __restrict__ part, Rows rows, int d, int nk, int bm, int S_all, int tiles_m,
                                                              float scale, uint16_t* __restrict__ dx, int64_t lddx) {
  const int M = rows_of(rows), p = rows.p, P = rows.P;
  if (M <= 0 && p) return;
  const int lane = LANES > 1 ? threadIdx.x / (256 / LANES) : 0;
  const int64_t chunk = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x % (256 / LANES);
  const int per = d / 8;
  const bool in = chunk < (int64_t)rows.T * per;
  const int t = in ? (int)(chunk / per) : 0, c = in ? (int)(chunk - (int64_t)t * per) * 8 : 0;
  const int j = !in ? -1 : rows.count ? rows.pos[t] : label_at(rows, t) >= 0 ? t : -1;
  const bool here = j >= 0 && j / P == p;
  f32x4 v[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
  if (here) {
    const int vm = div_up(M, bm), S = stretches(S_all, tiles_m, vm, nk);
    const int64_t pitch = (int64_t)vm * bm * d;
    const float* src = part + (int64_t)(j - p * P) * d + c;
#pragma unroll 4
    for (int s = lane; s < S; s += LANES) {
      const f32x4* q = reinterpret_cast<const f32x4*>(src + s * pitch);
      v[0] += q[0]; v[1] += q[1];
    }
  }
  if (LANES > 1) {
    __shared__ f32x4 sum[2][256];
    sum[0][threadIdx.x] = v[0]; sum[1][threadIdx.x] = v[1];
    __syncthreads();
    if (lane) return;
#pragma unroll
    for (int x = 1; x < LANES; ++x) {
      v[0] += sum[0][threadIdx.x + x * (256 / LANES)];
      v[1] += sum[1][threadIdx.x + x * (256 / LANES)];
    }
  }
  v[0] *= scale; v[1] *= scale;
  if (in && (here || (j < 0 && p == 0))) *reinterpret_cast<u32x4*>(dx + (int64_t)t * lddx + c) = f32_to_bf16x8(v);
}

// ---- dW ----------------------------------------------------------------------
// What dz loses to bf16 at the labels, given back to an update of a master (gathered rows; up to 256 have all of dz in two parts).  A label's entry is
// near -r, the others of its row add up to r: in the W row of a token that few others share its rounding is nearly all of the error, 2^-9 of
// that token's step.  (The master of 257 rows of V 1000, d 128: 1.6e-5 of itself off without, 6e-7 with, update by 1 / 257 of 0.1.)
// The tile's rows of W are the labels of a few rows only.  They are looked up, SEG rows at a time, in order; then a product of the usual
// kind goes over them alone, 64 at a time: of a matrix that has the rest of dz, rounded to bf16, where the label is and zeros elsewhere, with the
// same rows of x.  The first rows' labels are asked for ahead of the tile's walk, the next 64 rows of x ahead of the product of those before.
// Bound by its chain of round trips, 2 to 3 us a tile.  The step without / with it, us: 4096 rows, V 32000, d 2048 1464 / 1474; 600, V 10000, d 512
// 65.6 / 67.2; 2048, V 1000, d 512, a tile of which has 512 of the rows, 49.6 / 55.2.
constexpr int SEG = 4096, REST = 64;
template <int BT> constexpr int kRestLds = REST * (BT + 256) * 2 + SEG * 6 + 64;
struct Labels { int label[SEG / 512]; float dz[SEG / 512]; };           // of a lane's rows of a segment
__device__ __forceinline__ Labels ask_labels(const RowInfo* __restrict__ info, int seg0, int end) {
  Labels s;
#pragma unroll
  for (int i = 0; i < SEG / 512; ++i) {
    const int row = seg0 + ((threadIdx.x >> 6) * (SEG / 512) + i) * 64 + (threadIdx.x & 63);
    s.label[i] = -1; s.dz[i] = 0.f;
    if (row < end) { s.label[i] = info[row].label; s.dz[i] = info[row].at_label; }
  }
  return s;
}
template <int BT, int TM, int TN>
__device__ __forceinline__ void labels_rest(const GradArgs& a, Labels seg, f32x4 (&acc)[TM][TN], int m0, int n0, int wm0, int wn0, int first, int end) {
  char* const A = dtl_smem;
  char* const B = A + REST * BT * 2;
  int* const list = reinterpret_cast<int*>(B + REST * 256 * 2);         // row of the tile * SEG + row of the segment
  uint16_t* const rest = reinterpret_cast<uint16_t*>(list + SEG);
  int* const found = reinterpret_cast<int*>(rest + SEG);                // by the waves
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l = tid & 63;
  const int64_t bs = 32ll * a.rows.R;
  for (int seg0 = first; seg0 < end; seg0 += SEG) {
    constexpr int PER = SEG / 512;
    if (seg0 != first) seg = ask_labels(a.info, seg0, end);
    int count = 0;
    uint64_t who[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      who[i] = __builtin_amdgcn_ballot_w64((unsigned)(seg.label[i] - m0) < (unsigned)BT);
      count += __popcll(who[i]);
    }
    __syncthreads();                                                    // the operands' ring, or the segment before, is done with
    if (l == 0) found[wave] = count;
    __syncthreads();
    int to = 0, total = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) {
      const int n = found[w];
      to += w < wave ? n : 0;
      total += n;
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (who[i] >> l & 1) {
        const int k = to + __popcll(who[i] & ((1ull << l) - 1));
        list[k] = (seg.label[i] - m0) * SEG + (wave * PER + i) * 64 + l;
        rest[k] = rv_f32_to_bf16(seg.dz[i] - __uint_as_float((uint32_t)rv_f32_to_bf16(seg.dz[i]) << 16));
      }
      to += __popcll(who[i]);
    }
    __syncthreads();
    constexpr int XS = REST * 256 / 8 / 512;
    u32x4 x[XS];
    auto ask_rows = [&](int h0) {
#pragma unroll
      for (int i = 0; i < XS; ++i) {
        const int c = (i * 512 + tid) % 32, k = h0 + (i * 512 + tid) / 32;
        int col = n0 + c * 8;
        col = col < a.d ? col : a.d - 8;
        x[i] = u32x4{0u, 0u, 0u, 0u};
        if (k < total) x[i] = *reinterpret_cast<const u32x4*>(a.xw + (col >> 5) * bs + (int64_t)(seg0 + list[k] % SEG) * 32 + (col & 31));
      }
    };
    ask_rows(0);
    for (int h0 = 0; h0 < total; h0 += REST) {
      if (h0) __syncthreads();                                          // the 64 before are done with
#pragma unroll
      for (int i = 0; i < REST * BT / 8 / 512; ++i) {
        const int c = (i * 512 + tid) % (BT / 8), k = (i * 512 + tid) / (BT / 8), col = h0 + k < total ? list[h0 + k] / SEG : -1;
        u32x4 v = {0u, 0u, 0u, 0u};
        if (col >> 3 == c) {
          const uint32_t r = (uint32_t)rest[h0 + k] << 16 * (col & 1);
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = (col & 7) >> 1 == e ? r : 0u;
        }
        *reinterpret_cast<u32x4*>(A + k * (BT * 2) + ((c ^ km_swizzle<BT>(k & 31)) << 4)) = v;
      }
#pragma unroll
      for (int i = 0; i < XS; ++i) {
        const int c = (i * 512 + tid) % 32, k = (i * 512 + tid) / 32;
        *reinterpret_cast<u32x4*>(B + k * 512 + ((c ^ km_swizzle<256>(k & 31)) << 4)) = x[i];
      }
      __syncthreads();
      if (h0 + REST < total) ask_rows(h0 + REST);
#pragma unroll 1
      for (int k = 0; k < REST && h0 + k < total; k += 32) {
        bf16x8 fa[TM], fb[TN];
#pragma unroll
        for (int i = 0; i < TM; ++i) fa[i] = dtl_frag<true, BT, 32>(A + k * (BT * 2), wm0 + i * 16, 0);
#pragma unroll
        for (int j = 0; j < TN; ++j) fb[j] = dtl_frag<true, 256, 32>(B + k * 512, wn0 + j * 16, 0);
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
          for (int i = 0; i < TM; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[j], fa[i], acc[i][j], 0, 0, 0);
      }
    }
  }
}

// 256x256 tiles, the contraction over the rows: 7783 rows, V 128000, d 2048 3.0 ms, 1.36 PFLOP/s; 2048, V 50257, d 1024 0.21 ms, 1.0 (788 tiles are
// three rounds of the CUs and a twelfth, which is dealt out in halves); few rows are bound by writing dW: 5 rows of V 41302, d 704 with the update
// 74 us with dx, 4.7 TB/s.
// KIND 0: bf16 dw.  1: the update of Eq. 2 on an fp32 master (w' = w - eta dW, one fused multiply-add) and its bf16 version.
// 2: fp32 sums of one of S stretches of the rows (few tiles), or of the first piece.  3: added to those of the pieces before.
constexpr int WB = 256, W_NS = 4, W_NW = 8;
__device__ __forceinline__ int row_stretches(int S, int nk) { return S < nk ? S : nk; }
template <int KIND>
__device__ __forceinline__ void weight_grad_body(const GradArgs& a, int id) {
  const int d = a.d, V = a.rows.V, Vp = a.Vp, M = rows_of(a.rows);
  if (M <= 0 && a.rows.p) return;
  const int64_t bs = 32ll * a.rows.R;
  const int nk = row_tiles(a.rows, M), vm = div_up(V, WB), vn = div_up(d, WB), tiles = vm * vn, parts = KIND == 2 ? row_stretches(a.S_w, nk) : 1;
  constexpr bool kHalves = KIND != 2;
  if (id >= (kHalves ? halved_grid(tiles) : tiles * parts)) return;
  int half = -1;
  id = kHalves ? dealt_tile(id, tiles, half) : xcd_range(id, tiles * parts);
  const int s = id / tiles;
  const int in = id - s * tiles, bn = in % vn, bm = in / vn;
  const int k0 = nk * s / parts, k1 = nk * (s + 1) / parts;
  const int first = k0 * 32, end = k1 * 32 < M ? k1 * 32 : M;
  const bool labels = KIND != 0 && a.info;
  const Labels seg = ask_labels(a.info, first, labels ? end : 0);
  auto tile = [&](auto rows_of_tile, int bm) {
    constexpr int BT = rows_of_tile;
    auto own = [&](auto& acc, int, int n0, int wm0, int wn0) {
      constexpr int TM = BT / 2 / 16, TN = WB / (W_NW / 2) / 16;
      const int m0 = bm * BT;
      if (labels) labels_rest<BT>(a, seg, acc, m0, n0, wm0, wn0, first, end);
      Epi o{};
      o.ldo = d;
      if constexpr (KIND == 0) {
        o.out = a.dw;
        f32x4 scaled[TM][TN];
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int j = 0; j < TN; ++j) scaled[i][j] = acc[i][j] * a.scale;
        write_tile_staged<BT, WB, 64 * W_NW, f32x4, TM, TN, EPI_BF16>(scaled, o, m0, n0, wm0, wn0, V, d, dtl_smem);
      } else if constexpr (KIND == 1) {
        o.out = a.master_out; o.resid = a.master; o.ldr = d; o.out2 = a.version; o.eta = a.eta;
        f32_tile_through_lds<BT, WB, W_NW, f32x4, TM, TN, 2, true>(acc, o, m0, n0, wm0, wn0, V, d, dtl_smem);
      } else if constexpr (KIND == 2) {
        o.out = a.sums + (int64_t)s * V * d;
        write_tile<f32x4, TM, TN, EPI_F32>(acc, o, m0 + wm0, n0 + wn0, V, d);
      } else {
        o.out = a.sums; o.resid = a.sums; o.ldr = d;
        f32_tile_through_lds<BT, WB, W_NW, f32x4, TM, TN, 3, false>(acc, o, m0, n0, wm0, wn0, V, d, dtl_smem);
      }
    };
    // (The loads of dz run over whole strips, the results end at V.  The tile's first column of dz is its base: offsets from the matrix's own
    // would pass 31 bits from 2^31 elements of e on.)
    gemm_dtl_body<BT, WB, 32, W_NS, W_NW, true, true, EPI_OWN>(a.dz + (int64_t)(bm * BT / 32) * bs + (int64_t)k0 * 32 * 32, 32, bs,
                                                               a.xw + (int64_t)k0 * 32 * 32, 32, bs, Vp - bm * BT, d, (k1 - k0) * 32, 0, bn, Epi{},
                                                               nullptr, 0, own);
  };
  if (!kHalves || half < 0) tile(std::integral_constant<int, WB>{}, bm);
  else if (kHalves && (2 * bm + half) * (WB / 2) < V) tile(std::integral_constant<int, WB / 2>{}, 2 * bm + half);
}
template <int KIND>
__global__ __launch_bounds__(512, 2) void weight_grad_kernel(GradArgs a) { weight_grad_body<KIND>(a, blockIdx.x); }
// dx in tiles of 128 and dW in one launch, where neither keeps the chip busy for long.  (With dx in tiles of 256, which do, it costs: 8192 tokens,
// V 128000, d 2048 10.64 ms apart, 10.81 together; 4096, V 32000 1.47 / 1.49; half of 4096, V 50257, d 1024 720 / 710 us.)
// dW's workgroups, the longer ones, come first where there are few of them, or stretches of many rows, and dx's fill the chip beside them.  us,
// dx / dW first: 600 tokens, V 10000, d 512 (80 workgroups of dW) 63 / 58; 6738, V 1347, d 320, update (12 tiles in stretches) 83 / 78; but 256,
// V 30522, d 448 (240) 59.8 / 60.7, 100, V 32000, d 1024 (500) 67 / 71.
template <int KIND>
__global__ __launch_bounds__(512, 2) void both_grads_kernel(GradArgs a) {
  const int id = (int)blockIdx.x - a.w_first;
  if (id >= 0 && id < a.dx_grid) input_grad_body<128>(a, id);
  else weight_grad_body<KIND>(a, id < 0 ? blockIdx.x : id - a.dx_grid);
}
// fp32 sums of stretches or pieces -> dw, or the update
__global__ __launch_bounds__(256) void weight_grad_join_kernel(const float* __restrict__ sums, int S, Rows rows, int pieces, int64_t n,
                                                               uint16_t* __restrict__ dw, const float* __restrict__ master, float* __restrict__ master_out,
                                                               uint16_t* __restrict__ version, float scale, float eta) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (i >= n) return;
  int parts = 1;
  if (pieces == 1) {
    parts = row_stretches(S, row_tiles(rows, rows_of(rows)));
  }
  f32x4 v[2] = {reinterpret_cast<const f32x4*>(sums + i)[0], reinterpret_cast<const f32x4*>(sums + i)[1]};
  for (int s = 1; s < parts; ++s) {
    const f32x4* q = reinterpret_cast<const f32x4*>(sums + s * n + i);
    v[0] += q[0]; v[1] += q[1];
  }
  if (dw) {
    v[0] *= scale; v[1] *= scale;
    *reinterpret_cast<u32x4*>(dw + i) = f32_to_bf16x8(v);
    return;
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const f32x4 m = reinterpret_cast<const f32x4*>(master + i)[h];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[h][k] = __fmaf_rn(-eta, v[h][k], m[k]);
    reinterpret_cast<f32x4*>(master_out + i)[h] = v[h];
  }
  *reinterpret_cast<u32x4*>(version + i) = f32_to_bf16x8(v);
}

// ---- host ----------------------------------------------------------------------

// The 256x256 tile, or 128x128 ones, two workgroups to a CU, where they take less of the chip's time (rounds * area / efficiency, the
// ratio of the two as in gemm_bf16.hip).  A last round of halves counts three quarters where the walk is long enough: 2048 rows, V 9000, d 2048
// (288 tiles) 96 us with tiles of 256, 101 of 128; 4096, V 4400, d 1024 (288) 61 / 62.5; but 8192, V 2500, d 512 (320) 45 / 43.
bool big_tiles(int rows, int cols, int d) {
  const int64_t b = (int64_t)div_up(rows, 256) * div_up(cols, 256), m = (int64_t)div_up(rows, 128) * div_up(cols, 128);
  const double rounds = (double)((b + 255) / 256) - (d >= 1024 && b % 256 && whole_tiles((int)b) < b ? 0.25 : 0);
  return rounds * 65536 <= (double)((m + 511) / 512) * 2 * 16384 / 0.83;
}
// Tile and stretches of a product [M, N] over nk k-tiles whose fp32 sums a kernel adds: the least modelled time, us, of tiles of 256 and, with
// `small`, of 128 whose walk is split over the two halves of a workgroup; one workgroup to a CU.  A round is a start and a walk, whose
// step takes longer where the launch fills the chip (the forms 5256 and 1128 of gemm_bf16.hip, by 32 in k); the sums are written and read
// at 5 TB/s.
CutForm cut_form(int M, int N, int nk, bool small) {
  CutForm best{256, 1};
  float least = 3e38f;
  for (int form = 0; form < (small ? 2 : 1); ++form) {
    const int B = form ? 128 : 256;
    const float start = form ? 4.3f : 8.9f, t0 = form ? 0.235f : 0.51f, t1 = form ? 0.24f : 0.64f;
    const float tiles = (float)div_up(M, B) * div_up(N, B);
    for (int S = 1; S <= kMostParts && (S == 1 || S * 8 <= nk); S += S < 8 ? 1 : S < 16 ? 2 : S < 32 ? 4 : 8) {
      const float fill = tiles * S < 256.f ? tiles * S / 256.f : 1.f;
      const float time = ceilf(tiles * S / 256.f) * (start + ceilf((float)nk / S) * (t0 + (t1 - t0) * fill * fill)) + (float)M * N * S * 8 / 5e6f;
      if (time < least) { least = time; best = {B, S}; }
    }
  }
  return best;
}

bool make_plan(Plan& q, int64_t T, int64_t d, int64_t V, int64_t ldw, int64_t rows, bool grads) {
  if (T < 1 || T > (1 << 20) || d < 64 || d % 64 || d > 16384 || V < 1 || V > (1 << 24) || ldw < d || ldw % 8 || ldw > (1 << 20) || rows < 0) return false;
  if (V * ldw >= (1ll << 31)) return false;       // offsets in the logits' product
  q.T = (int)T; q.d = (int)d; q.V = (int)V; q.Vp = round_up((int)V, STRIP); q.grads = grads; q.ldw = ldw;
  // pieces of nearly the same size, of whole tiles of the logits' product: of 128 rows where that is all, else of 256
  auto tiles = [](int64_t n) { return n <= 128 ? 128 : (n + 255) / 256 * 256; };
  int64_t most = kMostE / (q.Vp > q.d ? q.Vp : q.d);
  most = most < 256 ? 128 : most / 256 * 256;
  if (rows && rows < most) most = tiles(rows);
  q.pieces = (int)((T + most - 1) / most);
  const int64_t P = tiles((T + q.pieces - 1) / q.pieces);
  q.pieces = (int)((T + P - 1) / P);
  q.P = (int)P;
  q.few = T <= kFewRows;
  const int most_rows = q.T < q.P ? q.T : q.P;
  const int both_parts = q.few && grads ? 2 * round_up(most_rows, 32) : 0;   // (rows of dz in two parts)
  q.R = both_parts > q.P ? both_parts : q.P;
  size_t at = 0;
  q.count = q.pos = q.idx = q.lab = q.xw = q.info = q.tail = q.e = q.part = q.acc = 0;
  auto take = [&](size_t bytes) { const size_t was = at; at += (bytes + 255) / 256 * 256; return was; };
  const size_t all = (size_t)q.pieces * P;
  if (!q.few) { q.count = take(4); q.pos = take(4 * all); q.idx = take(4 * all); q.lab = take(4 * all); }
  q.target = take(4 * P);
  q.stat = take((size_t)8 * (q.Vp / STRIP) * P);
  if (!q.few || grads) q.xw = take((size_t)2 * (q.few ? 1 : q.pieces) * q.R * d);
  if (grads) {
    q.info = take(sizeof(RowInfo) * P);
    q.tail = take((size_t)2 * 64 * ldw);
    q.e = take((size_t)2 * q.R * q.Vp);
    q.dx = cut_form(most_rows, q.d, q.Vp / 32, true);
    q.part = take((size_t)div_up(most_rows, q.dx.tile) * q.dx.S * q.dx.tile * q.d * 4);
    q.S_w = q.pieces > 1 ? 1 : cut_form(q.V, q.d, (q.few ? both_parts : q.P) / 32, false).S;
    q.acc = q.pieces > 1 || q.S_w > 1 ? take((size_t)4 * q.S_w * V * d) : 0;
  }
  q.bytes = at;
  return true;
}

constexpr int kBigLds = 4 * 2 * dtl_tile_bytes(256, 32), kMidLds = 4 * 2 * dtl_tile_bytes(128, 32), kSplitLds = split_lds<128, 128, 2, 4>();
constexpr int kWeightLds = WB * stage_pitch(WB) > upd_image_bytes(WB, WB) ? WB * stage_pitch(WB) : upd_image_bytes(WB, WB);
constexpr int kBothLds = kSplitLds > kWeightLds ? kSplitLds : kWeightLds;
static_assert(kWeightLds >= kBigLds && kWeightLds >= kRestLds<WB> && kBothLds <= 160 * 1024, "LDS of one CU");

Rows rows_at(const Plan& q, char* work, const rv_loss_desc& a, int p) {
  Rows r{};
  if (!q.few) {
    r.count = (const int*)(work + q.count); r.lab = (const int*)(work + q.lab); r.idx = (const int*)(work + q.idx); r.pos = (const int*)(work + q.pos);
  }
  r.label = a.label;
  r.T = q.T; r.V = q.V; r.p = p; r.P = q.P; r.R = q.R;
  r.twice = q.few && (a.master || (a.dw && q.T <= 64)) ? 1 : 0;
  return r;
}

// the copy of the piece's rows of x
uint16_t* copy_of_x(const Plan& q, char* work, int p) { return (uint16_t*)(work + q.xw) + (q.few ? 0 : (int64_t)p * q.P * q.d); }
// its first row of x, where rows are not gathered
const uint16_t* rows_of_x(const Plan& q, const rv_loss_desc& a, int p) { return (const uint16_t*)a.x + (int64_t)p * q.P * a.ldx; }

// stretches of dW's rows (the plan's are those of dz in two parts; the up to eight k-tiles of up to 256 rows in one part are one: cut_form)
int weight_stretches(const Plan& q, const Rows& rows) { return q.few && !rows.twice ? 1 : q.S_w; }

template <bool STORE>
rv_status launch_logits(const Plan& q, char* work, const rv_loss_desc& a, const Rows& rows, hipStream_t st) {
  const uint16_t* w = (const uint16_t*)a.w;
  const uint16_t* x = q.few ? rows_of_x(q, a, rows.p) : copy_of_x(q, work, rows.p);
  const int64_t ldx = q.few ? a.ldx : 32, x_bs = q.few ? 32 : 32ll * q.P;
  const LogitsOut o{STORE ? (uint16_t*)(work + q.e) : nullptr, (float2*)(work + q.stat), (float*)(work + q.target), q.P, q.R, q.V, q.Vp};
  const int most = q.T < q.P ? q.T : q.P;
  if (big_tiles(most, q.Vp, q.d)) {
    constexpr auto kern = logits_kernel<256, 256, 4, 8, STORE>;
    if (rv_allow_lds<kern>(kBigLds) != hipSuccess) return RV_E_DEVICE;
    // (fewer tile rows than all rows have may be dealt out in halves where those are not)
    hipLaunchKernelGGL(kern, dim3(div_up(most, 256) * div_up(q.Vp, 256) + 128), dim3(512), kBigLds, st, x, ldx, x_bs, w, q.ldw, q.d, rows, o);
  } else {
    constexpr auto kern = logits_kernel<128, 128, 4, 4, STORE>;
    if (rv_allow_lds<kern>(kMidLds) != hipSuccess) return RV_E_DEVICE;
    hipLaunchKernelGGL(kern, dim3(div_up(most, 128) * div_up(q.Vp, 128)), dim3(256), kMidLds, st, x, ldx, x_bs, w, q.ldw, q.d, rows, o);
  }
  return rv_launch_status();
}

template <auto Kern>
rv_status launch_512(const GradArgs& g, int grid, int lds, hipStream_t st) {
  if (rv_allow_lds<Kern>(lds) != hipSuccess) return RV_E_DEVICE;
  hipLaunchKernelGGL(Kern, dim3(grid), dim3(512), lds, st, g);
  return rv_launch_status();
}
// KIND of dW, -1: none
template <int KIND>
rv_status launch_grads(const Plan& q, char* work, const rv_loss_desc& a, const Rows& rows, hipStream_t st) {
  GradArgs g{};
  g.dz = (const uint16_t*)(work + q.e); g.xw = copy_of_x(q, work, rows.p); g.w = (const uint16_t*)a.w;
  g.ldw = q.ldw; g.rows = rows; g.d = q.d; g.Vp = q.Vp;
  // (fewer tile rows than all rows have, more stretches: never more workgroups than this, nor more memory)
  g.S_dx = q.dx.S; g.tiles_m = div_up(q.T < q.P ? q.T : q.P, q.dx.tile);
  g.dx_grid = a.dx ? g.tiles_m * div_up(q.d, q.dx.tile) * q.dx.S : 0;
  g.tail = (const uint16_t*)(work + q.tail); g.part = (float*)(work + q.part);
  g.S_w = weight_stretches(q, rows); g.sums = (float*)(work + q.acc);
  g.dw = (uint16_t*)a.dw; g.master = a.master; g.master_out = a.master_out; g.version = (uint16_t*)a.version;
  g.scale = a.scale; g.eta = a.eta * a.scale;
  g.info = a.master && rows.count ? (const RowInfo*)(work + q.info) : nullptr;
  const int w_tiles = div_up(q.V, WB) * div_up(q.d, WB), w_grid = KIND == 2 ? w_tiles * g.S_w : halved_grid(w_tiles);
  // together, but for an update in place: dx reads the weights that it overwrites
  const bool both = KIND >= 0 && a.dx && q.dx.tile == 128 &&
                    !(KIND == 1 && rv_overlap(a.w, 2 * (size_t)q.V * q.ldw, a.version, 2 * (size_t)q.V * q.d));
  if (a.dx && !both) {
    if (q.dx.tile == 256) RV_TRY((launch_512<input_grad_kernel<256>>(g, g.dx_grid, kBigLds, st)));
    else RV_TRY((launch_512<input_grad_kernel<128>>(g, g.dx_grid, kSplitLds, st)));
  }
  if constexpr (KIND >= 0) {
    g.w_first = w_grid <= (KIND == 2 ? 256 : 128) ? w_grid : 0;
    if (both) RV_TRY((launch_512<both_grads_kernel<KIND>>(g, g.dx_grid + w_grid, kBothLds, st)));
    else RV_TRY((launch_512<weight_grad_kernel<KIND>>(g, w_grid, kWeightLds, st)));
  }
  if (!a.dx) return RV_OK;
  const int64_t chunks = (int64_t)q.T * (q.d / 8);
  auto join = [&](auto k, int lanes) {
    hipLaunchKernelGGL(k, dim3((unsigned)((chunks * lanes + 255) / 256)), dim3(256), 0, st, g.part, rows, q.d, q.Vp / 32, q.dx.tile, g.S_dx, g.tiles_m,
                       a.scale, (uint16_t*)a.dx, a.lddx);
  };
  if (g.S_dx > 8) join(input_grad_join_kernel<8>, 8);
  else join(input_grad_join_kernel<1>, 1);
  return rv_launch_status();
}

bool misaligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) != 0; }

rv_status run(const rv_loss_desc& a, bool grads) {
  Plan q;
  if (!make_plan(q, a.T, a.d, a.V, a.ldw, a.rows, grads)) return RV_E_INVAL;
  if (!a.x || !a.w || !a.label || !a.loss || !a.work || a.work_bytes < q.bytes) return RV_E_INVAL;
  if (a.ldx < a.d || a.ldx % 8 || a.ldx > (1 << 20) || misaligned(a.x, 16) || misaligned(a.w, 16) || misaligned(a.work, 256) || misaligned(a.label, 8) ||
      misaligned(a.loss, 4) || misaligned(a.lse, 4) || misaligned(a.row_scale, 4)) return RV_E_INVAL;
  const bool update = grads && a.master;
  if (grads) {
    if (!a.dx && !a.dw && !a.master) return RV_E_INVAL;
    if (a.dx && (a.lddx < a.d || a.lddx % 8 || misaligned(a.dx, 16))) return RV_E_INVAL;
    if (a.dw && (a.master || misaligned(a.dw, 16))) return RV_E_INVAL;
    if ((a.master != nullptr) != (a.master_out != nullptr) || (a.master != nullptr) != (a.version != nullptr)) return RV_E_INVAL;
    if (misaligned(a.master, 16) || misaligned(a.master_out, 16) || misaligned(a.version, 16)) return RV_E_INVAL;
  }
  const hipStream_t st = (hipStream_t)a.stream;
  char* work = (char*)a.work;
  const uint16_t* w = (const uint16_t*)a.w;
  const int tail_rows = grads ? q.Vp - q.V / 32 * 32 : 0;
  if (!q.few) {
    int per = 4;
    while (per * 1024 < q.T) per *= 2;
    const int row_blocks = div_up(q.T, per);
    hipLaunchKernelGGL(gather_kernel, dim3(row_blocks + tail_rows), dim3(256), 0, st, (const uint16_t*)a.x, a.ldx, a.label, q.T, q.d, q.V, q.P, per,
                       (int*)(work + q.count), (int*)(work + q.pos), (int*)(work + q.idx), (int*)(work + q.lab), (uint16_t*)(work + q.xw), a.loss, a.lse, w,
                       q.ldw, (uint16_t*)(work + q.tail), row_blocks);
    RV_TRY(rv_launch_status());
  }
  const int strips = q.Vp / STRIP, most = q.T < q.P ? q.T : q.P;
  const int S_w = grads ? weight_stretches(q, rows_at(q, work, a, 0)) : 1;
  const bool cut = q.pieces > 1 || S_w > 1;                   // dW through fp32 sums
  for (int p = 0; p < q.pieces; ++p) {
    const Rows rows = rows_at(q, work, a, p);
    if (grads) RV_TRY(launch_logits<true>(q, work, a, rows, st));
    else RV_TRY(launch_logits<false>(q, work, a, rows, st));
    RowInfo* info = grads ? (RowInfo*)(work + q.info) : nullptr;
    hipLaunchKernelGGL(join_kernel, dim3(div_up(most, 16)), dim3(1024), 0, st, (const float2*)(work + q.stat), (const float*)(work + q.target), rows, strips,
                       a.row_scale, a.loss, a.lse, info);
    RV_TRY(rv_launch_status());
    if (!grads) continue;
    // strips a block takes one after the other: up to 8, fewer where that leaves fewer than 2048 blocks
    const int64_t dz_blocks = (int64_t)div_up(most, 64) * strips / 2048;
    const int per_dz = dz_blocks < 1 ? 1 : dz_blocks < 8 ? (int)dz_blocks : 8, strip_blocks = div_up(strips, per_dz);
    hipLaunchKernelGGL(dz_kernel, dim3(div_up(most, 64), strip_blocks + (q.few ? div_up(q.d / 32, 8) + tail_rows : 0)), dim3(256), 0, st,
                       (uint16_t*)(work + q.e), (const float2*)(work + q.stat), info, rows, strips, per_dz, strip_blocks,
                       copy_of_x(q, work, p), q.d, rows_of_x(q, a, p), a.ldx, w, q.ldw, (uint16_t*)(work + q.tail));
    RV_TRY(rv_launch_status());
    if (!a.dw && !update) RV_TRY(launch_grads<-1>(q, work, a, rows, st));
    else if (p > 0) RV_TRY(launch_grads<3>(q, work, a, rows, st));
    else if (cut) RV_TRY(launch_grads<2>(q, work, a, rows, st));
    else if (update) RV_TRY(launch_grads<1>(q, work, a, rows, st));
    else RV_TRY(launch_grads<0>(q, work, a, rows, st));
  }
  if (grads && (a.dw || update) && cut) {
    const int64_t n = (int64_t)q.V * q.d;
    hipLaunchKernelGGL(weight_grad_join_kernel, dim3((unsigned)((n / 8 + 255) / 256)), dim3(256), 0, st, (const float*)(work + q.acc), S_w,
                       rows_at(q, work, a, 0), q.pieces, n, (uint16_t*)a.dw, a.master, a.master_out, (uint16_t*)a.version, a.scale, a.eta * a.scale);
    RV_TRY(rv_launch_status());
  }
  return RV_OK;
}

}  // namespace

extern "C" rv_status rv_loss_work(int T, int d, int V, int64_t ldw, int rows, int gradients, size_t* bytes) {
  Plan q;
  if (!bytes || !make_plan(q, T, d, V, ldw, rows, gradients != 0)) return RV_E_INVAL;
  *bytes = q.bytes;
  return RV_OK;
}
extern "C" rv_status rv_loss_forward(const rv_loss_desc* a) { return a ? run(*a, false) : RV_E_INVAL; }
extern "C" rv_status rv_loss_step(const rv_loss_desc* a) { return a ? run(*a, true) : RV_E_INVAL; }

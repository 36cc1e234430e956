// The loss at the end of a chain of peers: softmax cross entropy of every token against a vocabulary, and its gradients.
//
//   z = x W^T           x bf16 [T, d], W bf16 [V, d], z in fp32 registers only
//   loss_t = lse_t - z[t, y_t],   lse_t = ln sum_v exp z[t, v]
//   dz[t, v] = g_t (exp(z[t, v] - lse_t) - [v = y_t])
//   dx = dz W,  dW = dz^T x       three products of 2 T V d flop each; the forward alone is one
//
// The logits are never written.  A wave of the first product holds 64 columns of the vocabulary - a strip - of its rows; it takes
// each row's maximum m over the strip (fp32) and writes the pair (m, sum of exp2(z log2 e - m)) and, for the gradients, the
// exponentials e themselves in bf16.  They lie in (0, 1] whatever the logits are, so that their rounding is half a step of the
// probability (2^-9 relative) - logits in bf16 would move it by |z| 2^-9.  The pairs of a row's strips are then joined to its
// lse, and  dz = e exp2(m - lse2) g  overwrites e in place, rounded once more: bf16 is what the matrix instructions take, and both
// roundings together stay below that of dx and dW themselves.  The label's own column gets  g expm1(z_y - lse)  from the fp32 logit:
// where the model is nearly certain, p - 1 from a rounded p would have no digits left.
// Computing z again for the gradients instead of keeping e would be a fourth product: 4 bytes of e and dz written and 6 read per
// logit are (at 5 TB/s) 2 ps, the product 2 d / 1.3 PFLOP/s = 1.6 ps at d 1024, 3.2 ps at 2048.
// One piece of rows is kept at a time (e and strips of `rows` rows, at most 2 GiB of e where the caller leaves the choice), so the work
// memory has a bound that does not grow with T; from the second piece on the weight gradient is added up in fp32.
//
// Rows whose label lies outside [0, V) - prompts, padding - take no part: a first kernel gathers the others, in order, into a copy of
// x without gaps, in blocks of 32 columns (rv_mat), and all kernels behind it go by the number of rows it counted.  So nothing
// such a row holds (NaN of an unwritten buffer) reaches a product, and a batch that is half prompt costs half.
#include <math.h>
#include "gemm_core.h"

namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr int STRIP = 64;
constexpr int64_t kMostE = 1ll << 30;    // elements of e, of a piece's rows: offsets in a product are 31 bits, and 2 GiB of work memory

// what a row of the piece needs in the backward
struct RowInfo { float lse2, g, at_label; int label; };

struct Plan {
  int T, d, V, Vp, P, pieces;            // V rounded up to whole strips; rows of a piece and their number
  bool grads;
  int64_t ldw;
  size_t count, pos, idx, lab, info, target, stat, xw, tail, e, part, acc, bytes;
};

__host__ __device__ inline int div_up(int a, int b) { return (a + b - 1) / b; }
__host__ __device__ inline int round_up(int a, int b) { return div_up(a, b) * b; }

// rows of piece p (device count n)
__device__ __forceinline__ int piece_rows(int n, int p, int P) {
  const int left = n - p * P;
  return left < P ? left : P;
}

// ---- rows that take part ----------------------------------------------------------------------
// A block takes `per` (up to 64) consecutive rows; where they go follows from the number of labels before them that take part, which
// it counts itself: T labels are 8 T bytes out of L2, at most a thousand blocks do it, and a scan of its own would be a launch more.
// pos[t] = place among the rows kept or -1; idx, lab: the other way round.  The block of the last rows leaves their number.
// Behind the row blocks, with `tail`: 64 rows that stand for rows V / 32 * 32 .. of W, zeros behind its last (see input_grad_kernel).
__global__ __launch_bounds__(256) void gather_kernel(const uint16_t* __restrict__ x, int64_t ldx, const int64_t* __restrict__ label, int T,
                                                     int d, int V, int P, int per, int* __restrict__ count, int* __restrict__ pos,
                                                     int* __restrict__ idx, int* __restrict__ lab, uint16_t* __restrict__ xw,
                                                     float* __restrict__ loss, float* __restrict__ lse, const uint16_t* __restrict__ w,
                                                     int64_t ldw, uint16_t* __restrict__ tail, int row_blocks) {
  const int tid = threadIdx.x, l = tid & 63;
  if ((int)blockIdx.x >= row_blocks) {
    const int r = blockIdx.x - row_blocks, v = V / 32 * 32 + r;
    for (int c = tid; c < d / 8; c += 256) {
      u32x4 u = {0u, 0u, 0u, 0u};
      if (v < V) u = *reinterpret_cast<const u32x4*>(w + (int64_t)v * ldw + c * 8);
      *reinterpret_cast<u32x4*>(tail + (int64_t)r * ldw + c * 8) = u;
    }
    return;
  }
  __shared__ int part[4], place[64];
  const int t0 = blockIdx.x * per, rows = T - t0 < per ? T - t0 : per;
  auto takes = [&](int64_t y) { return y >= 0 && y < V; };
  int before = 0;
  for (int t = tid; t < t0; t += 256) before += takes(label[t]) ? 1 : 0;
#pragma unroll
  for (int o = 32; o; o >>= 1) before += __shfl_xor(before, o, 64);
  if (l == 0) part[tid >> 6] = before;
  __syncthreads();
  if (tid < 64) {
    before = part[0] + part[1] + part[2] + part[3];
    const int64_t y = l < rows ? label[t0 + l] : -1;
    const bool in = takes(y);
    const uint64_t all = __builtin_amdgcn_ballot_w64(in);
    const int j = before + __popcll(all & ((1ull << l) - 1));
    place[l] = in ? j : -1;
    if (l < rows) {
      pos[t0 + l] = in ? j : -1;
      if (in) { idx[j] = t0 + l; lab[j] = (int)y; }
      else { loss[t0 + l] = 0.f; if (lse) lse[t0 + l] = 0.f; }
    }
    if (l == 0 && t0 + rows == T) *count = before + __popcll(all);
  }
  __syncthreads();
  const int chunks = rows * (d / 8);
  for (int i = tid; i < chunks; i += 256) {
    // four chunks of a block of 32 columns in neighbouring lanes, then the next row: what is written is runs of 64 bytes a row
    const int q = i & 3, r = (i >> 2) % rows, cb = (i >> 2) / rows, j = place[r];
    if (j < 0) continue;
    const int p = j / P, jr = j - p * P;
    const u32x4 u = *reinterpret_cast<const u32x4*>(x + (int64_t)(t0 + r) * ldx + cb * 32 + q * 8);
    *reinterpret_cast<u32x4*>(xw + (int64_t)p * P * d + (int64_t)cb * 32 * P + 32 * jr + q * 8) = u;
  }
}

// ---- the logits' product ----------------------------------------------------------------------
// Workgroup -> tile: down a column of tiles first, over the tile rows that are there (the count is known on the device alone: a map over
// the rows of all tokens would leave whole XCDs without work where half of the rows are out).
struct LogitsOut {
  uint16_t* e;         // [Vp / 32][P][32]
  float2* stat;        // [Vp / 64][P]
  float* target;       // [P] the label's logit
  const int* lab;      // [P]
  int P, V, Vp;
};

template <bool STORE, int TM, int TN>
__device__ __forceinline__ void strip_epilogue(const f32x4 (&acc)[TM][TN], const LogitsOut& o, int mw, int nw, int M) {
  static_assert(TN * 16 == STRIP, "a wave's columns are one strip");
  if (nw >= o.Vp || mw >= M) return;
  const int l = threadIdx.x & 63, grp = l >> 4, strip = nw / STRIP;
  const bool ragged = nw + STRIP > o.V;     // (wave-uniform)
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int row = mw + i * 16 + (l & 15);
    const bool ok = row < M;
    f32x4 a[TN];
#pragma unroll
    for (int c = 0; c < TN; ++c) {
      a[c] = acc[i][c];
      if (ragged) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (nw + c * 16 + 4 * grp + k >= o.V) a[c][k] = -INFINITY;
      }
    }
    const int y = ok ? o.lab[row] - nw : -1;
    if (__builtin_amdgcn_ballot_w64(y >= 0 && y < STRIP)) {   // few strips hold a label of their rows
      float at = 0.f;
      bool mine = false;
#pragma unroll
      for (int c = 0; c < TN; ++c)
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (y == c * 16 + 4 * grp + k) { at = a[c][k]; mine = true; }
      if (mine) o.target[row] = at;
    }
    float m = a[0][0];
#pragma unroll
    for (int c = 0; c < TN; ++c)
#pragma unroll
      for (int k = 0; k < 4; ++k) m = fmaxf(m, a[c][k]);
    m = fmaxf(m, __shfl_xor(m, 16, 64));
    m = fmaxf(m, __shfl_xor(m, 32, 64));
    m *= kLog2e;
    const float base = m == -INFINITY ? 0.f : m;   // (a strip of -inf alone: its sum is zero)
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < TN; ++c)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        a[c][k] = __builtin_amdgcn_exp2f(__fmaf_rn(a[c][k], kLog2e, -base));
        sum += a[c][k];
      }
    sum += __shfl_xor(sum, 16, 64);
    sum += __shfl_xor(sum, 32, 64);
    if (grp == 0 && ok) o.stat[(int64_t)strip * o.P + row] = float2{m, sum};
    if (STORE) {
      // Two quads of a lane are 16 columns apart; the swap of lane rows of 16 gives even rows eight consecutive columns of the first
      // quad and odd ones of the second, and a wave's 16 bytes a lane are one run of 1 KiB of the block of 32 columns.
#pragma unroll
      for (int b = 0; b < TN / 2; ++b) {
        u32x4 v;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const auto s = __builtin_amdgcn_permlane16_swap(rv_pack_bf16x2(a[2 * b][2 * h], a[2 * b][2 * h + 1]),
                                                          rv_pack_bf16x2(a[2 * b + 1][2 * h], a[2 * b + 1][2 * h + 1]), false, false);
          v[h] = s[0]; v[2 + h] = s[1];
        }
        const int col = grp & 1 ? 16 + 4 * (grp - 1) : 4 * grp;
        if (ok) *reinterpret_cast<u32x4*>(o.e + ((int64_t)(2 * strip + b) * o.P + row) * 32 + col) = v;
      }
    }
  }
}

template <int BM, int BN, int NS, int NW, bool STORE>
__global__ __launch_bounds__(64 * NW, 2) void logits_kernel(const uint16_t* __restrict__ xw, const uint16_t* __restrict__ w, int64_t ldw, int d,
                                                            const int* __restrict__ count, int p, LogitsOut o) {
  const int M = piece_rows(*count, p, o.P);
  if (M <= 0) return;
  const int vm = div_up(M, BM), vn = div_up(o.Vp, BN);
  const int id = blockIdx.x;
  if (id >= vm * vn) return;
  const int bm = id % vm, bn = id / vm;
  auto own = [&](const auto& acc, int m0, int n0, int wm0, int wn0) { strip_epilogue<STORE>(acc, o, m0 + wm0, n0 + wn0, M); };
  gemm_dtl_body<BM, BN, 32, NS, NW, false, false, EPI_OWN>(xw, 32, 32ll * o.P, w, ldw, 32, M, o.V, d, bm, bn, Epi{}, nullptr, 0, own);
}

// ---- strips joined to rows ----------------------------------------------------------------------
// 16 rows to a block, 64 lanes to a row: a strip's pairs of 16 rows are one line.
__global__ __launch_bounds__(1024) void join_kernel(const float2* __restrict__ stat, const float* __restrict__ target, const int* __restrict__ lab,
                                                    const int* __restrict__ idx, const int* __restrict__ count, int p, int P, int strips,
                                                    float scale, const float* __restrict__ row_scale, float* __restrict__ loss,
                                                    float* __restrict__ lse, RowInfo* __restrict__ info) {
  __shared__ float2 part[64][17];
  const int M = piece_rows(*count, p, P), r = threadIdx.x & 15, sl = threadIdx.x >> 4, row = blockIdx.x * 16 + r;
  if ((int)blockIdx.x * 16 >= M) return;
  auto join = [](float2 a, float2 b) {
    const float m = fmaxf(a.x, b.x), base = m == -INFINITY ? 0.f : m;
    return float2{m, a.y * __builtin_amdgcn_exp2f(a.x - base) + b.y * __builtin_amdgcn_exp2f(b.x - base)};
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
  const int t = idx[row];
  const float lse2 = v.x + __builtin_amdgcn_logf(v.y), ln = lse2 * kLn2, at = target[row];   // v_log_f32 is log2
  loss[t] = ln - at;
  if (lse) lse[t] = ln;
  if (info) {
    const float g = row_scale ? scale * row_scale[t] : scale;
    info[row] = RowInfo{lse2, g, g * expm1f(at - ln), lab[row]};
  }
}

// ---- e -> dz, in place ----------------------------------------------------------------------
// 64 rows to a block, four lanes to a row's 64 bytes of a block of columns, `per` strips one after the other.  Rows from the last one up to
// whole tiles of 32 become zeros, of dz here and of the copy of x below: the weight gradient's product walks over them.
__global__ __launch_bounds__(256) void dz_kernel(uint16_t* __restrict__ e, const float2* __restrict__ stat, const RowInfo* __restrict__ info,
                                                 const int* __restrict__ count, int p, int P, int strips, int per, uint16_t* __restrict__ xw, int d) {
  const int n = *count;
  int M = piece_rows(n, p, P);
  if (M <= 0) {
    if (p) return;
    M = 0;                                        // no row at all: one tile of zeros
  }
  const int row = blockIdx.x * 64 + threadIdx.x / 4, q = threadIdx.x & 3;
  const int end = round_up(M > 0 ? M : 1, 32);
  if (row >= end) return;
  const int s0 = blockIdx.y * per, s1 = s0 + per < strips ? s0 + per : strips;
  uint16_t* base = e + (int64_t)row * 32 + q * 8;
  const int64_t bs = 32ll * P;
  if (row >= M) {
    const u32x4 zero = {0u, 0u, 0u, 0u};
    for (int s = s0; s < s1; ++s) {
      *reinterpret_cast<u32x4*>(base + 2 * s * bs) = zero;
      *reinterpret_cast<u32x4*>(base + (2 * s + 1) * bs) = zero;
    }
    if (blockIdx.y == 0) {
      for (int cb = 0; cb < d / 32; ++cb) *reinterpret_cast<u32x4*>(xw + ((int64_t)cb * P + row) * 32 + q * 8) = zero;
    }
    return;
  }
  const RowInfo r = info[row];
#pragma unroll 2
  for (int s = s0; s < s1; ++s) {
    const float f = r.g * __builtin_amdgcn_exp2f(stat[(int64_t)s * P + row].x - r.lse2);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      u32x4* at = reinterpret_cast<u32x4*>(base + (2 * s + h) * bs);
      f32x4 v[2];
      bf16x8_to_f32(v, *at);
      const int y = r.label - ((2 * s + h) * 32 + q * 8);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k >> 2][k & 3] = y == k ? r.at_label : v[k >> 2][k & 3] * f;
      *at = f32_to_bf16x8(v);
    }
  }
}

// ---- dx ----------------------------------------------------------------------
// dx has few tiles and a contraction as long as the vocabulary: it is cut into S stretches where the tiles alone do not fill the chip.
// S is the count that wastes least of the last round of workgroups, each stretch counted as a 32nd of the walk for what its sums cost
// to write and read; the same on the device (which knows the rows) and on the host (the work memory of the worst case).
constexpr int kMostParts = 64, kMostPartTiles = 512;
__host__ __device__ inline int stretches(int tiles, int slots_log2, int nk) {
  const int slots = 1 << slots_log2;
  int best = 1, best_rounds = (tiles + slots - 1) >> slots_log2;
  for (int S = 2; S <= kMostParts && tiles * S <= kMostPartTiles && S * 8 <= nk; ++S) {
    const int rounds = (tiles * S + slots - 1) >> slots_log2;
    if (rounds * best * 33 < best_rounds * S * 32) { best = S; best_rounds = rounds; }
  }
  return best;
}
template <int BM, int BN, int NS, int NW, int SLOTS>
__global__ __launch_bounds__(64 * NW, 2) void input_grad_kernel(const uint16_t* __restrict__ dz, const uint16_t* __restrict__ w, int64_t ldw, int d,
                                                                int V, int Vp, const int* __restrict__ count, int p, int P,
                                                                const uint16_t* __restrict__ tail, float* __restrict__ part) {
  const int M = piece_rows(*count, p, P);
  if (M <= 0) return;
  const int vm = div_up(M, BM), vn = div_up(d, BN), tiles = vm * vn, nk = Vp / 32;
  const int S = stretches(tiles, SLOTS, nk);
  const int id = blockIdx.x;
  if (id >= tiles * S) return;
  const int s = id / tiles, in = id - s * tiles, bm = in % vm, bn = in / vm;
  const int k0 = (int)((int64_t)nk * s / S), k1 = (int)((int64_t)nk * (s + 1) / S);
  Epi out{};
  out.out = part + (int64_t)s * vm * BM * d; out.ldo = d;
  gemm_dtl_body<BM, BN, 32, NS, NW, false, true, EPI_F32, true>(dz + (int64_t)k0 * 32 * P, 32, 32ll * P, w + (int64_t)k0 * 32 * ldw, ldw, 32, M, d,
                                                                (k1 - k0) * 32, bm, bn, out, tail, V / 32 - k0);
}
// the stretches' sums, added in order and rounded, to the rows they belong to; zeros to the rows that take no part
template <int BM, int BN, int SLOTS>
__global__ __launch_bounds__(256) void input_grad_join_kernel(const float* __restrict__ part, const int* __restrict__ pos, const int* __restrict__ count,
                                                              int p, int P, int T, int d, int Vp, uint16_t* __restrict__ dx, int64_t lddx) {
  const int M = piece_rows(*count, p, P);
  if (M <= 0 && p) return;
  const int vm = div_up(M > 0 ? M : 0, BM), S = stretches(vm * div_up(d, BN), SLOTS, Vp / 32);
  const int64_t pitch = (int64_t)vm * BM * d;
  const int64_t chunk = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int per = d / 8;
  if (chunk >= (int64_t)T * per) return;
  const int t = (int)(chunk / per), c = (int)(chunk - (int64_t)t * per) * 8, j = pos[t];
  u32x4 r = {0u, 0u, 0u, 0u};
  if (j >= 0) {
    if (j / P != p) return;
    const float* src = part + (int64_t)(j - p * P) * d + c;
    f32x4 v[2] = {reinterpret_cast<const f32x4*>(src)[0], reinterpret_cast<const f32x4*>(src)[1]};
    for (int s = 1; s < S; ++s) {
      const f32x4* q = reinterpret_cast<const f32x4*>(src + s * pitch);
      v[0] += q[0]; v[1] += q[1];
    }
    r = f32_to_bf16x8(v);
  } else if (p) {
    return;
  }
  *reinterpret_cast<u32x4*>(dx + (int64_t)t * lddx + c) = r;
}

// ---- dW ----------------------------------------------------------------------
// KIND 0: bf16 dw.  1: the update of Eq. 2 on an fp32 master (w' = w - eta dW, one fused multiply-add) and its bf16 version.
// 2: fp32 sums of one of S stretches of the rows (few tiles), or of the first piece.  3: added to those of the pieces before.
constexpr int WB = 256, W_NS = 4, W_NW = 8;
__device__ __forceinline__ int row_stretches(int S, int nk) { return S < nk ? S : nk; }
template <int KIND>
__global__ __launch_bounds__(64 * W_NW, 2) void weight_grad_kernel(const uint16_t* __restrict__ dz, const uint16_t* __restrict__ xw, int d, int V, int Vp,
                                                                   const int* __restrict__ count, int p, int P, int S, float* __restrict__ sums,
                                                                   uint16_t* __restrict__ dw, const float* __restrict__ master,
                                                                   float* __restrict__ master_out, uint16_t* __restrict__ version, float eta) {
  int M = piece_rows(*count, p, P);
  if (M <= 0) {
    if (p) return;
    M = 1;                                        // (a tile of zeros: dz_kernel)
  }
  const int nk = div_up(M, 32), vm = div_up(V, WB), vn = div_up(d, WB), tiles = vm * vn, parts = KIND == 2 ? row_stretches(S, nk) : 1;
  const int id = blockIdx.x, s = id / tiles;
  if (s >= parts) return;
  const int in = id - s * tiles, bn = in % vn, bm = in / vn;
  const int k0 = nk * s / parts, k1 = nk * (s + 1) / parts;
  auto own = [&](const auto& acc, int m0, int n0, int wm0, int wn0) {
    constexpr int TM = WB / 2 / 16, TN = WB / (W_NW / 2) / 16;
    Epi o{};
    o.ldo = d;
    if constexpr (KIND == 0) {
      o.out = dw;
      write_tile_staged<WB, WB, 64 * W_NW, f32x4, TM, TN, EPI_BF16>(acc, o, m0, n0, wm0, wn0, V, d, dtl_smem);
    } else if constexpr (KIND == 1) {
      o.out = master_out; o.resid = master; o.ldr = d; o.out2 = version; o.eta = eta;
      f32_tile_through_lds<WB, WB, W_NW, f32x4, TM, TN, 2, true>(acc, o, m0, n0, wm0, wn0, V, d, dtl_smem);
    } else if constexpr (KIND == 2) {
      o.out = sums + (int64_t)s * V * d;
      write_tile<f32x4, TM, TN, EPI_F32>(acc, o, m0 + wm0, n0 + wn0, V, d);
    } else {
      o.out = sums; o.resid = sums; o.ldr = d;
      f32_tile_through_lds<WB, WB, W_NW, f32x4, TM, TN, 3, false>(acc, o, m0, n0, wm0, wn0, V, d, dtl_smem);
    }
  };
  // (the loads of dz run over whole strips, the results end at V)
  gemm_dtl_body<WB, WB, 32, W_NS, W_NW, true, true, EPI_OWN>(dz + (int64_t)k0 * 32 * 32, 32, 32ll * P, xw + (int64_t)k0 * 32 * 32, 32, 32ll * P, Vp, d,
                                                             (k1 - k0) * 32, bm, bn, Epi{}, nullptr, 0, own);
}
// fp32 sums of stretches or pieces -> dw, or the update
__global__ __launch_bounds__(256) void weight_grad_join_kernel(const float* __restrict__ sums, int S, const int* __restrict__ count, int pieces, int P, int64_t n,
                                                               uint16_t* __restrict__ dw, const float* __restrict__ master, float* __restrict__ master_out,
                                                               uint16_t* __restrict__ version, float eta) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (i >= n) return;
  int parts = 1;
  if (pieces == 1) {
    const int M = piece_rows(*count, 0, P);
    parts = row_stretches(S, div_up(M > 0 ? M : 1, 32));
  }
  f32x4 v[2] = {reinterpret_cast<const f32x4*>(sums + i)[0], reinterpret_cast<const f32x4*>(sums + i)[1]};
  for (int s = 1; s < parts; ++s) {
    const f32x4* q = reinterpret_cast<const f32x4*>(sums + s * n + i);
    v[0] += q[0]; v[1] += q[1];
  }
  if (dw) {
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
// ratio of the two as in gemm_bf16.hip)
bool big_tiles(int rows, int cols) {
  const int64_t b = (int64_t)div_up(rows, 256) * div_up(cols, 256), m = (int64_t)div_up(rows, 128) * div_up(cols, 128);
  return (double)((b + 255) / 256) * 65536 <= (double)((m + 511) / 512) * 2 * 16384 / 0.83;
}
bool big_input_grad(int rows, int d) { return rows > 128 && d > 128; }
int weight_stretches(int V, int d, int P) {
  const int tiles = div_up(V, WB) * div_up(d, WB);
  return stretches(tiles, 8, P / 32);
}

bool make_plan(Plan& q, int64_t T, int64_t d, int64_t V, int64_t ldw, int64_t rows, bool grads) {
  if (T < 1 || T > (1 << 24) || d < 64 || d % 64 || d > 16384 || V < 1 || V > (1 << 24) || ldw < d || ldw % 8 || rows < 0) return false;
  if (V * ldw >= (1ll << 31)) return false;       // offsets in the logits' product
  q.T = (int)T; q.d = (int)d; q.V = (int)V; q.Vp = round_up((int)V, STRIP); q.grads = grads; q.ldw = ldw;
  int64_t most = kMostE / (q.Vp > q.d ? q.Vp : q.d) / 64 * 64;
  if (rows && rows < most) most = (rows + 63) / 64 * 64;
  const int64_t whole = (T + 63) / 64 * 64;
  q.pieces = (int)((whole + most - 1) / most);
  // pieces of nearly the same size, of whole tiles where there are several
  int64_t P = whole;
  if (q.pieces > 1) {
    const int64_t step = most >= 512 ? 256 : 64;
    P = (T + q.pieces - 1) / q.pieces;
    P = (P + step - 1) / step * step;
    if (P > most) P = most;
    q.pieces = (int)((T + P - 1) / P);
  }
  q.P = (int)P;
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t was = at; at += (bytes + 255) / 256 * 256; return was; };
  const size_t all = (size_t)q.pieces * P;
  q.count = take(4);
  q.pos = take(4 * all); q.idx = take(4 * all); q.lab = take(4 * all);
  q.target = take(4 * P);
  q.stat = take((size_t)8 * (q.Vp / STRIP) * P);
  q.xw = take((size_t)2 * all * d);
  if (grads) {
    q.info = take(sizeof(RowInfo) * P);
    q.tail = take((size_t)2 * 64 * ldw);
    q.e = take((size_t)2 * P * q.Vp);
    // dx: the rows' tiles, or kMostPartTiles of them where the contraction is cut
    const int b = big_input_grad(q.P, q.d) ? 256 : 128;
    const size_t tiles = (size_t)div_up(q.P, b) * div_up(q.d, b);
    q.part = take((tiles > kMostPartTiles ? tiles : kMostPartTiles) * b * b * 4);
    q.acc = 0;
    const int S = q.pieces > 1 ? 1 : weight_stretches(q.V, q.d, q.P);
    if (q.pieces > 1 || S > 1) q.acc = take((size_t)4 * S * V * d);
  }
  q.bytes = at;
  return true;
}

template <auto Kern>
hipError_t allow_lds(int bytes) {
  static const hipError_t done = hipFuncSetAttribute((const void*)Kern, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  return done;
}
constexpr int kBigLds = 4 * 2 * dtl_tile_bytes(256, 32), kMidLds = 4 * 2 * dtl_tile_bytes(128, 32);
constexpr int kWeightLds = WB * stage_pitch(WB) > upd_image_bytes(WB, WB) ? WB * stage_pitch(WB) : upd_image_bytes(WB, WB);
static_assert(kWeightLds >= kBigLds && kWeightLds <= 160 * 1024, "LDS of one CU");

template <bool STORE>
rv_status launch_logits(const Plan& q, char* work, const uint16_t* w, int p, hipStream_t st) {
  const uint16_t* xw = (const uint16_t*)(work + q.xw) + (int64_t)p * q.P * q.d;
  const LogitsOut o{STORE ? (uint16_t*)(work + q.e) : nullptr, (float2*)(work + q.stat), (float*)(work + q.target), (const int*)(work + q.lab) + (int64_t)p * q.P,
                    q.P, q.V, q.Vp};
  const int* count = (const int*)(work + q.count);
  const int rows = q.T < q.P ? q.T : q.P;
  if (big_tiles(rows, q.Vp)) {
    constexpr auto kern = logits_kernel<256, 256, 4, 8, STORE>;
    if (allow_lds<kern>(kBigLds) != hipSuccess) return RV_E_DEVICE;
    hipLaunchKernelGGL(kern, dim3(div_up(rows, 256) * div_up(q.Vp, 256)), dim3(512), kBigLds, st, xw, w, q.ldw, q.d, count, p, o);
  } else {
    constexpr auto kern = logits_kernel<128, 128, 4, 4, STORE>;
    if (allow_lds<kern>(kMidLds) != hipSuccess) return RV_E_DEVICE;
    hipLaunchKernelGGL(kern, dim3(div_up(rows, 128) * div_up(q.Vp, 128)), dim3(256), kMidLds, st, xw, w, q.ldw, q.d, count, p, o);
  }
  return rv_launch_status();
}

template <int B, int NW, int SLOTS, int LDS>
rv_status launch_input_grad(const Plan& q, char* work, const rv_loss_desc& a, int p, hipStream_t st) {
  constexpr auto kern = input_grad_kernel<B, B, 4, NW, SLOTS>;
  if (allow_lds<kern>(LDS) != hipSuccess) return RV_E_DEVICE;
  const int* count = (const int*)(work + q.count);
  float* part = (float*)(work + q.part);
  const int rows = q.T < q.P ? q.T : q.P, vm = div_up(rows, B), vn = div_up(q.d, B);
  int grid = vm * vn;                             // of the largest launch that a number of rows up to `rows` asks for
  for (int m = 1; m <= vm; ++m) {
    const int n = m * vn * stretches(m * vn, SLOTS, q.Vp / 32);
    if (n > grid) grid = n;
  }
  hipLaunchKernelGGL(kern, dim3(grid), dim3(64 * NW), LDS, st, (const uint16_t*)(work + q.e), (const uint16_t*)a.w, q.ldw, q.d, q.V, q.Vp, count, p,
                     q.P, (const uint16_t*)(work + q.tail), part);
  RV_TRY(rv_launch_status());
  const int64_t chunks = (int64_t)q.T * (q.d / 8);
  hipLaunchKernelGGL((input_grad_join_kernel<B, B, SLOTS>), dim3((unsigned)((chunks + 255) / 256)), dim3(256), 0, st, part, (const int*)(work + q.pos), count, p,
                     q.P, q.T, q.d, q.Vp, (uint16_t*)a.dx, a.lddx);
  return rv_launch_status();
}

template <int KIND>
rv_status launch_weight_grad(const Plan& q, char* work, const rv_loss_desc& a, int p, int S, hipStream_t st) {
  constexpr auto kern = weight_grad_kernel<KIND>;
  if (allow_lds<kern>(kWeightLds) != hipSuccess) return RV_E_DEVICE;
  const int tiles = div_up(q.V, WB) * div_up(q.d, WB);
  hipLaunchKernelGGL(kern, dim3(tiles * S), dim3(64 * W_NW), kWeightLds, st, (const uint16_t*)(work + q.e),
                     (const uint16_t*)(work + q.xw) + (int64_t)p * q.P * q.d, q.d, q.V, q.Vp, (const int*)(work + q.count), p, q.P, S, (float*)(work + q.acc),
                     (uint16_t*)a.dw, a.master, a.master_out, (uint16_t*)a.version, a.eta);
  return rv_launch_status();
}

bool misaligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) != 0; }

rv_status run(const rv_loss_desc& a, bool grads) {
  Plan q;
  if (!make_plan(q, a.T, a.d, a.V, a.ldw, a.rows, grads)) return RV_E_INVAL;
  if (!a.x || !a.w || !a.label || !a.loss || !a.work || a.work_bytes < q.bytes) return RV_E_INVAL;
  if (a.ldx < a.d || a.ldx % 8 || misaligned(a.x, 16) || misaligned(a.w, 16) || misaligned(a.work, 256) || misaligned(a.label, 8) ||
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
  int* count = (int*)(work + q.count);
  int* lab = (int*)(work + q.lab);
  int per = 4;
  while (per < 64 && per * 1024 < q.T) per *= 2;
  const int row_blocks = div_up(q.T, per), tail_blocks = grads ? q.Vp - q.V / 32 * 32 : 0;
  hipLaunchKernelGGL(gather_kernel, dim3(row_blocks + tail_blocks), dim3(256), 0, st, (const uint16_t*)a.x, a.ldx, a.label, q.T, q.d, q.V, q.P, per, count,
                     (int*)(work + q.pos), (int*)(work + q.idx), lab, (uint16_t*)(work + q.xw), a.loss, a.lse, w, q.ldw,
                     grads ? (uint16_t*)(work + q.tail) : nullptr, row_blocks);
  RV_TRY(rv_launch_status());
  const int strips = q.Vp / STRIP, S = grads && q.pieces == 1 ? weight_stretches(q.V, q.d, q.P) : 1;
  const int rows = q.T < q.P ? q.T : q.P;
  for (int p = 0; p < q.pieces; ++p) {
    if (grads) RV_TRY(launch_logits<true>(q, work, w, p, st));
    else RV_TRY(launch_logits<false>(q, work, w, p, st));
    RowInfo* info = grads ? (RowInfo*)(work + q.info) : nullptr;
    hipLaunchKernelGGL(join_kernel, dim3(div_up(rows, 16)), dim3(1024), 0, st, (const float2*)(work + q.stat), (const float*)(work + q.target),
                       lab + (int64_t)p * q.P, (const int*)(work + q.idx) + (int64_t)p * q.P, count, p, q.P, strips, a.scale, a.row_scale, a.loss, a.lse, info);
    RV_TRY(rv_launch_status());
    if (!grads) continue;
    const int per_dz = 8;
    hipLaunchKernelGGL(dz_kernel, dim3(div_up(rows, 64), div_up(strips, per_dz)), dim3(256), 0, st, (uint16_t*)(work + q.e), (const float2*)(work + q.stat), info,
                       count, p, q.P, strips, per_dz, (uint16_t*)(work + q.xw) + (int64_t)p * q.P * q.d, q.d);
    RV_TRY(rv_launch_status());
    if (a.dx) {
      if (big_input_grad(q.P, q.d)) RV_TRY((launch_input_grad<256, 8, 8, kBigLds>(q, work, a, p, st)));
      else RV_TRY((launch_input_grad<128, 4, 9, kMidLds>(q, work, a, p, st)));
    }
    if (!a.dw && !update) continue;
    if (q.pieces == 1 && S == 1) {
      if (update) RV_TRY(launch_weight_grad<1>(q, work, a, p, 1, st));
      else RV_TRY(launch_weight_grad<0>(q, work, a, p, 1, st));
    } else if (p == 0) {
      RV_TRY(launch_weight_grad<2>(q, work, a, p, S, st));
    } else {
      RV_TRY(launch_weight_grad<3>(q, work, a, p, 1, st));
    }
  }
  if (grads && (a.dw || update) && (q.pieces > 1 || S > 1)) {
    const int64_t n = (int64_t)q.V * q.d;
    hipLaunchKernelGGL(weight_grad_join_kernel, dim3((unsigned)((n / 8 + 255) / 256)), dim3(256), 0, st, (const float*)(work + q.acc), S, count, q.pieces, q.P, n,
                       (uint16_t*)a.dw, a.master, a.master_out, (uint16_t*)a.version, a.eta);
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

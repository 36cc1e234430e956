// Attention of a decoder's tokens to an encoder's states of another length, forward and backward: bf16 operands, fp32 scores, softmax
// statistics and sums.
//
//   s = q k^T / sqrt(dh),  p = softmax over the keys of the sequence,  o = p v
//   dv = p^T do,  ds = p (do v^T - rowsum(do o)),  dq = ds k / sqrt(dh),  dk = ds^T q / sqrt(dh)
//
// The `share` query heads of a key/value head see the same keys: their tokens are taken as ONE list of share * Sq rows, row r being
// token r % Sq of head r / Sq.  So a key/value head is streamed once for all of them, the gradients of a shared head are sums over
// one list in one workgroup, without atomics, and a single token of eight heads is eight rows of a matrix product.
//
// Scores are formed transposed to the side that a wave owns, as in attention.hip: the owned index (32 rows, or 32 keys in the dK/dV
// kernel) is the lane, the streamed one runs over the 16 registers of an accumulator; row statistics are scalars of a lane and the
// probabilities are already the B operand of the second product.  The streamed side goes global -> LDS directly, in tiles of 64 rows,
// through a ring of slots with one barrier a tile; 16-byte chunks are permuted by row (swizzle) so that ONE copy of a tile serves both
// the reads of whole rows and the transposing reads without bank conflicts.
// Keys behind a sequence's length are never read: a tile's rows are clamped to the last key, whose repeats are masked by a select.
// The work is cut along the streamed side where the rows alone do not fill the chip; the parts' sums (with their maxima, in the
// forward) are joined by a second kernel in a fixed order.
#include <math.h>
#include "attention_core.h"

namespace {

struct CrossArgs {
  const uint16_t* q; const uint16_t* k; const uint16_t* v;
  int64_t ldq, ldk, ldv;
  const int* klen;                       // device [B] or null
  uint16_t* out; int64_t ldo;
  float* lse2;                           // [B][Hkv][R]
  // backward
  const uint16_t* o; const uint16_t* dout; int64_t lddo;
  uint16_t* dq; uint16_t* dk; uint16_t* dv;
  int64_t lddq, lddk, lddv;
  float* stat_lse; float* stat_d;        // [B][Hkv][Rp]: see cross_stat_kernel
  float* part; float2* part_ml;          // forward: sums of the parts
  float* q_part; float* kv_part;         // backward
  int B, Sq, Sk, share, Hkv, R, Rp, kv_grid;
  Grid fwd, bq, bkv;
  float c2, scale;                       // log2(e) / sqrt(dh), 1 / sqrt(dh)
};

__device__ __forceinline__ int keys_at(const CrossArgs& a, int b) {
  if (!a.klen) return a.Sk;
  const int n = a.klen[b];
  return n < 0 ? 0 : n < a.Sk ? n : a.Sk;
}
__device__ __forceinline__ int keys_of(const CrossArgs& a, int b) { return __builtin_amdgcn_readfirstlane(keys_at(a, b)); }   // (b: wave-uniform)
// What the sums over n keys end with, from their running maximum m and sum tot: the factor of the output and the row's log2-sum.  Without
// keys 0 and -inf; keys whose scores are all -inf have no softmax, 0 / 0, and the backward has to see that.
__device__ __forceinline__ float inverse(int n, float tot) { return n == 0 ? 0.f : 1.0f / tot; }
__device__ __forceinline__ float log2_sum(int n, float m, float tot) {
  return n == 0 ? -INFINITY : tot == 0.f ? NAN : m + __builtin_amdgcn_logf(tot);   // v_log_f32 is log2
}
// element offset of row r of (b, hkv) in a matrix of tokens whose rows are ld apart, heads of DH columns
template <int DH>
__device__ __forceinline__ int64_t row_at(const CrossArgs& a, int b, int h, int r, int64_t ld) {
  const int g = r / a.Sq, t = r - g * a.Sq;
  return ((int64_t)b * a.Sq + t) * ld + (h * a.share + g) * DH;
}

// Softmax of a tile of scores s (SUBS x 32 keys from k0 on) with the running maximum m and sum l of a lane's row, in base 2: s becomes
// exp2(s c2 - m); the factor for what was summed before is returned.  The empty asm keeps the mask of the last tile behind its branch:
// without it the compiler made selects of it that every tile paid for, a third of a tile's vector instructions.
template <int SUBS>
__device__ __forceinline__ float softmax_tile(f32x16 (&s)[SUBS], float c2, int k0, int n, float& m, float& lsum) {
  const int grp = (threadIdx.x & 63) >> 5;
  if (k0 + SUBS * 32 > n) {            // (wave-uniform) only the last tile ends inside
    asm volatile("");
#pragma unroll
    for (int sub = 0; sub < SUBS; ++sub)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (k0 + sub * 32 + acc_row(r, grp) >= n) s[sub][r] = -INFINITY;
  }
  float mx = s[0][0];
#pragma unroll
  for (int sub = 0; sub < SUBS; ++sub)
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[sub][r]);
  mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
  const float mn = fmaxf(m, mx * c2), base = mn == -INFINITY ? 0.f : mn;   // (scores of -inf alone so far: nothing yet)
  const float alpha = __builtin_amdgcn_exp2f(m - base);
  m = mn;
  float ps = 0.f;
#pragma unroll
  for (int sub = 0; sub < SUBS; ++sub)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float p = __builtin_amdgcn_exp2f(__fmaf_rn(s[sub][r], c2, -base));
      s[sub][r] = p;
      ps += p;
    }
  lsum = lsum * alpha + ps;
  return alpha;
}

// ---- forward ----------------------------------------------------------------------------------
// Four waves of 32 rows, two slots: two workgroups (heads of 128) or four (64) to a CU.  4 x 4096 x 4096 tokens of 16 heads of 128 572 us,
// 961 TFLOP/s, of 64 325 us, 846; the same with operands of zeros 427 and 264 us: the power cap bounds it, as it bounds the library's product
// (1.37 PFLOP/s) - the matrix cores are busy 49 % of cycles, vector instructions and LDS take their part of the power.  Eight waves and three
// slots: 561 / 314 us there, 4 % slower over sequences of unequal lengths.
template <int DH, int NW, int NS>
__global__ __launch_bounds__(64 * NW, NW / 4) void cross_fwd_kernel(CrossArgs a) {
  char* smem = dtl_smem;
  constexpr int SLOT = 2 * kTileBytes<DH>;               // keys, values
  const int parts = a.fwd.parts;
  Where w;
  if (!where(a, a.fwd, blockIdx.x, gridDim.x, w)) return;
  const int n = keys_of(a, w.b), nt = (n + TILE - 1) / TILE;
  const int t0 = (int)((int64_t)nt * w.part / parts), t1 = (int)((int64_t)nt * (w.part + 1) / parts);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, grp = l >> 5;
  const int r = w.block * OWN * NW + wave * OWN + (l & 31);
  const bool active = w.block * OWN * NW + wave * OWN < a.R;
  const int rc = r < a.R ? r : a.R - 1;
  const uint16_t* K = a.k + (int64_t)w.b * a.Sk * a.ldk + w.h * DH;
  const uint16_t* V = a.v + (int64_t)w.b * a.Sk * a.ldv + w.h * DH;

  f32x16 o[DH / 32];
  clear(o);
  float m = -INFINITY, lsum = 0.f;

  const TileLoads<DH, NW> loads(wave);
  constexpr int LPT = 2 * TileLoads<DH, NW>::N;
  auto issue = [&](int t) {
    char* to = smem + (t - t0) % NS * SLOT;
    loads.keys(K, a.ldk, t * TILE, n, to);
    loads.keys(V, a.ldv, t * TILE, n, to + kTileBytes<DH>);
  };
#pragma unroll
  for (int i = 0; i < NS - 1; ++i)
    if (t0 + i < t1) issue(t0 + i);
  Frag qf[DH / 16];
  load_owned<DH>(qf, a.q + row_at<DH>(a, w.b, w.h, rc, a.ldq));
  settle(qf);
  auto tile = [&](int k0, const char* Ks) {
    const char* Vs = Ks + kTileBytes<DH>;
    f32x16 s[2];
    clear(s);
    in_a_row<DH / 8, DH == 128 ? 6 : 3>([&](int i) { return frag_rows<DH>(Ks, i % 2 * 32, i / 2); },
                        [&](int i, const Frag& f) { s[i % 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, qf[i / 2], s[i % 2], 0, 0, 0); });
    const float alpha = softmax_tile(s, a.c2, k0, n, m, lsum);
    if (__builtin_amdgcn_ballot_w64(alpha != 1.0f)) {    // maxima that have settled leave the sums as they are
#pragma unroll
      for (int dt = 0; dt < DH / 32; ++dt) o[dt] *= alpha;
    }
#pragma unroll
    for (int sub = 0; sub < 2; ++sub)
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        const Frag p = pack_frag(s[sub], ks);
#pragma unroll
        for (int dt = 0; dt < DH / 32; ++dt)
          o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_cols<DH>(Vs, sub * 32 + ks * 16, dt * 32), p, o[dt], 0, 0, 0);
      }
  };
  for (int t = t0; t < t1; ++t) {
    if (t + NS - 2 < t1) wait_loads<LPT * (NS - 2)>();
    else wait_loads<0>();
    __syncthreads();                                     // tile t is there, and everyone has left tile t - 1
    if (t + NS - 1 < t1) issue(t + NS - 1);
    if (!active) continue;
    tile(t * TILE, smem + (t - t0) % NS * SLOT);
  }
  if (!active || r >= a.R) return;
  const float tot = lsum + __shfl_xor(lsum, 32, 64);
  if (parts == 1) {
    store_owned<DH>(o, inverse(n, tot), a.out + row_at<DH>(a, w.b, w.h, r, a.ldo));
    if (grp == 0) a.lse2[(int64_t)w.unit * a.R + r] = log2_sum(n, m, tot);
  } else {
    const int64_t at = ((int64_t)w.part * a.B * a.Hkv + w.unit) * a.R + r;
    store_owned32<DH>(o, a.part + at * DH);
    if (grp == 0) a.part_ml[at] = float2{m, tot};
  }
}

// Up to 32 rows to a key/value head - single tokens: bound by reading the keys and values once.  Each of the waves (two for heads of 128, four for
// 64) walks over tiles of 32 keys of its own, with a ring of its own and no barrier; their sums meet in LDS at the end.  Rings of 64 KB, so that two
// workgroups share a CU: two tokens of 32 heads over 8 and 100001 keys 145 us, 5.7 TB/s (a large copy 5.0); 16 tokens of 16 heads of 64, up to
// 1500 keys, 17 us.
constexpr int TOKEN_KEYS = 32, kTokenGrid = 256;
template <int DH> constexpr int kTokenWaves = DH == 128 ? 2 : 4;
constexpr int kTokenSlots = 2;
template <int DH> constexpr int kTokenRing = kTokenSlots * 2 * TOKEN_KEYS * DH * 2;   // of a wave
template <int DH>
__global__ __launch_bounds__(64 * kTokenWaves<DH>) void cross_token_kernel(CrossArgs a) {
  constexpr int TOKEN_NW = kTokenWaves<DH>, NS = kTokenSlots, HALF = TOKEN_KEYS * DH * 2, SLOT = 2 * HALF;
  const int parts = a.fwd.parts;
  Where w;
  if (!where(a, a.fwd, blockIdx.x, gridDim.x, w)) return;
  const int n = keys_of(a, w.b), nt = (n + TOKEN_KEYS - 1) / TOKEN_KEYS;
  const int t0 = (int)((int64_t)nt * w.part / parts), t1 = (int)((int64_t)nt * (w.part + 1) / parts);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, grp = l >> 5, r = l & 31;
  char* ring = dtl_smem + wave * kTokenRing<DH>;
  const uint16_t* K = a.k + (int64_t)w.b * a.Sk * a.ldk + w.h * DH;
  const uint16_t* V = a.v + (int64_t)w.b * a.Sk * a.ldv + w.h * DH;
  f32x16 o[DH / 32];
  clear(o);
  float m = -INFINITY, lsum = 0.f;
  const TileLoads<DH, 1, TOKEN_KEYS> loads(0);
  constexpr int LPT = 2 * TileLoads<DH, 1, TOKEN_KEYS>::N;
  const int mine = t1 - t0 > wave ? (t1 - t0 - wave + TOKEN_NW - 1) / TOKEN_NW : 0;      // tiles t0 + wave, + TOKEN_NW, ...
  auto issue = [&](int i) {
    char* to = ring + i % NS * SLOT;
    const int k0 = (t0 + wave + i * TOKEN_NW) * TOKEN_KEYS;
    loads.keys(K, a.ldk, k0, n, to);
    loads.keys(V, a.ldv, k0, n, to + HALF);
  };
#pragma unroll
  for (int i = 0; i < NS - 1; ++i)
    if (i < mine) issue(i);
  Frag qf[DH / 16];
  load_owned<DH>(qf, a.q + row_at<DH>(a, w.b, w.h, r < a.R ? r : a.R - 1, a.ldq));
  settle(qf);
  for (int i = 0; i < mine; ++i) {
    // the slot that is filled next was read a tile ago; its reads have come back before the load goes out
    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
    if (i + NS - 1 < mine) { issue(i + NS - 1); wait_loads<LPT * (NS - 1)>(); }
    else wait_loads<0>();
    const char* Ks = ring + i % NS * SLOT;
    const char* Vs = Ks + HALF;
    f32x16 s[1];
    clear(s);
    in_a_row<DH / 16, 4>([&](int i) { return frag_rows<DH>(Ks, 0, i); },
                         [&](int i, const Frag& f) { s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, qf[i], s[0], 0, 0, 0); });
    const int k0 = (t0 + wave + i * TOKEN_NW) * TOKEN_KEYS;
    const float alpha = softmax_tile(s, a.c2, k0, n, m, lsum);
    if (__builtin_amdgcn_ballot_w64(alpha != 1.0f)) {
#pragma unroll
      for (int dt = 0; dt < DH / 32; ++dt) o[dt] *= alpha;
    }
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      const Frag p = pack_frag(s[0], ks);
#pragma unroll
      for (int dt = 0; dt < DH / 32; ++dt)
        o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_cols<DH>(Vs, ks * 16, dt * 32), p, o[dt], 0, 0, 0);
    }
  }
  lsum += __shfl_xor(lsum, 32, 64);
  // the waves' sums: registers through LDS, an equal share of them to each wave
  __syncthreads();
  float* image = reinterpret_cast<float*>(dtl_smem);     // [wave][DH / 2][64], then the pairs
  float2* ml = reinterpret_cast<float2*>(image + TOKEN_NW * (DH / 2) * 64);
#pragma unroll
  for (int dt = 0; dt < DH / 32; ++dt)
#pragma unroll
    for (int x = 0; x < 16; ++x) image[(wave * (DH / 2) + dt * 16 + x) * 64 + l] = o[dt][x];
  if (grp == 0) ml[wave * 32 + r] = float2{m, lsum};
  __syncthreads();
  float top = -INFINITY, tot = 0.f, f[TOKEN_NW];
#pragma unroll
  for (int i = 0; i < TOKEN_NW; ++i) top = fmaxf(top, ml[i * 32 + r].x);
  const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
  for (int i = 0; i < TOKEN_NW; ++i) {
    f[i] = __builtin_amdgcn_exp2f(ml[i * 32 + r].x - base);
    tot += ml[i * 32 + r].y * f[i];
  }
  if (r >= a.R) return;
  const int64_t at = ((int64_t)w.part * a.B * a.Hkv + w.unit) * a.R + r;
  const float inv = inverse(n, tot);
  uint16_t* out = a.out + row_at<DH>(a, w.b, w.h, r, a.ldo);
  constexpr int PER = DH / 2 / TOKEN_NW;                 // registers of a wave's share
#pragma unroll
  for (int x = 0; x < PER; x += 4) {
    const int reg = wave * PER + x;
    f32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = 0.f;
#pragma unroll
      for (int i = 0; i < TOKEN_NW; ++i) v[e] += image[(i * (DH / 2) + reg + e) * 64 + l] * f[i];
    }
    const int col = (reg >> 4) * 32 + acc_row(reg & 15, grp);
    if (parts > 1) *reinterpret_cast<f32x4*>(a.part + at * DH + col) = v;
    else *reinterpret_cast<u32x2*>(out + col) = u32x2{rv_pack_bf16x2(v.x * inv, v.y * inv), rv_pack_bf16x2(v.z * inv, v.w * inv)};
  }
  if (wave != 0 || grp != 0) return;
  if (parts > 1) a.part_ml[at] = float2{top, tot};
  else a.lse2[(int64_t)w.unit * a.R + r] = log2_sum(n, top, tot);
}

// parts -> out, lse2.  Eight columns to a lane; LANES lanes share the parts of one (a chain of up to 64 round trips else: single tokens of 8
// heads over 32 parts took 20 us with one lane).
template <int DH, int LANES>
__global__ __launch_bounds__(256) void cross_join_kernel(CrossArgs a) {
  constexpr int W = 256 / LANES;                         // column groups of a block
  static_assert(W % (DH / 8) == 0, "whole rows");
  __shared__ f32x4 sums[2][256];
  __shared__ float2 pairs[256];
  const int64_t rows = (int64_t)a.B * a.Hkv * a.R;
  const int lane = threadIdx.x / W;
  const int64_t i = (int64_t)blockIdx.x * W + threadIdx.x % W, row = i / (DH / 8);
  const int c = (int)(i % (DH / 8)) * 8;
  float m = -INFINITY, tot = 0.f;
  f32x4 v[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
  auto add = [&](float2 ml, f32x4 x, f32x4 y) {
    const float mn = fmaxf(m, ml.x), base = mn == -INFINITY ? 0.f : mn;
    const float was = __builtin_amdgcn_exp2f(m - base), f = __builtin_amdgcn_exp2f(ml.x - base);
    v[0] = v[0] * was + x * f;
    v[1] = v[1] * was + y * f;
    tot = tot * was + ml.y * f;
    m = mn;
  };
  if (row < rows) {
#pragma unroll 4
    for (int s = lane; s < a.fwd.parts; s += LANES) {
      const int64_t at = s * rows + row;
      const f32x4* p = reinterpret_cast<const f32x4*>(a.part + at * DH + c);
      add(a.part_ml[at], p[0], p[1]);
    }
  }
  if (LANES > 1) {
    sums[0][threadIdx.x] = v[0]; sums[1][threadIdx.x] = v[1]; pairs[threadIdx.x] = float2{m, tot};
    __syncthreads();
    if (lane) return;
#pragma unroll
    for (int x = 1; x < LANES; ++x) add(pairs[threadIdx.x + x * W], sums[0][threadIdx.x + x * W], sums[1][threadIdx.x + x * W]);
  }
  if (row >= rows) return;
  const int unit = (int)(row / a.R), r = (int)(row - (int64_t)unit * a.R), n = keys_at(a, unit / a.Hkv);
  const float inv = inverse(n, tot);
  v[0] *= inv; v[1] *= inv;
  *reinterpret_cast<u32x4*>(a.out + row_at<DH>(a, unit / a.Hkv, unit % a.Hkv, r, a.ldo) + c) = f32_to_bf16x8(v);
  if (c == 0) a.lse2[row] = log2_sum(n, m, tot);
}

// ---- backward ----------------------------------------------------------------------------------
// What the accumulators of the scores and of do v^T begin with, for every row in the order of the list: -lse / c2, so that a probability is
// exp2(c2 acc), and -D = -rowsum(do o), so that acc is dp - D.  Behind the last row and for a row without keys -inf, which makes the
// probabilities zero, and 0.
template <int DH>
__global__ __launch_bounds__(256) void cross_stat_kernel(CrossArgs a) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / (DH / 8);
  const int c = (int)(i % (DH / 8)) * 8;
  if (row >= (int64_t)a.B * a.Hkv * a.Rp) return;         // (whole rows: DH / 8 lanes go together)
  const int unit = (int)(row / a.Rp), r = (int)(row - (int64_t)unit * a.Rp);
  float d = 0.f, lse = INFINITY;
  if (r < a.R) {
    const int b = unit / a.Hkv, h = unit % a.Hkv;
    f32x4 x[2], y[2];
    bf16x8_to_f32(x, *reinterpret_cast<const u32x4*>(a.o + row_at<DH>(a, b, h, r, a.ldo) + c));
    bf16x8_to_f32(y, *reinterpret_cast<const u32x4*>(a.dout + row_at<DH>(a, b, h, r, a.lddo) + c));
#pragma unroll
    for (int k = 0; k < 8; ++k) d = __fmaf_rn(x[k >> 2][k & 3], y[k >> 2][k & 3], d);
    lse = a.lse2[(int64_t)unit * a.R + r];
    lse = lse == -INFINITY ? INFINITY : lse / a.c2;
  }
#pragma unroll
  for (int o = 1; o < DH / 8; o *= 2) d += __shfl_xor(d, o, 64);
  if (c == 0) { a.stat_lse[row] = -lse; a.stat_d[row] = lse == INFINITY ? 0.f : -d; }
}

// dQ: a wave owns 32 rows, keys and values stream.  Three products a pair of tiles, two of which the next kernel forms again: keeping p and ds
// for it would move 4 bytes a pair, more time than they take (512 flop at heads of 128).
template <int DH, int NW, int NS>
__device__ __forceinline__ void bwd_q_body(const CrossArgs& a, int id, int grid) {
  char* smem = dtl_smem;
  constexpr int SLOT = 2 * kTileBytes<DH>;
  const int parts = a.bq.parts;
  Where w;
  if (!where(a, a.bq, id, grid, w)) return;
  const int n = keys_of(a, w.b), nt = (n + TILE - 1) / TILE;
  const int t0 = (int)((int64_t)nt * w.part / parts), t1 = (int)((int64_t)nt * (w.part + 1) / parts);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, grp = l >> 5;
  const int r = w.block * OWN * NW + wave * OWN + (l & 31);
  const bool active = w.block * OWN * NW + wave * OWN < a.R;
  const int rc = r < a.R ? r : a.R - 1;
  const uint16_t* K = a.k + (int64_t)w.b * a.Sk * a.ldk + w.h * DH;
  const uint16_t* V = a.v + (int64_t)w.b * a.Sk * a.ldv + w.h * DH;
  f32x16 dq[DH / 32];
  clear(dq);
  const TileLoads<DH, NW> loads(wave);
  constexpr int LPT = 2 * TileLoads<DH, NW>::N;
  auto issue = [&](int t) {
    char* to = smem + (t - t0) % NS * SLOT;
    loads.keys(K, a.ldk, t * TILE, n, to);
    loads.keys(V, a.ldv, t * TILE, n, to + kTileBytes<DH>);
  };
#pragma unroll
  for (int i = 0; i < NS - 1; ++i)
    if (t0 + i < t1) issue(t0 + i);
  Frag qf[DH / 16], of[DH / 16];
  load_owned<DH>(qf, a.q + row_at<DH>(a, w.b, w.h, rc, a.ldq));
  load_owned<DH>(of, a.dout + row_at<DH>(a, w.b, w.h, rc, a.lddo));
  float lse = a.stat_lse[(int64_t)w.unit * a.Rp + rc], D = a.stat_d[(int64_t)w.unit * a.Rp + rc];
  settle(qf); settle(of);
  asm volatile("" : "+v"(lse), "+v"(D));
  auto tile = [&](int first, const char* Ks) {
    const char* Vs = Ks + kTileBytes<DH>;
#pragma unroll(DH == 128 ? 1 : 2)
    for (int sub = 0; sub < 2; ++sub) {
      f32x16 s[1], dp[1];
#pragma unroll
      for (int x = 0; x < 16; ++x) { s[0][x] = lse; dp[0][x] = D; }
      in_a_row<DH / 8, DH == 128 ? 4 : 2>([&](int i) { return frag_rows<DH>(i % 2 ? Vs : Ks, sub * 32, i / 2); },
                          [&](int i, const Frag& f) {
                            if (i % 2) dp[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, of[i / 2], dp[0], 0, 0, 0);
                            else s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, qf[i / 2], s[0], 0, 0, 0);
                          });
      const int k0 = first + sub * 32;
#pragma unroll
      for (int x = 0; x < 16; ++x) dp[0][x] *= __builtin_amdgcn_exp2f(s[0][x] * a.c2);
      if (k0 + 32 > n) {
        asm volatile("");
#pragma unroll
        for (int x = 0; x < 16; ++x)
          if (k0 + acc_row(x, grp) >= n) dp[0][x] = 0.f;
      }
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        const Frag ds = pack_frag(dp[0], ks);
#pragma unroll
        for (int dt = 0; dt < DH / 32; ++dt)
          dq[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_cols<DH>(Ks, sub * 32 + ks * 16, dt * 32), ds, dq[dt], 0, 0, 0);
      }
    }
  };
  for (int t = t0; t < t1; ++t) {
    if (t + NS - 2 < t1) wait_loads<LPT * (NS - 2)>();
    else wait_loads<0>();
    __syncthreads();
    if (t + NS - 1 < t1) issue(t + NS - 1);
    if (!active) continue;
    tile(t * TILE, smem + (t - t0) % NS * SLOT);
  }
  if (!active || r >= a.R) return;
  if (n == 1) of_one_key(dq);
  if (parts == 1) store_owned<DH>(dq, a.scale, a.dq + row_at<DH>(a, w.b, w.h, r, a.lddq));
  else store_owned32<DH>(dq, a.q_part + (((int64_t)w.part * a.B * a.Hkv + w.unit) * a.R + r) * DH);
}

// dK, dV: a wave owns 32 keys, the rows (queries and do) stream.
template <int DH, int NW, int NS>
__device__ __forceinline__ void bwd_kv_body(const CrossArgs& a, int id, int grid) {
  char* smem = dtl_smem;
  constexpr int SLOT = 2 * kTileBytes<DH> + 2 * TILE * 4;   // queries, do, lse, D
  const int parts = a.bkv.parts;
  Where w;
  if (!where(a, a.bkv, id, grid, w)) return;
  const int n = keys_of(a, w.b), j0 = w.block * OWN * NW;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, grp = l >> 5;
  const int j = j0 + wave * OWN + (l & 31);
  const int nt = j0 < n ? (a.R + TILE - 1) / TILE : 0;      // keys behind the sequence: zeros
  const int t0 = (int)((int64_t)nt * w.part / parts), t1 = (int)((int64_t)nt * (w.part + 1) / parts);
  const bool active = j0 + wave * OWN < n;
  // Heads of 128: keys, values, their two gradients and the scores are 256 registers by themselves; the values stay in LDS, which has
  // bandwidth left (29 % of cycles)
  constexpr bool kValuesInLds = DH == 128;
  Frag* vl = reinterpret_cast<Frag*>(smem + NS * SLOT + wave * OWN * DH * 2) + l;
  Frag kf[DH / 16], vf[DH / 16];
  f32x16 dk[DH / 32], dv[DH / 32];
  clear(dk); clear(dv);
  const TileLoads<DH, NW> loads(wave);
  const float* stat = (wave & 1 ? a.stat_d : a.stat_lse) + (int64_t)w.unit * a.Rp;   // (even waves bring the lse, odd ones D)
  auto issue = [&](int t) {
    char* to = smem + (t - t0) % NS * SLOT;
    loads.rows([&](int r, int64_t& tok, int& c) {
      const int g = r / a.Sq, at = r - g * a.Sq;
      tok = (int64_t)w.b * a.Sq + at;
      c = (w.h * a.share + g) * DH;
    }, a.R, a.q, a.ldq, a.dout, a.lddo, t * TILE, to, to + kTileBytes<DH>);
    load_floats(stat + t * TILE, to + 2 * kTileBytes<DH> + (wave & 1) * TILE * 4);
  };
  // One slot: the next tile is asked for when everyone has left this one.  The first tile goes out ahead of the wave's own keys: with few
  // rows a workgroup is one chain of round trips.
  static_assert(NS == 1 || NS == 2, "slots");
  if (t0 < t1) issue(t0);
  if (active) {
    const int jc = j < n ? j : n - 1;
    load_owned<DH>(kf, a.k + ((int64_t)w.b * a.Sk + jc) * a.ldk + w.h * DH);
    load_owned<DH>(vf, a.v + ((int64_t)w.b * a.Sk + jc) * a.ldv + w.h * DH);
    settle(kf); settle(vf);
    if (kValuesInLds) {
#pragma unroll
      for (int kk = 0; kk < DH / 16; ++kk) vl[kk * 64] = vf[kk];
    }
  }
  auto tile = [&](const char* Qs) {
    const char* Os = Qs + kTileBytes<DH>;
    const float* lse = reinterpret_cast<const float*>(Os + kTileBytes<DH>);
#pragma unroll(DH == 128 ? 1 : 2)
    for (int sub = 0; sub < 2; ++sub) {
      f32x16 s[1], dp[1];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4 ls = *reinterpret_cast<const f32x4*>(lse + sub * 32 + 8 * q + 4 * grp);
        const f32x4 D = *reinterpret_cast<const f32x4*>(lse + TILE + sub * 32 + 8 * q + 4 * grp);
#pragma unroll
        for (int x = 0; x < 4; ++x) { s[0][4 * q + x] = ls[x]; dp[0][4 * q + x] = D[x]; }
      }
      struct Two { Frag rows, values; };
      in_a_row<DH / 8, DH == 128 ? 4 : 2>([&](int i) {
                            Two t;
                            t.rows = frag_rows<DH>(i % 2 ? Os : Qs, sub * 32, i / 2);
                            if (kValuesInLds && i % 2) t.values = vl[i / 2 * 64];
                            return t;
                          },
                          [&](int i, const Two& t) {
                            if (i % 2) dp[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(t.rows, kValuesInLds ? t.values : vf[i / 2], dp[0], 0, 0, 0);
                            else s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(t.rows, kf[i / 2], s[0], 0, 0, 0);
                          });
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        s[0][x] = __builtin_amdgcn_exp2f(s[0][x] * a.c2);
        dp[0][x] *= s[0][x];
      }
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        const Frag p = pack_frag(s[0], ks), ds = pack_frag(dp[0], ks);
#pragma unroll
        for (int dt = 0; dt < DH / 32; ++dt) {
          dv[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_cols<DH>(Os, sub * 32 + ks * 16, dt * 32), p, dv[dt], 0, 0, 0);
          dk[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_cols<DH>(Qs, sub * 32 + ks * 16, dt * 32), ds, dk[dt], 0, 0, 0);
        }
      }
    }
  };
  for (int t = t0; t < t1; ++t) {
    wait_loads<0>();                                       // (at most one tile is on the way)
    __syncthreads();
    if (NS == 2 && t + 1 < t1) issue(t + 1);
    if (active) tile(smem + (t - t0) % NS * SLOT);
    if (NS == 1 && t + 1 < t1) {
      __syncthreads();
      issue(t + 1);
    }
  }
  if (j >= a.Sk) return;
  if (n == 1) of_one_key(dk);
  if (j >= n) { clear(dk); clear(dv); }                     // (repeats of the last key)
  if (parts == 1) {
    store_owned<DH>(dk, a.scale, a.dk + ((int64_t)w.b * a.Sk + j) * a.lddk + w.h * DH);
    store_owned<DH>(dv, 1.0f, a.dv + ((int64_t)w.b * a.Sk + j) * a.lddv + w.h * DH);
  } else {
    float* to = a.kv_part + (((int64_t)w.part * a.B * a.Hkv + w.unit) * a.Sk + j) * 2 * DH;
    store_owned32<DH>(dk, to);
    store_owned32<DH>(dv, to + DH);
  }
}
template <int DH, int NW, int NS_KV> constexpr int kKvLds = NS_KV * (2 * kTileBytes<DH> + 2 * TILE * 4) + (DH == 128 ? NW * OWN * DH * 2 : 0);
template <int DH, int NW, int NS_KV> constexpr int kBwdLds = kKvLds<DH, NW, NS_KV> > 4 * kTileBytes<DH> ? kKvLds<DH, NW, NS_KV> : 4 * kTileBytes<DH>;
// 4 x 4096 x 4096 tokens, 16 heads of 128: 1709 us, 804 TFLOP/s of the gradients' five products (1126 of the seven that are formed), with zeros for
// operands 1374: the power cap again; 64: 905 us, 759.
// Both in one launch, the longer workgroups (dK and dV: four products to dQ's three) first: where neither fills the chip by itself, and for
// the last workgroups of the one to run beside the first of the other.
template <int DH, int NW, int NS_KV>
__global__ __launch_bounds__(64 * NW, DH == 128 ? 2 : 3) void cross_bwd_kernel(CrossArgs a) {
  if ((int)blockIdx.x < a.kv_grid) bwd_kv_body<DH, NW, NS_KV>(a, blockIdx.x, a.kv_grid);
  else bwd_q_body<DH, NW, 2>(a, blockIdx.x - a.kv_grid, gridDim.x - a.kv_grid);
}
// parts -> dq (KV false), or dk and dv
template <int DH, bool KV>
__global__ __launch_bounds__(256) void cross_bwd_join_kernel(CrossArgs a) {
  constexpr int W = KV ? 2 * DH : DH;
  const int per = KV ? a.Sk : a.R, parts = KV ? a.bkv.parts : a.bq.parts;
  const float* sums = KV ? a.kv_part : a.q_part;
  const int64_t rows = (int64_t)a.B * a.Hkv * per;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / (W / 8);
  const int c = (int)(i % (W / 8)) * 8;
  if (row >= rows) return;
  f32x4 v[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll 4
  for (int s = 0; s < parts; ++s) {
    const f32x4* p = reinterpret_cast<const f32x4*>(sums + (s * rows + row) * W + c);
    v[0] += p[0]; v[1] += p[1];
  }
  const int unit = (int)(row / per), r = (int)(row - (int64_t)unit * per), b = unit / a.Hkv, h = unit % a.Hkv;
  const bool values = KV && c >= DH;
  if (!values) { v[0] *= a.scale; v[1] *= a.scale; }
  uint16_t* to = !KV ? a.dq + row_at<DH>(a, b, h, r, a.lddq) + c
                 : values ? a.dv + ((int64_t)b * a.Sk + r) * a.lddv + h * DH + c - DH : a.dk + ((int64_t)b * a.Sk + r) * a.lddk + h * DH + c;
  *reinterpret_cast<u32x4*>(to) = f32_to_bf16x8(v);
}

// ---- host ----------------------------------------------------------------------------------
struct CrossPlan {
  bool token;                              // up to 32 rows to a key/value head
  int R, Rp, fwd_parts, q_parts, kv_parts;
  int at_once;                             // sequences
  size_t fwd_ml, fwd_bytes;                // forward: [sums][pairs]
  size_t d, part, kv_part, bwd_bytes;      // backward: [lse][D][sums of dq][of dk and dv]
};
bool make_cross_plan(CrossPlan& p, int64_t B, int64_t Sq, int64_t Sk, int64_t H, int64_t Hkv, int64_t dh, bool backward) {
  if (B < 1 || Sq < 1 || Sk < 1 || H < 1 || Hkv < 1 || H % Hkv || (dh != 64 && dh != 128)) return false;
  if (B > (1 << 20) || Sq > (1 << 24) || Sk > (1 << 24) || H > (1 << 16)) return false;
  const int64_t U = B * Hkv, R = H / Hkv * Sq;
  if (R > (1ll << 30) || U * up(R, OWN) > (1ll << 30) || U * up(Sk, OWN) > (1ll << 30)) return false;
  if (U * R * dh / 8 > (1ll << 38) || U * Sk * dh / 8 > (1ll << 38)) return false;
  p.R = (int)R; p.Rp = (int)(up(R, TILE) * TILE);
  p.token = R <= OWN;
  p.fwd_parts = p.token ? parts_for(U, up(Sk, TOKEN_KEYS), kTokenGrid, 8) : parts_for(U * up(R, OWN * 4), up(Sk, TILE), 512, 4);
  p.q_parts = parts_for(U * up(R, OWN * 4), up(Sk, TILE), 512, 4);
  // half as many for dK and dV: dQ's workgroups run beside them, and a part costs 8 bytes a key's element.  us, 512 / 256: 1024 of 16 heads over 4 of
  // 128, 2048 keys 250 / 231; 1500 of 12 heads over 400 60 / 53; 512 of 16 over 4, 577 keys, 8 sequences 91 / 97.  (256 for dQ, too: 162 rows
  // over up to 6893 keys 194 / 233.)
  p.kv_parts = parts_for(U * up(Sk, OWN * 4), up(R, TILE), 256, 4);
  // threads of the largest launch, a sequence; of blocks that are dealt out in groups (deal) up to eight for seven more
  auto dealt = [&](int64_t blocks, int parts) { const int64_t n = blocks * parts; return Hkv * (n + (n < 8 ? n : 8) - 1); };
  auto larger = [](int64_t x, int64_t y) { return x > y ? x : y; };
  int64_t threads;
  if (backward) {
    threads = larger(256 * (dealt(up(Sk, OWN * 4), p.kv_parts) + dealt(up(R, OWN * 4), p.q_parts)),
                     512 * (dealt(up(Sk, OWN * 8), p.kv_parts) + dealt(up(R, OWN * 8), p.q_parts)));
    threads = larger(threads, Hkv * p.Rp * (dh / 8));
    if (p.kv_parts > 1) threads = larger(threads, Hkv * Sk * (dh / 4));
  } else {
    threads = 256 * (p.token ? dealt(1, p.fwd_parts) : dealt(up(R, OWN * 4), p.fwd_parts));
    if (p.fwd_parts > 1) threads = larger(threads, Hkv * R * dh);
  }
  if (threads > kMostThreads) return false;
  p.at_once = (int)(B < kMostThreads / threads ? B : kMostThreads / threads);
  auto round = [](size_t b) { return (b + 255) / 256 * 256; };
  const bool parts = p.fwd_parts > 1;
  p.fwd_ml = parts ? round((size_t)4 * p.fwd_parts * U * R * dh) : 0;
  p.fwd_bytes = parts ? p.fwd_ml + round((size_t)8 * p.fwd_parts * U * R) : 0;
  p.d = round((size_t)4 * U * p.Rp);
  p.part = 2 * p.d;
  p.kv_part = p.part + (p.q_parts > 1 ? round((size_t)4 * p.q_parts * U * R * dh) : 0);
  p.bwd_bytes = p.kv_part + (p.kv_parts > 1 ? round((size_t)8 * p.kv_parts * U * Sk * dh) : 0);
  return true;
}

CrossArgs common_args(const CrossPlan& p, const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, const int32_t* klen, int B, int Sq,
                      int Sk, int H, int Hkv, int dh) {
  CrossArgs a{};
  a.q = (const uint16_t*)q; a.k = (const uint16_t*)k; a.v = (const uint16_t*)v;
  a.ldq = ldq; a.ldk = ldk; a.ldv = ldv; a.klen = klen;
  a.B = B; a.Sq = Sq; a.Sk = Sk; a.share = H / Hkv; a.Hkv = Hkv; a.R = p.R; a.Rp = p.Rp;
  a.scale = 1.0f / sqrtf((float)dh);
  a.c2 = 1.4426950408889634f * a.scale;
  return a;
}

// the sequences from b0 on, as many as go into a launch; the work memory of those before is free when they are done
CrossArgs sequences(CrossArgs a, const CrossPlan& p, int b0) {
  const int64_t q = (int64_t)b0 * a.Sq, k = (int64_t)b0 * a.Sk;
  a.B = a.B - b0 < p.at_once ? a.B - b0 : p.at_once;
  a.q += q * a.ldq; a.k += k * a.ldk; a.v += k * a.ldv;
  if (a.klen) a.klen += b0;
  a.lse2 += (int64_t)b0 * a.Hkv * a.R;
  if (a.out) a.out += q * a.ldo;
  if (a.o) { a.o += q * a.ldo; a.dout += q * a.lddo; a.dq += q * a.lddq; a.dk += k * a.lddk; a.dv += k * a.lddv; }
  return a;
}

template <int DH>
rv_status forward(CrossArgs a, const CrossPlan& p, char* work, hipStream_t st) {
  const int64_t U = (int64_t)a.B * a.Hkv;
  a.part = (float*)work; a.part_ml = (float2*)(work + p.fwd_ml);
  if (p.token) {
    constexpr int waves = kTokenWaves<DH>, ring = waves * kTokenRing<DH>, image = waves * (DH / 2 * 64 * 4 + 32 * 8);
    const int64_t grid = deal(a.fwd, a, a.klen != nullptr, 1, p.fwd_parts);
    RV_TRY((launch<cross_token_kernel<DH>>(a, grid, 64 * waves, ring > image ? ring : image, st)));
  } else {
    const int64_t grid = deal(a.fwd, a, a.klen != nullptr, up(a.R, OWN * 4), p.fwd_parts);
    RV_TRY((launch<cross_fwd_kernel<DH, 4, 2>>(a, grid, 256, 2 * 2 * kTileBytes<DH>, st)));
  }
  if (p.fwd_parts == 1) return RV_OK;
  if (p.fwd_parts > 4) RV_TRY((launch<cross_join_kernel<DH, 8>>(a, up(U * a.R * (DH / 8), 32), 256, 0, st)));
  else RV_TRY((launch<cross_join_kernel<DH, 1>>(a, up(U * a.R * (DH / 8), 256), 256, 0, st)));
  return RV_OK;
}
template <int DH, int NW, int NS_KV>
rv_status backward(CrossArgs a, const CrossPlan& p, char* work, hipStream_t st) {
  const int64_t U = (int64_t)a.B * a.Hkv;
  a.stat_lse = (float*)work; a.stat_d = (float*)(work + p.d); a.q_part = (float*)(work + p.part); a.kv_part = (float*)(work + p.kv_part);
  RV_TRY((launch<cross_stat_kernel<DH>>(a, up(U * a.Rp * (DH / 8), 256), 256, 0, st)));
  const int64_t kv = deal(a.bkv, a, a.klen != nullptr, up(a.Sk, OWN * NW), p.kv_parts), q = deal(a.bq, a, a.klen != nullptr, up(a.R, OWN * NW), p.q_parts);
  a.kv_grid = (int)kv;
  RV_TRY((launch<cross_bwd_kernel<DH, NW, NS_KV>>(a, kv + q, 64 * NW, kBwdLds<DH, NW, NS_KV>, st)));
  if (p.q_parts > 1) RV_TRY((launch<cross_bwd_join_kernel<DH, false>>(a, up(U * a.R * (DH / 8), 256), 256, 0, st)));
  if (p.kv_parts > 1) RV_TRY((launch<cross_bwd_join_kernel<DH, true>>(a, up(U * a.Sk * (DH / 4), 256), 256, 0, st)));
  return RV_OK;
}

}  // namespace

extern "C" rv_status rv_k_cross_attention_work(int B, int Sq, int Sk, int n_heads, int n_kv_heads, int d_head, int backward, size_t* bytes) {
  CrossPlan p;
  if (!bytes || !make_cross_plan(p, B, Sq, Sk, n_heads, n_kv_heads, d_head, backward != 0)) return RV_E_INVAL;
  *bytes = backward ? p.bwd_bytes : p.fwd_bytes;
  return RV_OK;
}

extern "C" rv_status rv_k_cross_attention_fwd(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, const int32_t* klen,
                                              void* out, int64_t ldo, float* lse2, int B, int Sq, int Sk, int n_heads, int n_kv_heads, int d_head,
                                              void* work, size_t work_bytes, void* stream) {
  CrossPlan p;
  if (!make_cross_plan(p, B, Sq, Sk, n_heads, n_kv_heads, d_head, false)) return RV_E_INVAL;
  const int64_t cols = (int64_t)n_heads * d_head, kcols = (int64_t)n_kv_heads * d_head;
  if (bad(q, 16) || bad(k, 16) || bad(v, 16) || bad(out, 16) || bad(lse2, 4) || ((uintptr_t)klen & 3)) return RV_E_INVAL;
  if (bad_pitch(ldq, cols) || bad_pitch(ldk, kcols) || bad_pitch(ldv, kcols) || bad_pitch(ldo, cols)) return RV_E_INVAL;
  if (p.fwd_bytes && (bad(work, 256) || work_bytes < p.fwd_bytes)) return RV_E_INVAL;
  CrossArgs a = common_args(p, q, ldq, k, ldk, v, ldv, klen, B, Sq, Sk, n_heads, n_kv_heads, d_head);
  a.out = (uint16_t*)out; a.ldo = ldo; a.lse2 = lse2;
  for (int b = 0; b < B; b += p.at_once) {
    const CrossArgs some = sequences(a, p, b);
    RV_TRY(d_head == 64 ? forward<64>(some, p, (char*)work, (hipStream_t)stream) : forward<128>(some, p, (char*)work, (hipStream_t)stream));
  }
  return RV_OK;
}

extern "C" rv_status rv_k_cross_attention_bwd(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, const int32_t* klen,
                                              const void* out, int64_t ldo, const void* dout, int64_t lddo, const float* lse2, void* dq, int64_t lddq,
                                              void* dk, int64_t lddk, void* dv, int64_t lddv, int B, int Sq, int Sk, int n_heads, int n_kv_heads,
                                              int d_head, void* work, size_t work_bytes, void* stream) {
  CrossPlan p;
  if (!make_cross_plan(p, B, Sq, Sk, n_heads, n_kv_heads, d_head, true)) return RV_E_INVAL;
  const int64_t cols = (int64_t)n_heads * d_head, kcols = (int64_t)n_kv_heads * d_head;
  if (bad(q, 16) || bad(k, 16) || bad(v, 16) || bad(out, 16) || bad(dout, 16) || bad(lse2, 4) || bad(dq, 16) || bad(dk, 16) || bad(dv, 16) ||
      ((uintptr_t)klen & 3)) return RV_E_INVAL;
  if (bad_pitch(ldq, cols) || bad_pitch(ldk, kcols) || bad_pitch(ldv, kcols) || bad_pitch(ldo, cols) || bad_pitch(lddo, cols) || bad_pitch(lddq, cols) ||
      bad_pitch(lddk, kcols) || bad_pitch(lddv, kcols)) return RV_E_INVAL;
  if (bad(work, 256) || work_bytes < p.bwd_bytes) return RV_E_INVAL;
  CrossArgs a = common_args(p, q, ldq, k, ldk, v, ldv, klen, B, Sq, Sk, n_heads, n_kv_heads, d_head);
  a.o = (const uint16_t*)out; a.ldo = ldo; a.dout = (const uint16_t*)dout; a.lddo = lddo; a.lse2 = (float*)lse2;
  a.dq = (uint16_t*)dq; a.lddq = lddq; a.dk = (uint16_t*)dk; a.lddk = lddk; a.dv = (uint16_t*)dv; a.lddv = lddv;
  const hipStream_t st = (hipStream_t)stream;
  // Heads of 128: two waves to a SIMD either way (registers).  Eight that share two slots are the faster where there are rounds of them,
  // two workgroups of four with a slot each where one is short of work or ends early.  us, eight / four: 4 x 4096 x 4096 tokens, 16 heads (2048
  // workgroups of eight) 1711 / 1830; 162 tokens of 32 heads over 16 and up to 6893 keys (1184) 223 / 195; 1024 of 16 over 4 and up to 2048
  // (384) 219 / 193.  Heads of 64 are faster with four: three waves to a SIMD, 4 x 4096 x 4096 892 / 979.
  const int64_t eights = (int64_t)B * n_kv_heads * (up(Sk, 8 * OWN) * p.kv_parts + up(p.R, 8 * OWN) * p.q_parts);
  const bool by_eight = p.R > 4 * OWN && Sk > 4 * OWN && eights >= 1536;
  for (int b = 0; b < B; b += p.at_once) {
    const CrossArgs some = sequences(a, p, b);
    RV_TRY(d_head == 64 ? (backward<64, 4, 2>(some, p, (char*)work, st))
           : by_eight   ? (backward<128, 8, 2>(some, p, (char*)work, st))
                        : (backward<128, 4, 1>(some, p, (char*)work, st)));
  }
  return RV_OK;
}

// Positions as rotations of queries and keys, with the norm of each head in the same pass, forward and backward.
//
//   n = x rsqrt(mean(x^2) + eps) gamma over a head's columns (or x);   with angle = position * frequency, c and s its cosine and sine times the
//   amplitude:  (a, b) -> (a c - b s, b c + a s) for every pair of the head's first `rot` columns
//   backward: dn by the opposite angle, xh = x rsqrt(..):  dx = rsqrt(..) (dn gamma - xh mean(dn gamma xh)),  dgamma = sum dn xh
//
// Bound by memory: every element is read and written once (backward with a norm: read twice as much), 16 bytes to an access.  A lane holds
// 16 columns of a head, two chunks of eight that contain the pairs of one another, so a head is 4 or 8 neighbouring lanes and its norm a sum
// over them.  Cosines and sines are formed once for each (token, frequency) of a workgroup's tokens and reach the heads through LDS.
// An angle is formed as a fraction of a turn of which a product of 64-bit numbers keeps all its bits, and is rounded to 32 bits once (angles).
#include <math.h>
#include "../../include/rv_kernels.h"
#include "common.h"

namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kMostTokens = 32;                  // of a workgroup at one time
constexpr int kGammaGroups = 1024;               // workgroups that add up the norms' gradients, a partial row each

// What a workgroup works on: queries, keys or values, so that addresses and the norm's weight are those of all its lanes.
struct Side {
  const uint16_t* x; int64_t ldx;                // forward: what is turned; backward: the forward's input, with a norm
  const uint16_t* g; int64_t ldg;                // backward: the gradient of the output
  uint16_t* out; int64_t ldo;
  const uint16_t* gamma;
  float* part;                                   // backward: partial rows [groups][dh] of the norm's gradient
  int heads, tw, groups;                         // tw: tokens of a workgroup at one time; groups: workgroups
  float per_token;                               // 1 / items of a token
};
struct RotArgs {
  Side side[3];
  const double* freq;
  const int* pos; const int* start; const int* length;
  int64_t tokens;
  int S, rot, rows, sinks;
  float amplitude, eps;
};

struct Token { int64_t row; int live; };         // row of k_out and v_out, or -1

// Chunks of eight columns that lane j of a head's L holds: with halves, j and its partner where they are turned, the rest in order behind.
template <int L, bool PAIRS>
__device__ __forceinline__ void chunks(int j, int rh, int& a, int& b) {
  a = PAIRS || j < rh ? j : j + rh;
  b = PAIRS || j >= rh ? j + L : j + rh;
}

template <int L>
__device__ __forceinline__ float head_sum(float v) {             // over a head's lanes, left in each of them
  v = rv_dpp_add<0xB1>(v);
  v = rv_dpp_add<0x4E>(v);
  return L == 8 ? rv_dpp_add<0x141>(v) : v;
}

__device__ __forceinline__ void widen(float (&x)[16], const u32x4& a, const u32x4& b) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(a[i] << 16); x[2 * i + 1] = __uint_as_float(a[i] & 0xFFFF0000u);
    x[8 + 2 * i] = __uint_as_float(b[i] << 16); x[8 + 2 * i + 1] = __uint_as_float(b[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void narrow(const float (&x)[16], u32x4& a, u32x4& b) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    a[i] = rv_pack_bf16x2(x[2 * i], x[2 * i + 1]);
    b[i] = rv_pack_bf16x2(x[8 + 2 * i], x[8 + 2 * i + 1]);
  }
}

// x turned by the angles of a token (cs: cosine and sine of every frequency), BACK: by their opposites
template <int L, bool PAIRS, bool BACK>
__device__ __forceinline__ void turn(float (&x)[16], const float2* cs, int j, int rh) {
  if (PAIRS) {
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int chunk = j + half * L;
      if (chunk >= 2 * rh) continue;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 w = cs[chunk * 4 + i];
        const float s = BACK ? -w.y : w.y, a = x[8 * half + 2 * i], b = x[8 * half + 2 * i + 1];
        x[8 * half + 2 * i] = __fmaf_rn(a, w.x, -(b * s));
        x[8 * half + 2 * i + 1] = __fmaf_rn(b, w.x, a * s);
      }
    }
  } else if (j < rh) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 w = cs[j * 8 + i];
      const float s = BACK ? -w.y : w.y, a = x[i], b = x[8 + i];
      x[i] = __fmaf_rn(a, w.x, -(b * s));
      x[8 + i] = __fmaf_rn(b, w.x, a * s);
    }
  }
}

// p f / (2 pi) less a whole number: f / (2 pi) as the sum of two 64-bit numbers (2^-104 of itself off), whole turns taken out of the exact product with the
// first.  For |p| <= 2^31 + 2^24 and |f| <= 2^40 the fraction is off by 2^-34 turns at most, and by 2^-26 when it is rounded to 32 bits.  (One product
// of 64 bits was off by 2^-53 of all the turns: 2^-24 of one at f = 1 and position 2^31.)
__device__ __forceinline__ float turn_fraction(double p, double f) {
  constexpr double kTurn = 0.15915494309189535, kTurnRest = -9.839338337591243e-18;      // 1 / (2 pi)
  const double h = f * kTurn, rest = fma(f, kTurnRest, fma(f, kTurn, -h));
  const double t = fma(p, rest, fma(p, h, -rint(p * h)));
  return (float)(t - rint(t));
}

// What a workgroup's tokens t0 .. share: where they go and their angles.
__device__ __forceinline__ void angles(const RotArgs& a, int64_t t0, int tw, bool in_cache, bool turned, Token* token, float2* cs) {
  const int half = a.rot / 2;
  for (int i = threadIdx.x; i < tw; i += 256) {
    const int64_t t = t0 + i;
    Token to{-1, 0};
    if (t < a.tokens) {
      const int b = (int)(t / a.S), at = (int)(t - (int64_t)b * a.S);
      const int n = a.length ? a.length[b] : a.S;
      to.live = at < n;
      to.row = t;
      if (in_cache) {
        // the row of the position, unless a later token of this call takes it
        int64_t p = a.start ? a.start[b] : 0;
        if (p < 0) p = 0;
        const int64_t end = p + (n < a.S ? n : a.S), ring = a.rows - a.sinks;
        p += at;
        const bool stays = to.live && (p < a.sinks || p + ring >= end);
        to.row = !stays ? -1 : (int64_t)b * a.rows + (p < a.sinks ? p : a.sinks + (p - a.sinks) % ring);
      }
    }
    token[i] = to;
  }
  for (int i = threadIdx.x; turned && i < tw * half; i += 256) {
    const int w = i / half, f = i - w * half;
    const int64_t t = t0 + w;
    if (t >= a.tokens) break;
    const int b = (int)(t / a.S);
    int64_t p;
    if (a.pos) p = a.pos[t];
    else {
      p = a.start ? a.start[b] : 0;
      p = (p < 0 ? 0 : p) + (t - (int64_t)b * a.S);
    }
    float s, c;
    sincospif(2.0f * turn_fraction((double)p, a.freq[f]), &s, &c);
    cs[w * half + f] = float2{c * a.amplitude, s * a.amplitude};
  }
  __syncthreads();
}

// an item of a workgroup: (token, head, lane of the head)
struct Item { int w, head; };
template <int L>
__device__ __forceinline__ Item item_at(const Side& d, int it) {
  Item x;
  x.w = (int)(((float)it + 0.5f) * d.per_token);               // exact: it < 2^20
  x.head = it / L - x.w * d.heads;
  return x;
}

// the norm's factor of a head
template <int L>
__device__ __forceinline__ float inverse_rms(const float (&x)[16], float eps) {
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) ss = __fmaf_rn(x[i], x[i], ss);
  return 1.0f / sqrtf(head_sum<L>(ss) * (1.0f / (16 * L)) + eps);
}

// Workgroup -> side and its number there
__device__ __forceinline__ int side_of(const RotArgs& a, int& id) {
  int s = 0;
  while (id >= a.side[s].groups) id -= a.side[s++].groups;
  return s;
}

// The next item's loads are out while one is turned.  Five workgroups to a CU (82 registers): 65536 tokens of 32 + 8 heads of 128 with norms 256 us, 5.2 TB/s (a
// large copy 4.9 to 5.4); with two items' loads out, and four workgroups, 277.
template <int L, bool PAIRS>
__global__ __launch_bounds__(256, 5) void rotary_fwd_kernel(RotArgs a) {
  constexpr int DH = 16 * L;
  __shared__ Token token[kMostTokens];
  __shared__ __align__(16) float2 cs[kMostTokens * DH / 2];
  int id = blockIdx.x;
  const int which = side_of(a, id);                             // queries, keys, values
  const Side d = a.side[which];
  const int j = threadIdx.x % L, rh = a.rot / 16, half = a.rot / 2;
  int ca, cb;
  chunks<L, PAIRS>(j, rh, ca, cb);
  for (int64_t t0 = (int64_t)id * d.tw; t0 < a.tokens; t0 += (int64_t)d.groups * d.tw) {
    const int n = (int)((a.tokens - t0 < d.tw ? a.tokens - t0 : d.tw) * d.heads * L);
    const uint16_t* from = d.x + t0 * d.ldx;
    u32x4 in[2];
    auto load = [&](int it) {
      if (it >= n) return;
      const Item x = item_at<L>(d, it);
      const uint16_t* at = from + x.w * d.ldx + x.head * DH;
      in[0] = *reinterpret_cast<const u32x4*>(at + ca * 8);
      in[1] = *reinterpret_cast<const u32x4*>(at + cb * 8);
    };
    // the first loads are out while the angles are formed
    load(threadIdx.x);
    angles(a, t0, d.tw, a.rows && which, which < 2, token, cs);
    for (int it = threadIdx.x; it < n; it += 256) {
      const Item x = item_at<L>(d, it);
      const Token to = token[x.w];
      u32x4 o[2] = {in[0], in[1]};
      load(it + 256);
      if (which < 2) {
        float v[16];
        widen(v, o[0], o[1]);
        if (d.gamma) {
          const float r = inverse_rms<L>(v, a.eps);
          float g[16];
          widen(g, *reinterpret_cast<const u32x4*>(d.gamma + ca * 8), *reinterpret_cast<const u32x4*>(d.gamma + cb * 8));
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] = v[i] * r * g[i];
        }
        turn<L, PAIRS, false>(v, cs + x.w * half, j, rh);
        narrow(v, o[0], o[1]);
      }
      if (!to.live) o[0] = o[1] = u32x4{0u, 0u, 0u, 0u};
      if (to.row < 0) continue;
      uint16_t* out = d.out + to.row * d.ldo + x.head * DH;
      *reinterpret_cast<u32x4*>(out + ca * 8) = o[0];
      *reinterpret_cast<u32x4*>(out + cb * 8) = o[1];
    }
    __syncthreads();
  }
}

// With a norm the forward's inputs are read beside the gradients, and the norm's gradient is added up: a lane's own columns over all its items, then
// over the lanes of a workgroup that hold the same columns, one partial row each.
template <int L, bool PAIRS, bool NORM>
__device__ __forceinline__ void bwd_body(const RotArgs& a, const Side& d, int id, Token* token, float2* cs) {
  constexpr int DH = 16 * L;
  const int j = threadIdx.x % L, rh = a.rot / 16, half = a.rot / 2;
  int ca, cb;
  chunks<L, PAIRS>(j, rh, ca, cb);
  float sum[NORM ? 16 : 1];
#pragma unroll
  for (int i = 0; i < (NORM ? 16 : 1); ++i) sum[i] = 0.f;
  u32x4 w[2];
  if constexpr (NORM) {
    w[0] = *reinterpret_cast<const u32x4*>(d.gamma + ca * 8);
    w[1] = *reinterpret_cast<const u32x4*>(d.gamma + cb * 8);
  }
  for (int64_t t0 = (int64_t)id * d.tw; t0 < a.tokens; t0 += (int64_t)d.groups * d.tw) {
    const int n = (int)((a.tokens - t0 < d.tw ? a.tokens - t0 : d.tw) * d.heads * L);
    const uint16_t* from = d.g + t0 * d.ldg;
    const uint16_t* was = d.x + t0 * d.ldx;
    uint16_t* out = d.out + t0 * d.ldo;
    u32x4 in[NORM ? 4 : 2];
    auto load = [&](int it) {
      if (it >= n) return;
      const Item x = item_at<L>(d, it);
      const uint16_t* at = from + x.w * d.ldg + x.head * DH;
      in[0] = *reinterpret_cast<const u32x4*>(at + ca * 8);
      in[1] = *reinterpret_cast<const u32x4*>(at + cb * 8);
      if constexpr (NORM) {
        const uint16_t* in_at = was + x.w * d.ldx + x.head * DH;
        in[2] = *reinterpret_cast<const u32x4*>(in_at + ca * 8);
        in[3] = *reinterpret_cast<const u32x4*>(in_at + cb * 8);
      }
    };
    load(threadIdx.x);
    angles(a, t0, d.tw, false, true, token, cs);
    for (int it = threadIdx.x; it < n; it += 256) {
      const Item x = item_at<L>(d, it);
      const bool live = token[x.w].live;
      float g[16], v[NORM ? 16 : 1];
      widen(g, in[0], in[1]);
      if constexpr (NORM) widen(v, in[2], in[3]);
      load(it + 256);
      turn<L, PAIRS, true>(g, cs + x.w * half, j, rh);
      if constexpr (NORM) {
        const float r = inverse_rms<L>(v, a.eps);
        float gamma[16], dot = 0.f;
        widen(gamma, w[0], w[1]);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          v[i] *= r;                                             // xh
          if (live) sum[i] = __fmaf_rn(g[i], v[i], sum[i]);
          g[i] *= gamma[i];
          dot = __fmaf_rn(g[i], v[i], dot);
        }
        dot = head_sum<L>(dot) * (1.0f / DH);
#pragma unroll
        for (int i = 0; i < 16; ++i) g[i] = r * __fmaf_rn(-v[i], dot, g[i]);
      }
      u32x4 o[2];
      narrow(g, o[0], o[1]);
      if (!live) o[0] = o[1] = u32x4{0u, 0u, 0u, 0u};
      uint16_t* to = out + x.w * d.ldo + x.head * DH;
      *reinterpret_cast<u32x4*>(to + ca * 8) = o[0];
      *reinterpret_cast<u32x4*>(to + cb * 8) = o[1];
    }
    __syncthreads();
  }
  if constexpr (NORM) {
    if (!d.part) return;
    float* lds = reinterpret_cast<float*>(cs);                   // [4 waves][DH]
#pragma unroll
    for (int i = 0; i < 16; ++i) {
#pragma unroll
      for (int o = L; o < 64; o *= 2) sum[i] += __shfl_xor(sum[i], o, 64);
      if ((threadIdx.x & 63) < L) lds[(threadIdx.x >> 6) * DH + (i < 8 ? ca : cb) * 8 + (i & 7)] = sum[i];
    }
    __syncthreads();
    const int c = threadIdx.x;
    if (c < DH) d.part[(int64_t)id * DH + c] = (lds[c] + lds[DH + c]) + (lds[2 * DH + c] + lds[3 * DH + c]);
  }
}
// Four workgroups to a CU (128 registers): 16384 tokens of 32 + 8 heads of 128 with norms 110 us, 4.6 TB/s; with sums for queries and keys in every
// workgroup, two to a CU, 148.
template <int L, bool PAIRS>
__global__ __launch_bounds__(256, 4) void rotary_bwd_kernel(RotArgs a) {
  __shared__ Token token[kMostTokens];
  __shared__ __align__(16) float2 cs[kMostTokens * 8 * L];
  int id = blockIdx.x;
  const Side d = a.side[side_of(a, id)];
  if (d.gamma) bwd_body<L, PAIRS, true>(a, d, id, token, cs);
  else bwd_body<L, PAIRS, false>(a, d, id, token, cs);
}

// partial rows [groups][DH] -> dgamma; a workgroup adds eight columns of the queries' norm or of the keys', 32 lanes to each
__global__ __launch_bounds__(256) void rotary_gamma_kernel(const float* part_q, int groups_q, float* dq, const float* part_k, int groups_k, float* dk, int dh) {
  __shared__ float sums[32][8];
  const bool keys = (int)blockIdx.x >= dh / 8;
  const float* part = keys ? part_k : part_q;
  float* to = keys ? dk : dq;
  if (!to) return;
  const int groups = keys ? groups_k : groups_q, c = (keys ? blockIdx.x - dh / 8 : blockIdx.x) * 8 + threadIdx.x % 8, lane = threadIdx.x / 8;
  float s = 0.f;
#pragma unroll 8
  for (int r = lane; r < groups; r += 32) s += part[(int64_t)r * dh + c];
  sums[lane][threadIdx.x % 8] = s;
  __syncthreads();
  if (threadIdx.x >= 8) return;
  s = 0.f;
#pragma unroll
  for (int r = 0; r < 32; ++r) s += sums[r][threadIdx.x];
  to[c] = s;
}

// ---- host ----------------------------------------------------------------------------------
bool bad(const void* p, uintptr_t to) { return !p || ((uintptr_t)p & (to - 1)); }
bool bad_pitch(int64_t ld, int64_t cols) { return ld < cols || ld % 8 || ld > (1 << 24); }
bool bad_matrix(const void* p, int64_t ld, int64_t cols) { return bad(p, 16) || bad_pitch(ld, cols); }

bool sizes_ok(int64_t B, int64_t S, int64_t H, int64_t Hkv, int64_t dh) {
  if (B < 1 || S < 1 || H < 0 || Hkv < 0 || H + Hkv < 1 || (dh != 64 && dh != 128)) return false;
  return B <= (1 << 20) && S <= (1 << 24) && B * S <= (1 << 30) && H <= (1 << 12) && Hkv <= (1 << 12);
}

// Workgroups and tokens of a side: up to 1024 items of 16 columns to a workgroup at one time, fewer where that leaves less than 512 workgroups (8 x 511 tokens of
// 25 + 25 heads of 64, a token of which is 100 items of either side: 14 us with one token to a workgroup, 9.6 with the seven of this rule).
void deal(Side& d, int64_t tokens, int dh, int64_t most) {
  const int items = d.heads * (dh / 16);
  if (!items) return;
  const int64_t w = 1024 / items < tokens / 512 ? 1024 / items : tokens / 512;
  d.tw = (int)(w < 1 ? 1 : w > kMostTokens ? kMostTokens : w);
  const int64_t groups = (tokens + d.tw - 1) / d.tw;
  d.groups = (int)(groups < most ? groups : most);
  d.per_token = 1.0f / (float)items;
}
constexpr int64_t kMostGroups = 1 << 20;

// of the backward with dgamma: the sides' workgroups in proportion to their heads
void deal_gamma(RotArgs& a, int dh) {
  const int64_t all = a.side[0].heads + a.side[1].heads;
  for (int i = 0; i < 2; ++i) {
    const int64_t most = kGammaGroups * a.side[i].heads / all;
    deal(a.side[i], a.tokens, dh, most < 1 ? 1 : most);
  }
}

rv_status common(const rv_rotary_desc* d, RotArgs& a) {
  if (!d || !sizes_ok(d->B, d->S, d->n_heads, d->n_kv_heads, d->d_head)) return RV_E_INVAL;
  if (d->rot < 0 || d->rot > d->d_head || d->rot % 16 || (d->layout != RV_ROT_HALF && d->layout != RV_ROT_PAIRS)) return RV_E_INVAL;
  if (d->rot && bad(d->freq, 8)) return RV_E_INVAL;
  if (!(fabsf(d->amplitude) <= 3e38f) || !(d->eps >= 0.f) || !(d->eps <= 3e38f)) return RV_E_INVAL;
  if (((uintptr_t)d->pos | (uintptr_t)d->start | (uintptr_t)d->length) & 3) return RV_E_INVAL;
  if (((uintptr_t)d->gamma_q | (uintptr_t)d->gamma_k) & 15) return RV_E_INVAL;
  a = RotArgs{};
  a.freq = d->freq; a.pos = d->pos; a.start = d->start; a.length = d->length;
  a.tokens = (int64_t)d->B * d->S;
  a.S = d->S; a.rot = d->rot;
  a.amplitude = d->amplitude; a.eps = d->eps;
  a.side[0].heads = d->n_heads; a.side[1].heads = d->n_kv_heads;
  a.side[0].gamma = d->n_heads ? (const uint16_t*)d->gamma_q : nullptr;
  a.side[1].gamma = d->n_kv_heads ? (const uint16_t*)d->gamma_k : nullptr;
  return RV_OK;
}

template <int L, bool PAIRS>
rv_status forward(const RotArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((rotary_fwd_kernel<L, PAIRS>), dim3(a.side[0].groups + a.side[1].groups + a.side[2].groups), dim3(256), 0, st, a);
  return rv_launch_status();
}
template <int L, bool PAIRS>
rv_status backward(const RotArgs& a, float* dgamma_q, float* dgamma_k, hipStream_t st) {
  const Side& q = a.side[0];
  const Side& k = a.side[1];
  hipLaunchKernelGGL((rotary_bwd_kernel<L, PAIRS>), dim3(q.groups + k.groups), dim3(256), 0, st, a);
  RV_TRY(rv_launch_status());
  if (!dgamma_q && !dgamma_k) return RV_OK;
  hipLaunchKernelGGL(rotary_gamma_kernel, dim3(2 * 16 * L / 8), dim3(256), 0, st, q.part, q.groups, dgamma_q, k.part, k.groups, dgamma_k, 16 * L);
  return rv_launch_status();
}

}  // namespace

extern "C" rv_status rv_k_rotary_frequencies(int rot, double base, int rule, double factor, double context, double low, double high, double* freq,
                                             float* amplitude) {
  if (rot < 2 || rot % 2 || rot > 1024 || !freq || !amplitude || !(base > 1.0) || !(base < 1e300)) return RV_E_INVAL;
  if (rule < RV_FREQ_PLAIN || rule > RV_FREQ_PARTS) return RV_E_INVAL;
  if (rule != RV_FREQ_PLAIN && (!(factor >= 1.0) || !(factor < 1e300))) return RV_E_INVAL;
  if (rule == RV_FREQ_BASE && rot < 4) return RV_E_INVAL;
  if (rule == RV_FREQ_PARTS && (!(context > 0.0) || !(context < 1e300) || !(low >= 0.0) || !(high > low) || !(high < 1e300))) return RV_E_INVAL;
  if (rule == RV_FREQ_BASE) base *= pow(factor, rot / (rot - 2.0));
  for (int i = 0; i < rot / 2; ++i) {
    double f = pow(base, -2.0 * i / rot);
    if (rule == RV_FREQ_LINEAR) f /= factor;
    if (rule == RV_FREQ_PARTS) {
      double keep = (context * f / 6.283185307179586 - low) / (high - low);
      keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
      f *= keep + (1.0 - keep) / factor;
    }
    freq[i] = f;
  }
  *amplitude = rule == RV_FREQ_PARTS ? (float)(0.1 * log(factor) + 1.0) : 1.0f;
  return RV_OK;
}

extern "C" rv_status rv_k_rotary_work(int B, int S, int n_heads, int n_kv_heads, int d_head, size_t* bytes) {
  if (!bytes || !sizes_ok(B, S, n_heads, n_kv_heads, d_head)) return RV_E_INVAL;
  RotArgs a{};
  a.tokens = (int64_t)B * S; a.side[0].heads = n_heads; a.side[1].heads = n_kv_heads;
  deal_gamma(a, d_head);
  *bytes = (size_t)(a.side[0].groups + a.side[1].groups) * d_head * 4;
  return RV_OK;
}

extern "C" rv_status rv_k_rotary_fwd(const rv_rotary_desc* d) {
  RotArgs a;
  RV_TRY(common(d, a));
  const int64_t cols = (int64_t)d->n_heads * d->d_head, kcols = (int64_t)d->n_kv_heads * d->d_head;
  if (cols && (bad_matrix(d->q, d->ldq, cols) || bad_matrix(d->q_out, d->ldq_out, cols))) return RV_E_INVAL;
  if (kcols && (bad_matrix(d->k, d->ldk, kcols) || bad_matrix(d->k_out, d->ldk_out, kcols))) return RV_E_INVAL;
  if (d->v && (!kcols || bad_matrix(d->v, d->ldv, kcols) || bad_matrix(d->v_out, d->ldv_out, kcols))) return RV_E_INVAL;
  if (d->rows < 0 || d->rows > (1 << 24) || d->sinks < 0 || (d->rows && !kcols)) return RV_E_INVAL;
  a.rows = d->rows;
  a.sinks = d->sinks < d->rows ? d->sinks : d->rows - 1;
  Side& q = a.side[0];
  Side& k = a.side[1];
  Side& v = a.side[2];
  q.x = (const uint16_t*)d->q; q.ldx = d->ldq; q.out = (uint16_t*)d->q_out; q.ldo = d->ldq_out;
  k.x = (const uint16_t*)d->k; k.ldx = d->ldk; k.out = (uint16_t*)d->k_out; k.ldo = d->ldk_out;
  v.x = (const uint16_t*)d->v; v.ldx = d->ldv; v.out = (uint16_t*)d->v_out; v.ldo = d->ldv_out;
  v.heads = d->v ? d->n_kv_heads : 0;
  for (Side& s : a.side) deal(s, a.tokens, d->d_head, kMostGroups);
  const hipStream_t st = (hipStream_t)d->stream;
  if (d->d_head == 64) return d->layout == RV_ROT_PAIRS ? forward<4, true>(a, st) : forward<4, false>(a, st);
  return d->layout == RV_ROT_PAIRS ? forward<8, true>(a, st) : forward<8, false>(a, st);
}

extern "C" rv_status rv_k_rotary_bwd(const rv_rotary_desc* d) {
  RotArgs a;
  RV_TRY(common(d, a));
  Side& q = a.side[0];
  Side& k = a.side[1];
  const int64_t cols = (int64_t)d->n_heads * d->d_head, kcols = (int64_t)d->n_kv_heads * d->d_head;
  if (cols && (bad_matrix(d->dq_out, d->lddq_out, cols) || bad_matrix(d->dq, d->lddq, cols))) return RV_E_INVAL;
  if (kcols && (bad_matrix(d->dk_out, d->lddk_out, kcols) || bad_matrix(d->dk, d->lddk, kcols))) return RV_E_INVAL;
  if (q.gamma && (bad_matrix(d->q, d->ldq, cols) || ((uintptr_t)d->dgamma_q & 3))) return RV_E_INVAL;
  if (k.gamma && (bad_matrix(d->k, d->ldk, kcols) || ((uintptr_t)d->dgamma_k & 3))) return RV_E_INVAL;
  if ((d->dgamma_q && !q.gamma) || (d->dgamma_k && !k.gamma)) return RV_E_INVAL;
  q.x = (const uint16_t*)d->q; q.ldx = d->ldq; q.g = (const uint16_t*)d->dq_out; q.ldg = d->lddq_out; q.out = (uint16_t*)d->dq; q.ldo = d->lddq;
  k.x = (const uint16_t*)d->k; k.ldx = d->ldk; k.g = (const uint16_t*)d->dk_out; k.ldg = d->lddk_out; k.out = (uint16_t*)d->dk; k.ldo = d->lddk;
  if (d->dgamma_q || d->dgamma_k) {
    size_t need = 0;
    RV_TRY(rv_k_rotary_work(d->B, d->S, d->n_heads, d->n_kv_heads, d->d_head, &need));
    if (bad(d->work, 256) || d->work_bytes < need) return RV_E_INVAL;
    deal_gamma(a, d->d_head);
    q.part = d->dgamma_q ? (float*)d->work : nullptr;
    k.part = d->dgamma_k ? (float*)d->work + (int64_t)q.groups * d->d_head : nullptr;
  } else {
    deal(q, a.tokens, d->d_head, kMostGroups);
    deal(k, a.tokens, d->d_head, kMostGroups);
  }
  const hipStream_t st = (hipStream_t)d->stream;
  if (d->d_head == 64)
    return d->layout == RV_ROT_PAIRS ? backward<4, true>(a, d->dgamma_q, d->dgamma_k, st) : backward<4, false>(a, d->dgamma_q, d->dgamma_k, st);
  return d->layout == RV_ROT_PAIRS ? backward<8, true>(a, d->dgamma_q, d->dgamma_k, st) : backward<8, false>(a, d->dgamma_q, d->dgamma_k, st);
}

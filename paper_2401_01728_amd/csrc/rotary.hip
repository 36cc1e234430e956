// Positions as rotations of queries and keys, with the norm of each head in the same pass, forward and backward.
//
//   n = x rsqrt(mean(x^2) + eps) gamma over a head's columns (or x);   with angle = position * frequency, c and s its cosine and sine times the
//   amplitude:  (a, b) -> (a c - b s, b c + a s) for every pair of the head's first `rot` columns
//   backward: dn by the opposite angle, xh = x rsqrt(..):  dx = rsqrt(..) (dn gamma - xh mean(dn gamma xh)),  dgamma = sum dn xh
//
// Bound by memory: every element is read and written once (backward with a norm: read twice as much), 16 bytes to an access.  A lane holds
// 16 columns of a head, two chunks of eight that contain the pairs of one another, so a head is 4 or 8 neighbouring lanes and its norm a sum
// over them.  Cosines and sines are formed once for each (token, frequency) of a workgroup's tokens and reach the heads through LDS.
// An angle is formed in 64 bits, as turns, and leaves them as a fraction of a turn: at position 2^31 it is off by 2^-24 turns.
#include <math.h>
#include "../../include/rv_kernels.h"
#include "common.h"

namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kMostTokens = 32;                  // of a workgroup at one time
constexpr int kGammaGroups = 1024;               // workgroups that add up the norms' gradients, a partial row each

struct RotArgs {
  const uint16_t* q; const uint16_t* k; const uint16_t* v;       // forward: what is turned; backward: the forward's inputs, with a norm
  int64_t ldq, ldk, ldv;
  const uint16_t* gq; const uint16_t* gk;        // backward: gradients of the outputs
  int64_t ldgq, ldgk;
  uint16_t* q_out; uint16_t* k_out; uint16_t* v_out;
  int64_t ldq_out, ldk_out, ldv_out;
  const uint16_t* gamma_q; const uint16_t* gamma_k;
  const double* freq;
  const int* pos; const int* start; const int* length;
  float* part;                                   // backward: [groups][2][dh]
  int64_t tokens;
  int S, H, Hkv, heads;                          // heads: all that an item may be of
  int rot, tw, rows, sinks;
  float amplitude, eps, per_token;               // per_token: 1 / items of a token
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

// What a workgroup's tokens t0 .. share: where they go and their angles.
__device__ __forceinline__ void angles(const RotArgs& a, int64_t t0, Token* token, float2* cs) {
  const int half = a.rot / 2;
  for (int i = threadIdx.x; i < a.tw; i += 256) {
    const int64_t t = t0 + i;
    Token to{-1, 0};
    if (t < a.tokens) {
      const int b = (int)(t / a.S), at = (int)(t - (int64_t)b * a.S);
      const int n = a.length ? a.length[b] : a.S;
      to.live = at < n;
      to.row = t;
      if (a.rows) {
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
  for (int i = threadIdx.x; i < a.tw * half; i += 256) {
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
    const double turns = (double)p * (a.freq[f] * 0.15915494309189535);       // 1 / (2 pi)
    float s, c;
    sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
    cs[w * half + f] = float2{c * a.amplitude, s * a.amplitude};
  }
  __syncthreads();
}

// an item of a workgroup: (token, head, lane of the head)
struct Item { int w, head; };
template <int L>
__device__ __forceinline__ Item item_at(const RotArgs& a, int it) {
  Item x;
  x.w = (int)(((float)it + 0.5f) * a.per_token);               // exact: it < 2^20
  x.head = it / L - x.w * a.heads;
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

constexpr int kAhead = 2;                        // items of a thread whose loads are out at one time

template <int L, bool PAIRS>
__global__ __launch_bounds__(256) void rotary_fwd_kernel(RotArgs a) {
  constexpr int DH = 16 * L;
  __shared__ Token token[kMostTokens];
  __shared__ __align__(16) float2 cs[kMostTokens * DH / 2];
  const int j = threadIdx.x % L, rh = a.rot / 16, half = a.rot / 2;
  int ca, cb;
  chunks<L, PAIRS>(j, rh, ca, cb);
  for (int64_t t0 = (int64_t)blockIdx.x * a.tw; t0 < a.tokens; t0 += (int64_t)gridDim.x * a.tw) {
    const int n = (int)((a.tokens - t0 < a.tw ? a.tokens - t0 : a.tw) * a.heads * L);
    u32x4 in[kAhead][2];
    auto load = [&](int it, u32x4 (&to)[2]) {
      if (it >= n) return;
      const Item x = item_at<L>(a, it);
      const int64_t t = t0 + x.w;
      const uint16_t* from = x.head < a.H           ? a.q + t * a.ldq + x.head * DH
                             : x.head < a.H + a.Hkv ? a.k + t * a.ldk + (x.head - a.H) * DH
                                                    : a.v + t * a.ldv + (x.head - a.H - a.Hkv) * DH;
      to[0] = *reinterpret_cast<const u32x4*>(from + ca * 8);
      to[1] = *reinterpret_cast<const u32x4*>(from + cb * 8);
    };
    // the first loads are out while the angles are formed
#pragma unroll
    for (int u = 0; u < kAhead; ++u) load(threadIdx.x + u * 256, in[u]);
    angles(a, t0, token, cs);
    for (int base = threadIdx.x; base < n; base += kAhead * 256) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int it = base + u * 256;
        if (it >= n) break;
        const Item x = item_at<L>(a, it);
        const Token to = token[x.w];
        const bool is_q = x.head < a.H, is_k = !is_q && x.head < a.H + a.Hkv;
        float v[16];
        widen(v, in[u][0], in[u][1]);
        load(it + kAhead * 256, in[u]);
        const uint16_t* gamma = is_q ? a.gamma_q : a.gamma_k;
        if ((is_q || is_k) && gamma) {
          const float r = inverse_rms<L>(v, a.eps);
          float g[16];
          widen(g, *reinterpret_cast<const u32x4*>(gamma + ca * 8), *reinterpret_cast<const u32x4*>(gamma + cb * 8));
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] = v[i] * r * g[i];
        }
        if (is_q || is_k) turn<L, PAIRS, false>(v, cs + x.w * half, j, rh);
        u32x4 o[2];
        narrow(v, o[0], o[1]);
        if (!to.live) o[0] = o[1] = u32x4{0u, 0u, 0u, 0u};
        const int64_t row = is_q ? t0 + x.w : to.row;
        if (row < 0) continue;
        uint16_t* out = is_q   ? a.q_out + row * a.ldq_out + x.head * DH
                        : is_k ? a.k_out + row * a.ldk_out + (x.head - a.H) * DH
                               : a.v_out + row * a.ldv_out + (x.head - a.H - a.Hkv) * DH;
        *reinterpret_cast<u32x4*>(out + ca * 8) = o[0];
        *reinterpret_cast<u32x4*>(out + cb * 8) = o[1];
      }
    }
    __syncthreads();
  }
}

// NORM: the forward's inputs are read beside the gradients, and the norms' gradients are added up: a lane's own columns over all its items, then
// over the lanes of a workgroup that hold the same columns, one partial row each.
template <int L, bool PAIRS, bool NORM>
__global__ __launch_bounds__(256) void rotary_bwd_kernel(RotArgs a) {
  constexpr int DH = 16 * L;
  __shared__ Token token[kMostTokens];
  __shared__ __align__(16) float2 cs[kMostTokens * DH / 2];
  const int j = threadIdx.x % L, rh = a.rot / 16, half = a.rot / 2;
  int ca, cb;
  chunks<L, PAIRS>(j, rh, ca, cb);
  float sum_q[NORM ? 16 : 1], sum_k[NORM ? 16 : 1];
#pragma unroll
  for (int i = 0; i < (NORM ? 16 : 1); ++i) sum_q[i] = sum_k[i] = 0.f;
  for (int64_t t0 = (int64_t)blockIdx.x * a.tw; t0 < a.tokens; t0 += (int64_t)gridDim.x * a.tw) {
    const int n = (int)((a.tokens - t0 < a.tw ? a.tokens - t0 : a.tw) * a.heads * L);
    u32x4 in[kAhead][NORM ? 4 : 2];
    auto load = [&](int it, u32x4 (&to)[NORM ? 4 : 2]) {
      if (it >= n) return;
      const Item x = item_at<L>(a, it);
      const int64_t t = t0 + x.w;
      const bool is_q = x.head < a.H;
      const int col = (is_q ? x.head : x.head - a.H) * DH;
      const uint16_t* from = is_q ? a.gq + t * a.ldgq + col : a.gk + t * a.ldgk + col;
      to[0] = *reinterpret_cast<const u32x4*>(from + ca * 8);
      to[1] = *reinterpret_cast<const u32x4*>(from + cb * 8);
      if (NORM && (is_q ? a.gamma_q : a.gamma_k)) {
        const uint16_t* was = is_q ? a.q + t * a.ldq + col : a.k + t * a.ldk + col;
        to[NORM ? 2 : 0] = *reinterpret_cast<const u32x4*>(was + ca * 8);
        to[NORM ? 3 : 1] = *reinterpret_cast<const u32x4*>(was + cb * 8);
      }
    };
#pragma unroll
    for (int u = 0; u < kAhead; ++u) load(threadIdx.x + u * 256, in[u]);
    angles(a, t0, token, cs);
    for (int base = threadIdx.x; base < n; base += kAhead * 256) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int it = base + u * 256;
        if (it >= n) break;
        const Item x = item_at<L>(a, it);
        const bool live = token[x.w].live, is_q = x.head < a.H;
        float g[16], v[NORM ? 16 : 1];
        widen(g, in[u][0], in[u][1]);
        if constexpr (NORM) widen(v, in[u][2], in[u][3]);
        load(it + kAhead * 256, in[u]);
        turn<L, PAIRS, true>(g, cs + x.w * half, j, rh);
        if constexpr (NORM) {
          const uint16_t* gamma = is_q ? a.gamma_q : a.gamma_k;
          if (gamma) {
            const float r = inverse_rms<L>(v, a.eps);
            float w[16], dot = 0.f;
            widen(w, *reinterpret_cast<const u32x4*>(gamma + ca * 8), *reinterpret_cast<const u32x4*>(gamma + cb * 8));
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              v[i] *= r;                                         // xh
              const float d = live ? g[i] * v[i] : 0.f;
              if (is_q) sum_q[i] += d;
              else sum_k[i] += d;
              g[i] *= w[i];
              dot = __fmaf_rn(g[i], v[i], dot);
            }
            dot = head_sum<L>(dot) * (1.0f / DH);
#pragma unroll
            for (int i = 0; i < 16; ++i) g[i] = r * __fmaf_rn(-v[i], dot, g[i]);
          }
        }
        u32x4 o[2];
        narrow(g, o[0], o[1]);
        if (!live) o[0] = o[1] = u32x4{0u, 0u, 0u, 0u};
        const int64_t t = t0 + x.w;
        uint16_t* out = is_q ? a.q_out + t * a.ldq_out + x.head * DH : a.k_out + t * a.ldk_out + (x.head - a.H) * DH;
        *reinterpret_cast<u32x4*>(out + ca * 8) = o[0];
        *reinterpret_cast<u32x4*>(out + cb * 8) = o[1];
      }
    }
    __syncthreads();
  }
  if constexpr (NORM) {
    if (!a.part) return;
    float* lds = reinterpret_cast<float*>(cs);                   // [4 waves][2][DH]: at most 4 KB
#pragma unroll
    for (int i = 0; i < 16; ++i) {
#pragma unroll
      for (int o = L; o < 64; o *= 2) { sum_q[i] += __shfl_xor(sum_q[i], o, 64); sum_k[i] += __shfl_xor(sum_k[i], o, 64); }
      if ((threadIdx.x & 63) < L) {
        const int col = (i < 8 ? ca : cb) * 8 + (i & 7);
        lds[((threadIdx.x >> 6) * 2 + 0) * DH + col] = sum_q[i];
        lds[((threadIdx.x >> 6) * 2 + 1) * DH + col] = sum_k[i];
      }
    }
    __syncthreads();
    if (threadIdx.x < 2 * DH) {
      const int i = threadIdx.x;
      a.part[(int64_t)blockIdx.x * 2 * DH + i] = (lds[i] + lds[2 * DH + i]) + (lds[4 * DH + i] + lds[6 * DH + i]);
    }
  }
}

// partial rows [groups][2][DH] -> dgamma_q, dgamma_k; a workgroup adds eight columns, 32 lanes to each
__global__ __launch_bounds__(256) void rotary_gamma_kernel(const float* part, int groups, int dh, float* dq, float* dk) {
  __shared__ float sums[32][8];
  const int c = blockIdx.x * 8 + threadIdx.x % 8, lane = threadIdx.x / 8;
  float s = 0.f;
#pragma unroll 8
  for (int r = lane; r < groups; r += 32) s += part[(int64_t)r * 2 * dh + c];
  sums[lane][threadIdx.x % 8] = s;
  __syncthreads();
  if (threadIdx.x >= 8) return;
  s = 0.f;
#pragma unroll
  for (int r = 0; r < 32; ++r) s += sums[r][threadIdx.x];
  float* to = c < dh ? dq : dk;
  if (to) to[c < dh ? c : c - dh] = s;
}

// ---- host ----------------------------------------------------------------------------------
bool bad(const void* p, uintptr_t to) { return !p || ((uintptr_t)p & (to - 1)); }
bool bad_pitch(int64_t ld, int64_t cols) { return ld < cols || ld % 8 || ld > (1 << 24); }
bool bad_matrix(const void* p, int64_t ld, int64_t cols) { return bad(p, 16) || bad_pitch(ld, cols); }

bool sizes_ok(int64_t B, int64_t S, int64_t H, int64_t Hkv, int64_t dh) {
  if (B < 1 || S < 1 || H < 0 || Hkv < 0 || H + Hkv < 1 || (dh != 64 && dh != 128)) return false;
  return B <= (1 << 20) && S <= (1 << 24) && B * S <= (1 << 30) && H <= (1 << 12) && Hkv <= (1 << 12);
}

// Tokens of a workgroup: up to 1536 items of 16 columns, fewer while that leaves less than 2048 workgroups.
int tokens_each(int64_t tokens, int64_t items) {
  int64_t w = 1536 / items;
  if (w > tokens / 2048) w = tokens / 2048;
  return (int)(w < 1 ? 1 : w > kMostTokens ? kMostTokens : w);
}

rv_status common(const rv_rotary_desc* d, RotArgs& a) {
  if (!d || !sizes_ok(d->B, d->S, d->n_heads, d->n_kv_heads, d->d_head)) return RV_E_INVAL;
  if (d->rot < 0 || d->rot > d->d_head || d->rot % 16 || (d->layout != RV_ROT_HALF && d->layout != RV_ROT_PAIRS)) return RV_E_INVAL;
  if (d->rot && bad(d->freq, 8)) return RV_E_INVAL;
  if (!(fabsf(d->amplitude) <= 3e38f) || !(d->eps >= 0.f) || !(d->eps <= 3e38f)) return RV_E_INVAL;
  if (((uintptr_t)d->pos | (uintptr_t)d->start | (uintptr_t)d->length) & 3) return RV_E_INVAL;
  if (((uintptr_t)d->gamma_q | (uintptr_t)d->gamma_k) & 15) return RV_E_INVAL;
  a = RotArgs{};
  a.gamma_q = (const uint16_t*)d->gamma_q; a.gamma_k = (const uint16_t*)d->gamma_k;
  a.freq = d->freq; a.pos = d->pos; a.start = d->start; a.length = d->length;
  a.tokens = (int64_t)d->B * d->S;
  a.S = d->S; a.H = d->n_heads; a.Hkv = d->n_kv_heads; a.rot = d->rot;
  a.amplitude = d->amplitude; a.eps = d->eps;
  return RV_OK;
}
void deal(RotArgs& a, int dh) {
  const int items = a.heads * (dh / 16);
  a.tw = tokens_each(a.tokens, items);
  a.per_token = 1.0f / (float)items;
}

template <int L, bool PAIRS>
rv_status forward(const RotArgs& a, hipStream_t st) {
  const int64_t groups = (a.tokens + a.tw - 1) / a.tw;
  hipLaunchKernelGGL((rotary_fwd_kernel<L, PAIRS>), dim3((unsigned)(groups < (1 << 20) ? groups : 1 << 20)), dim3(256), 0, st, a);
  return rv_launch_status();
}
template <int L, bool PAIRS>
rv_status backward(const RotArgs& a, float* dgamma_q, float* dgamma_k, hipStream_t st) {
  const int64_t groups = (a.tokens + a.tw - 1) / a.tw, most = a.part ? kGammaGroups : 1 << 20;
  const int grid = (int)(groups < most ? groups : most);
  if (a.gamma_q || a.gamma_k) hipLaunchKernelGGL((rotary_bwd_kernel<L, PAIRS, true>), dim3(grid), dim3(256), 0, st, a);
  else hipLaunchKernelGGL((rotary_bwd_kernel<L, PAIRS, false>), dim3(grid), dim3(256), 0, st, a);
  RV_TRY(rv_launch_status());
  if (!a.part) return RV_OK;
  hipLaunchKernelGGL(rotary_gamma_kernel, dim3(2 * 16 * L / 8), dim3(256), 0, st, a.part, grid, 16 * L, dgamma_q, dgamma_k);
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
  a.tokens = (int64_t)B * S; a.heads = n_heads + n_kv_heads;
  deal(a, d_head);
  const int64_t groups = (a.tokens + a.tw - 1) / a.tw;
  *bytes = (size_t)(groups < kGammaGroups ? groups : kGammaGroups) * 2 * d_head * 4;
  return RV_OK;
}

extern "C" rv_status rv_k_rotary_fwd(const rv_rotary_desc* d) {
  RotArgs a;
  RV_TRY(common(d, a));
  const int64_t cols = (int64_t)a.H * d->d_head, kcols = (int64_t)a.Hkv * d->d_head;
  if (a.H && (bad_matrix(d->q, d->ldq, cols) || bad_matrix(d->q_out, d->ldq_out, cols))) return RV_E_INVAL;
  if (a.Hkv && (bad_matrix(d->k, d->ldk, kcols) || bad_matrix(d->k_out, d->ldk_out, kcols))) return RV_E_INVAL;
  if (d->v && (!a.Hkv || bad_matrix(d->v, d->ldv, kcols) || bad_matrix(d->v_out, d->ldv_out, kcols))) return RV_E_INVAL;
  if (d->rows < 0 || d->rows > (1 << 24) || d->sinks < 0 || (d->rows && !a.Hkv)) return RV_E_INVAL;
  a.rows = d->rows;
  a.sinks = d->sinks < d->rows ? d->sinks : d->rows - 1;
  a.q = (const uint16_t*)d->q; a.ldq = d->ldq; a.q_out = (uint16_t*)d->q_out; a.ldq_out = d->ldq_out;
  a.k = (const uint16_t*)d->k; a.ldk = d->ldk; a.k_out = (uint16_t*)d->k_out; a.ldk_out = d->ldk_out;
  a.v = (const uint16_t*)d->v; a.ldv = d->ldv; a.v_out = (uint16_t*)d->v_out; a.ldv_out = d->ldv_out;
  a.heads = a.H + a.Hkv + (d->v ? a.Hkv : 0);
  deal(a, d->d_head);
  const hipStream_t st = (hipStream_t)d->stream;
  if (d->d_head == 64) return d->layout == RV_ROT_PAIRS ? forward<4, true>(a, st) : forward<4, false>(a, st);
  return d->layout == RV_ROT_PAIRS ? forward<8, true>(a, st) : forward<8, false>(a, st);
}

extern "C" rv_status rv_k_rotary_bwd(const rv_rotary_desc* d) {
  RotArgs a;
  RV_TRY(common(d, a));
  if (!a.H) a.gamma_q = nullptr;
  if (!a.Hkv) a.gamma_k = nullptr;
  const int64_t cols = (int64_t)a.H * d->d_head, kcols = (int64_t)a.Hkv * d->d_head;
  if (a.H && (bad_matrix(d->dq_out, d->lddq_out, cols) || bad_matrix(d->dq, d->lddq, cols))) return RV_E_INVAL;
  if (a.Hkv && (bad_matrix(d->dk_out, d->lddk_out, kcols) || bad_matrix(d->dk, d->lddk, kcols))) return RV_E_INVAL;
  if (a.gamma_q && (bad_matrix(d->q, d->ldq, cols) || ((uintptr_t)d->dgamma_q & 3))) return RV_E_INVAL;
  if (a.gamma_k && (bad_matrix(d->k, d->ldk, kcols) || ((uintptr_t)d->dgamma_k & 3))) return RV_E_INVAL;
  if ((d->dgamma_q && !a.gamma_q) || (d->dgamma_k && !a.gamma_k)) return RV_E_INVAL;
  a.q = (const uint16_t*)d->q; a.ldq = d->ldq; a.gq = (const uint16_t*)d->dq_out; a.ldgq = d->lddq_out; a.q_out = (uint16_t*)d->dq; a.ldq_out = d->lddq;
  a.k = (const uint16_t*)d->k; a.ldk = d->ldk; a.gk = (const uint16_t*)d->dk_out; a.ldgk = d->lddk_out; a.k_out = (uint16_t*)d->dk; a.ldk_out = d->lddk;
  a.heads = a.H + a.Hkv;
  deal(a, d->d_head);
  if (d->dgamma_q || d->dgamma_k) {
    size_t need = 0;
    RV_TRY(rv_k_rotary_work(d->B, d->S, d->n_heads, d->n_kv_heads, d->d_head, &need));
    if (bad(d->work, 256) || d->work_bytes < need) return RV_E_INVAL;
    a.part = (float*)d->work;
  }
  const hipStream_t st = (hipStream_t)d->stream;
  if (d->d_head == 64)
    return d->layout == RV_ROT_PAIRS ? backward<4, true>(a, d->dgamma_q, d->dgamma_k, st) : backward<4, false>(a, d->dgamma_q, d->dgamma_k, st);
  return d->layout == RV_ROT_PAIRS ? backward<8, true>(a, d->dgamma_q, d->dgamma_k, st) : backward<8, false>(a, d->dgamma_q, d->dgamma_k, st);
}
